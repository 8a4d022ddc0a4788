// Entry points of normalised rows, 8-bit codes and their products, and limited gradient steps: argument checks in front of
// the launchers of varco_scaled.h. They belong to no context and hold no state.
#include "varco_scaled.h"

#include <cmath>
#include <initializer_list>
#include <string>

#include "codes_device.h"
#include "varco_internal.h"

namespace {

int32_t refuse(int32_t code, const char* fn, const char* what) noexcept {
    try {
        return varco_fail(nullptr, code, (std::string(fn) + ": " + what).c_str());
    } catch (...) {
        return code;
    }
}
int32_t result(hipError_t e, const char* fn) noexcept { return e == hipSuccess ? VARCO_OK : refuse(VARCO_ERR_HIP, fn, hipGetErrorString(e)); }

bool at_multiple(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
int32_t check_type(int32_t dtype, const char* fn) {
    return dtype == VARCO_F32 || dtype == VARCO_BF16 ? VARCO_OK : refuse(VARCO_ERR_UNSUPPORTED, fn, "dtype is neither VARCO_F32 nor VARCO_BF16");
}
uintptr_t element(int32_t dtype) { return dtype == VARCO_BF16 ? 2 : 4; }
int32_t check_rows(int64_t n_rows, const char* fn) {
    return n_rows >= 0 && n_rows <= INT32_MAX ? VARCO_OK : refuse(VARCO_ERR_SHAPE, fn, "row count out of range");
}
int32_t check_width(int32_t width, const char* fn) {
    return width >= 1 && width <= VARCO_MAX_CODE_WIDTH ? VARCO_OK : refuse(VARCO_ERR_SHAPE, fn, "width out of range");
}
// A matrix argument: NULL where it may be, else at an address of its elements and with rows that do not overlap.
int32_t check_matrix(const void* p, int64_t ld, int32_t width, uintptr_t bytes, bool required, const char* fn) {
    if (!p) return required ? refuse(VARCO_ERR_INVALID_ARG, fn, "null pointer") : VARCO_OK;
    if (!at_multiple(p, bytes)) return refuse(VARCO_ERR_INVALID_ARG, fn, "a pointer that is no address of its elements");
    if (ld < width) return refuse(VARCO_ERR_SHAPE, fn, "leading dimension smaller than the width");
    return VARCO_OK;
}
// Rows in memory: n of `bytes` bytes, `step` bytes apart.
struct Rows {
    const void* at;
    int64_t n, bytes, step;
};
Rows rows_of(const void* p, int64_t n, int64_t ld, int64_t width, uintptr_t element) {
    return {p, n, width * int64_t(element), (n > 1 ? ld : width) * int64_t(element)};
}
Rows whole(const void* p, int64_t bytes) { return {p, 1, bytes, bytes}; }
// Whether a byte of a is one of b. Rows as far apart (columns of one wider matrix, say) and a single row are compared row by row, others by where they begin
// and end.
bool overlap(const Rows& a, const Rows& b) {
    if (!a.at || !b.at || a.n < 1 || b.n < 1 || a.bytes < 1 || b.bytes < 1) return false;
    if (a.n > 1 && (b.n == 1 || reinterpret_cast<uintptr_t>(b.at) < reinterpret_cast<uintptr_t>(a.at))) return overlap(b, a);
    const uintptr_t start = reinterpret_cast<uintptr_t>(a.at), other = reinterpret_cast<uintptr_t>(b.at);
    if (a.n == 1) {                              // the first row of b that ends behind a's start has to begin before a's end
        const int64_t k = start < other + b.bytes ? 0 : int64_t(start - other - b.bytes) / b.step + 1;
        return k < b.n && other + k * b.step < start + a.bytes;
    }
    if (other >= start + (a.n - 1) * a.step + a.bytes) return false;
    if (a.step != b.step) return true;
    const int64_t k = int64_t(other - start) / a.step, into = int64_t(other - start) % a.step;       // b begins in row k of a, or behind it
    return (k < a.n && into < a.bytes) || (k + 1 < a.n && a.step - into < b.bytes);
}
// What is written, against what is read: nothing of one may be the other's, but for all the rows themselves where `in_place`.
int32_t check_written(const Rows& written, std::initializer_list<Rows> read, bool in_place, const char* fn) {
    for (const Rows& r : read)
        if (overlap(written, r) && !(in_place && written.at == r.at && written.step == r.step))
            return refuse(VARCO_ERR_INVALID_ARG, fn, "an output overlaps what the call reads or another output");
    return VARCO_OK;
}
int32_t check_codes(const void* codes, const void* scales, bool required, const char* fn) {
    if (!codes && !scales && !required) return VARCO_OK;
    if (!codes || !scales) return refuse(VARCO_ERR_INVALID_ARG, fn, "null codes or scales");
    if (!at_multiple(codes, 16) || !at_multiple(scales, 4))
        return refuse(VARCO_ERR_INVALID_ARG, fn, "codes start at a multiple of 16 bytes, scales at one of 4");
    return VARCO_OK;
}
int32_t check_workspace(const void* workspace, int64_t have, int64_t need, const char* fn) {
    if (have < need || (need > 0 && !workspace)) return refuse(VARCO_ERR_STATE, fn, "the workspace is too small");
    return at_multiple(workspace, 256) ? VARCO_OK : refuse(VARCO_ERR_INVALID_ARG, fn, "the workspace is not 256-byte aligned");
}
int32_t check_tensors(int32_t n_tensors, std::initializer_list<const void* const*> lists, const int64_t* sizes, uintptr_t bytes, const char* fn) {
    if (n_tensors < 0) return refuse(VARCO_ERR_SHAPE, fn, "negative count of tensors");
    if (n_tensors > 1 << 20) return refuse(VARCO_ERR_SHAPE, fn, "more than 2^20 tensors");
    if (n_tensors == 0) return VARCO_OK;
    if (!sizes) return refuse(VARCO_ERR_INVALID_ARG, fn, "null array");
    int64_t total = 0;
    for (int32_t i = 0; i < n_tensors; ++i) {
        if (sizes[i] < 0 || sizes[i] > (int64_t(1) << 42)) return refuse(VARCO_ERR_SHAPE, fn, "element count of a tensor out of range");
        if ((total += sizes[i]) > (int64_t(1) << 42)) return refuse(VARCO_ERR_SHAPE, fn, "more than 2^42 elements");
    }
    for (const void* const* list : lists) {
        if (!list) return refuse(VARCO_ERR_INVALID_ARG, fn, "null array");
        for (int32_t i = 0; i < n_tensors; ++i)
            if (sizes[i] && (!list[i] || !at_multiple(list[i], bytes)))
                return refuse(VARCO_ERR_INVALID_ARG, fn, "a tensor that is null or at no address of its elements");
    }
    return VARCO_OK;
}
int32_t check_limit(float max_norm, const void* out, const char* fn) {
    if (!(max_norm >= 0.f)) return refuse(VARCO_ERR_INVALID_ARG, fn, "max_norm is negative or NaN");
    if (!out || !at_multiple(out, 4)) return refuse(VARCO_ERR_INVALID_ARG, fn, "out is null or at no address of a float");
    return VARCO_OK;
}
int64_t norm_bytes(int32_t dtype, int64_t n_rows, int32_t width) {
    const int32_t blocks = varco_norm_blocks(dtype, n_rows, width);
    return blocks > 1 ? int64_t(blocks) * width * 4 : 0;
}
}  // namespace

#define VARCO_CHECK(call)            \
    do {                             \
        if (int32_t rc_ = (call)) return rc_; \
    } while (0)

extern "C" int32_t varco_quantize_rows(int32_t dtype, int64_t n_rows, int32_t width, const void* x, int64_t ldx, const void* gate, int64_t ldg,
                                       void* codes, void* scales, varco_stream stream) {
    const char* const fn = "varco_quantize_rows";
    VARCO_CHECK(check_type(dtype, fn));
    VARCO_CHECK(check_rows(n_rows, fn));
    VARCO_CHECK(check_width(width, fn));
    if (n_rows == 0) return VARCO_OK;
    VARCO_CHECK(check_matrix(x, ldx, width, element(dtype), true, fn));
    VARCO_CHECK(check_matrix(gate, ldg, width, element(dtype), false, fn));
    VARCO_CHECK(check_codes(codes, scales, true, fn));
    const Rows code_rows = whole(codes, n_rows * code_ld(width)), scale_rows = whole(scales, n_rows * scale_ld(width));
    const Rows from = rows_of(x, n_rows, ldx, width, element(dtype)), by = rows_of(gate, n_rows, ldg, width, element(dtype));
    VARCO_CHECK(check_written(code_rows, {from, by, scale_rows}, false, fn));
    VARCO_CHECK(check_written(scale_rows, {from, by}, false, fn));
    return result(varco_launch_quantize_rows(dtype, n_rows, width, x, ldx, gate, ldg, static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales),
                                             static_cast<hipStream_t>(stream)), fn);
}

extern "C" int32_t varco_quantize_weights(int32_t n_in, int32_t n_out, const void* h, int64_t ldh, void* turned, void* turned_scales, void* codes,
                                          void* scales, varco_stream stream) {
    const char* const fn = "varco_quantize_weights";
    VARCO_CHECK(check_width(n_in, fn));
    VARCO_CHECK(check_width(n_out, fn));
    VARCO_CHECK(check_matrix(h, ldh, n_out, 4, true, fn));
    VARCO_CHECK(check_codes(turned, turned_scales, false, fn));
    VARCO_CHECK(check_codes(codes, scales, !turned, fn));
    const Rows from = rows_of(h, n_in, ldh, n_out, 4);
    const auto blocks = [](int64_t n) { return (n + kCodeBlock - 1) / kCodeBlock; };
    const Rows written[] = {whole(turned, n_out * code_ld(n_in)), whole(turned_scales, blocks(n_out) * scale_ld(n_in)), whole(codes, n_in * code_ld(n_out)),
                            whole(scales, blocks(n_in) * scale_ld(n_out))};
    for (int i = 0; i < 4; ++i) {
        VARCO_CHECK(check_written(written[i], {from}, false, fn));
        for (int j = 0; j < i; ++j) VARCO_CHECK(check_written(written[i], {written[j]}, false, fn));
    }
    return result(varco_launch_quantize_weights(n_in, n_out, static_cast<const float*>(h), ldh, static_cast<uint8_t*>(turned),
                                                static_cast<uint8_t*>(turned_scales), static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales),
                                                static_cast<hipStream_t>(stream)), fn);
}

extern "C" int32_t varco_scaled_transform(int32_t dtype, int64_t n_rows, int32_t n_in, int32_t n_out, const void* codes, const void* scales,
                                          const void* w_codes, const void* w_scales, void* c, int64_t ldc, int32_t accumulate, int32_t act,
                                          varco_stream stream) {
    const char* const fn = "varco_scaled_transform";
    VARCO_CHECK(check_type(dtype, fn));
    VARCO_CHECK(check_rows(n_rows, fn));
    VARCO_CHECK(check_width(n_in, fn));
    VARCO_CHECK(check_width(n_out, fn));
    if (act != VARCO_ACT_IDENTITY && act != VARCO_ACT_RELU) return refuse(VARCO_ERR_INVALID_ARG, fn, "unknown activation");
    if (n_rows == 0) return VARCO_OK;
    VARCO_CHECK(check_codes(codes, scales, true, fn));
    VARCO_CHECK(check_codes(w_codes, w_scales, true, fn));
    VARCO_CHECK(check_matrix(c, ldc, n_out, element(dtype), true, fn));
    VARCO_CHECK(check_written(rows_of(c, n_rows, ldc, n_out, element(dtype)),
                              {whole(codes, n_rows * code_ld(n_in)), whole(scales, n_rows * scale_ld(n_in)), whole(w_codes, n_out * code_ld(n_in)),
                               whole(w_scales, (n_out + kCodeBlock - 1) / kCodeBlock * scale_ld(n_in))}, false, fn));
    ScaledArgs a;
    a.n_rows = n_rows, a.n_in = n_in, a.n_out = n_out;
    a.x = static_cast<const uint8_t*>(codes), a.x_scales = static_cast<const uint8_t*>(scales);
    a.w = static_cast<const uint8_t*>(w_codes), a.w_scales = static_cast<const uint8_t*>(w_scales);
    a.c = c, a.ldc = ldc, a.accumulate = accumulate != 0, a.relu = act == VARCO_ACT_RELU;
    return result(varco_launch_scaled_transform(dtype, a, static_cast<hipStream_t>(stream)), fn);
}

extern "C" int32_t varco_scaled_weight_workspace(int64_t n_rows, int32_t n_in, int32_t n_out, int64_t* bytes) {
    const char* const fn = "varco_scaled_weight_workspace";
    if (!bytes) return refuse(VARCO_ERR_INVALID_ARG, fn, "null output");
    VARCO_CHECK(check_rows(n_rows, fn));
    VARCO_CHECK(check_width(n_in, fn));
    VARCO_CHECK(check_width(n_out, fn));
    *bytes = varco_scaled_weight_floats(n_rows, n_in, n_out) * 4;
    return VARCO_OK;
}

extern "C" int32_t varco_scaled_bwd_weight(int64_t n_rows, int32_t n_in, int32_t n_out, const void* y_codes, const void* y_scales,
                                           const void* d_codes, const void* d_scales, void* dh, int64_t ldh, int32_t accumulate, void* workspace,
                                           int64_t workspace_bytes, varco_stream stream) {
    const char* const fn = "varco_scaled_bwd_weight";
    VARCO_CHECK(check_rows(n_rows, fn));
    VARCO_CHECK(check_width(n_in, fn));
    VARCO_CHECK(check_width(n_out, fn));
    VARCO_CHECK(check_matrix(dh, ldh, n_out, 4, true, fn));
    if (n_rows > 0) {
        VARCO_CHECK(check_codes(y_codes, y_scales, true, fn));
        VARCO_CHECK(check_codes(d_codes, d_scales, true, fn));
    }
    VARCO_CHECK(check_workspace(workspace, workspace_bytes, varco_scaled_weight_floats(n_rows, n_in, n_out) * 4, fn));
    VARCO_CHECK(check_written(rows_of(dh, n_in, ldh, n_out, 4), {whole(y_codes, n_rows * code_ld(n_in)), whole(y_scales, n_rows * scale_ld(n_in)),
                                                                 whole(d_codes, n_rows * code_ld(n_out)), whole(d_scales, n_rows * scale_ld(n_out))}, false, fn));
    ScaledWeightArgs a;
    a.n_rows = n_rows, a.n_in = n_in, a.n_out = n_out;
    a.y = static_cast<const uint8_t*>(y_codes), a.y_scales = static_cast<const uint8_t*>(y_scales);
    a.d = static_cast<const uint8_t*>(d_codes), a.d_scales = static_cast<const uint8_t*>(d_scales);
    a.dh = static_cast<float*>(dh), a.ldh = ldh, a.accumulate = accumulate != 0, a.partial = static_cast<float*>(workspace);
    return result(varco_launch_scaled_bwd_weight(a, static_cast<hipStream_t>(stream)), fn);
}

extern "C" int32_t varco_rms_norm_fwd(int32_t dtype, int64_t n_rows, int32_t width, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                                      const void* gain, float eps, void* total, int64_t ldt, void* y, int64_t ldy, void* codes, void* scales,
                                      void* inv_rms, varco_stream stream) {
    const char* const fn = "varco_rms_norm_fwd";
    VARCO_CHECK(check_type(dtype, fn));
    VARCO_CHECK(check_rows(n_rows, fn));
    VARCO_CHECK(check_width(width, fn));
    if (!(eps >= 0.f) || std::isinf(eps)) return refuse(VARCO_ERR_INVALID_ARG, fn, "eps is negative or not finite");
    if (n_rows == 0) return VARCO_OK;
    const uintptr_t e = element(dtype);
    VARCO_CHECK(check_matrix(x, ldx, width, e, true, fn));
    VARCO_CHECK(check_matrix(residual, ldr, width, e, false, fn));
    VARCO_CHECK(check_matrix(gain, width, width, 4, false, fn));
    VARCO_CHECK(check_matrix(total, ldt, width, e, false, fn));
    VARCO_CHECK(check_matrix(y, ldy, width, e, false, fn));
    VARCO_CHECK(check_matrix(inv_rms, 1, 1, 4, false, fn));
    VARCO_CHECK(check_codes(codes, scales, false, fn));
    if (!total && !y && !codes && !inv_rms) return refuse(VARCO_ERR_INVALID_ARG, fn, "no output");
    if (total && total == y) return refuse(VARCO_ERR_INVALID_ARG, fn, "total and y are the same memory");
    const Rows from = rows_of(x, n_rows, ldx, width, e), added = rows_of(residual, n_rows, ldr, width, e);
    const Rows sum = rows_of(total, n_rows, ldt, width, e), normal = rows_of(y, n_rows, ldy, width, e);
    VARCO_CHECK(check_written(sum, {from, added}, true, fn));
    VARCO_CHECK(check_written(normal, {from, added}, true, fn));
    VARCO_CHECK(check_written(normal, {sum}, false, fn));
    if (codes) {
        const Rows code_rows = whole(codes, n_rows * code_ld(width)), scale_rows = whole(scales, n_rows * scale_ld(width));
        VARCO_CHECK(check_written(code_rows, {from, added, sum, normal, scale_rows}, false, fn));
        VARCO_CHECK(check_written(scale_rows, {from, added, sum, normal}, false, fn));
    }
    NormFwdArgs a;
    a.n_rows = n_rows, a.width = width;
    a.x = x, a.ldx = ldx, a.residual = residual, a.ldr = ldr;
    a.gain = static_cast<const float*>(gain), a.eps = eps;
    a.total = total, a.ldt = ldt, a.y = y, a.ldy = ldy;
    a.codes = static_cast<uint8_t*>(codes), a.scales = static_cast<uint8_t*>(scales), a.inv_rms = static_cast<float*>(inv_rms);
    return result(varco_launch_rms_norm_fwd(dtype, a, static_cast<hipStream_t>(stream)), fn);
}

extern "C" int32_t varco_rms_norm_workspace(int32_t dtype, int64_t n_rows, int32_t width, int64_t* bytes) {
    const char* const fn = "varco_rms_norm_workspace";
    if (!bytes) return refuse(VARCO_ERR_INVALID_ARG, fn, "null output");
    VARCO_CHECK(check_type(dtype, fn));
    VARCO_CHECK(check_rows(n_rows, fn));
    VARCO_CHECK(check_width(width, fn));
    *bytes = norm_bytes(dtype, n_rows, width);
    return VARCO_OK;
}

extern "C" int32_t varco_rms_norm_bwd(int32_t dtype, int64_t n_rows, int32_t width, const void* dy, int64_t lddy, const void* u, int64_t ldu,
                                      const void* gain, const void* inv_rms, const void* dtotal, int64_t lddt, void* dx, int64_t lddx, void* dgain,
                                      int32_t accumulate, void* workspace, int64_t workspace_bytes, varco_stream stream) {
    const char* const fn = "varco_rms_norm_bwd";
    VARCO_CHECK(check_type(dtype, fn));
    VARCO_CHECK(check_rows(n_rows, fn));
    VARCO_CHECK(check_width(width, fn));
    const uintptr_t e = element(dtype);
    if (n_rows > 0) {
        VARCO_CHECK(check_matrix(dy, lddy, width, e, true, fn));
        VARCO_CHECK(check_matrix(u, ldu, width, e, true, fn));
        VARCO_CHECK(check_matrix(inv_rms, 1, 1, 4, true, fn));
        VARCO_CHECK(check_matrix(dtotal, lddt, width, e, false, fn));
        VARCO_CHECK(check_matrix(dx, lddx, width, e, false, fn));
    }
    VARCO_CHECK(check_matrix(gain, width, width, 4, false, fn));
    VARCO_CHECK(check_matrix(dgain, width, width, 4, false, fn));
    if (!dx && !dgain) return n_rows == 0 ? VARCO_OK : refuse(VARCO_ERR_INVALID_ARG, fn, "no output");
    if (dgain) VARCO_CHECK(check_workspace(workspace, workspace_bytes, norm_bytes(dtype, n_rows, width), fn));
    VARCO_CHECK(check_written(rows_of(dx, n_rows, lddx, width, e), {rows_of(dy, n_rows, lddy, width, e), rows_of(u, n_rows, ldu, width, e),
                                                                     rows_of(dtotal, n_rows, lddt, width, e)}, true, fn));
    NormBwdArgs a;
    a.n_rows = n_rows, a.width = width;
    a.dy = dy, a.lddy = lddy, a.u = u, a.ldu = ldu;
    a.gain = static_cast<const float*>(gain), a.inv_rms = static_cast<const float*>(inv_rms);
    a.dtotal = dtotal, a.lddt = lddt, a.dx = dx, a.lddx = lddx;
    a.dgain = static_cast<float*>(dgain), a.accumulate = accumulate != 0, a.partial = static_cast<float*>(workspace);
    return result(varco_launch_rms_norm_bwd(dtype, a, static_cast<hipStream_t>(stream)), fn);
}

extern "C" int32_t varco_gradient_norm_workspace(int32_t n_tensors, const int64_t* sizes, int64_t* bytes) {
    const char* const fn = "varco_gradient_norm_workspace";
    if (!bytes) return refuse(VARCO_ERR_INVALID_ARG, fn, "null output");
    VARCO_CHECK(check_tensors(n_tensors, {}, sizes, 1, fn));
    *bytes = int64_t(varco_clip_partials(n_tensors, sizes)) * 8;
    return VARCO_OK;
}

extern "C" int32_t varco_gradient_norm(int32_t dtype, int32_t n_tensors, const void* const* grads, const int64_t* sizes, float max_norm, void* out,
                                       void* workspace, int64_t workspace_bytes, varco_stream stream) {
    const char* const fn = "varco_gradient_norm";
    VARCO_CHECK(check_type(dtype, fn));
    VARCO_CHECK(check_tensors(n_tensors, {grads}, sizes, element(dtype), fn));
    VARCO_CHECK(check_limit(max_norm, out, fn));
    const int32_t n = varco_clip_partials(n_tensors, sizes);
    VARCO_CHECK(check_workspace(workspace, workspace_bytes, int64_t(n) * 8, fn));
    hipStream_t st = static_cast<hipStream_t>(stream);
    double* const partial = static_cast<double*>(workspace);
    VARCO_CHECK(result(varco_launch_square_sums(dtype, n_tensors, grads, sizes, partial, st), fn));
    return result(varco_launch_norm_out(partial, n, max_norm, static_cast<float*>(out), st), fn);
}

extern "C" int32_t varco_clip_gradients(int32_t dtype, int32_t n_tensors, const void* const* grads, void* const* into, const int64_t* sizes,
                                        float max_norm, void* out, void* workspace, int64_t workspace_bytes, varco_stream stream) {
    const char* const fn = "varco_clip_gradients";
    VARCO_CHECK(check_type(dtype, fn));
    VARCO_CHECK(check_tensors(n_tensors, {grads, into}, sizes, element(dtype), fn));
    VARCO_CHECK(check_limit(max_norm, out, fn));
    const int32_t n = varco_clip_partials(n_tensors, sizes);
    VARCO_CHECK(check_workspace(workspace, workspace_bytes, int64_t(n) * 8, fn));
    hipStream_t st = static_cast<hipStream_t>(stream);
    double* const partial = static_cast<double*>(workspace);
    if (n == 0) return result(varco_launch_norm_out(partial, 0, max_norm, static_cast<float*>(out), st), fn);      // (no elements)
    VARCO_CHECK(result(varco_launch_square_sums(dtype, n_tensors, grads, sizes, partial, st), fn));
    return result(varco_launch_clip(dtype, n_tensors, grads, into, sizes, partial, n, max_norm, static_cast<float*>(out), st), fn);
}

extern "C" int32_t varco_sgd_step_clipped(int32_t n_tensors, void* const* w, const void* const* dw, const int64_t* sizes, float lr, float max_norm,
                                          void* out, void* workspace, int64_t workspace_bytes, varco_stream stream) {
    const char* const fn = "varco_sgd_step_clipped";
    VARCO_CHECK(check_tensors(n_tensors, {w, dw}, sizes, 4, fn));
    VARCO_CHECK(check_limit(max_norm, out, fn));
    const int32_t n = varco_clip_partials(n_tensors, sizes);
    VARCO_CHECK(check_workspace(workspace, workspace_bytes, int64_t(n) * 8, fn));
    hipStream_t st = static_cast<hipStream_t>(stream);
    double* const partial = static_cast<double*>(workspace);
    if (n == 0) return result(varco_launch_norm_out(partial, 0, max_norm, static_cast<float*>(out), st), fn);
    VARCO_CHECK(result(varco_launch_square_sums(VARCO_F32, n_tensors, dw, sizes, partial, st), fn));
    return result(varco_launch_sgd_clipped(n_tensors, w, dw, sizes, lr, partial, n, max_norm, static_cast<float*>(out), st), fn);
}
