// Weight gradients from codes: dh (+)= sum over rows r of y[r, i] d[r, j]. The scales of both operands change along the reduction (a
// scale belongs to a row), so they cannot be applied to sums; code times scale is a bf16 number exactly, and the products are formed
// on the bf16 matrix units from those: nothing is rounded before the fp32 accumulators.
// Codes are turned into bf16 on their way into LDS (v_cvt_scalef32_pk_bf16_fp8, which applies the scale), where they lie as in memory, and
// are transposed when they are read (ds_read_b64_tr_b16 hands lane i of a group of 16 the i-th column of a 4 x 16 block). Row pitch: 64
// bytes more than a multiple of 256, so that the four rows of such a block start in four different quarters of the banks.
// The rows are cut into slabs, one workgroup per slab and tile; the slabs' sums are added by a second launch in one order.
#include <algorithm>

#include "codes_device.h"
#include "varco_scaled.h"

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kTile = 128;           // inputs and outputs of a tile; a wavefront takes 64 x 64
constexpr int BK = 32;               // rows of a stage
constexpr int kPitch = kTile * 2 + 64;

// Sixteen codes as bf16.
__device__ __forceinline__ void to_bf16(const uint4& q, float scale, uint4 (&out)[2]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    uint32_t o[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false));
        o[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true));
    }
    out[0] = make_uint4(o[0], o[1], o[2], o[3]), out[1] = make_uint4(o[4], o[5], o[6], o[7]);
}

// Fragment of 16 columns x 32 rows whose first column's element of row 0 (this lane's share of the block) is at LDS byte `at`.
__device__ __forceinline__ bf16x8 fragment(uint32_t at) {
    using P = __attribute__((address_space(3))) shortx4*;
    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)at);
    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(at + 4 * kPitch));
    return __builtin_bit_cast(bf16x8, shortx8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
}

__global__ __launch_bounds__(kThreads) void scaled_tn_kernel(ScaledWeightArgs a, int32_t split, int64_t rows_per_split) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * BK * kPitch];
    const int32_t i0 = int32_t(blockIdx.y) * kTile, j0 = int32_t(blockIdx.z) * kTile;
    const int64_t r0 = int64_t(blockIdx.x) * rows_per_split, r1 = min(a.n_rows, r0 + rows_per_split);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wi = (wave >> 1) * 64, wj = (wave & 1) * 64;
    floatx4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = floatx4(0.f);
    const uint32_t base = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)lds));
    const uint32_t row = 8 * (lane >> 4) + ((lane >> 2) & 3), sub = 8 * (lane & 3);
    const uint32_t at_y = base + row * kPitch + sub + wi * 2, at_d = base + BK * kPitch + row * kPitch + sub + wj * 2;

    // a stage of 32 rows has 8 pieces of 16 codes per row and operand: one per thread
    const int tr = threadIdx.x >> 3, tp = threadIdx.x & 7;
    auto load = [&](const uint8_t* codes, const uint8_t* scales, int32_t width, int32_t c0, int64_t r, uint4& q, float& scale) {
        const int64_t ld = code_ld(width);
        const int32_t c = c0 + 16 * tp;
        q = make_uint4(0u, 0u, 0u, 0u), scale = 1.f;
        if (r >= r1 || c >= ld) return;
        q = *reinterpret_cast<const uint4*>(codes + r * ld + c);
        const uint32_t s = scales[r * scale_ld(width) + c0 / kCodeBlock];
        scale = __uint_as_float(s ? s << 23 : 0x400000u);
    };
    for (int64_t r = r0; r < r1; r += BK) {
        uint4 qy, qd, out[2];
        float sy, sd;
        load(a.y, a.y_scales, a.n_in, i0, r + tr, qy, sy);
        load(a.d, a.d_scales, a.n_out, j0, r + tr, qd, sd);
        __syncthreads();
        to_bf16(qy, sy, out);
        uint4* p = reinterpret_cast<uint4*>(lds + tr * kPitch + tp * 32);
        p[0] = out[0], p[1] = out[1];
        to_bf16(qd, sd, out);
        p = reinterpret_cast<uint4*>(lds + (BK + tr) * kPitch + tp * 32);
        p[0] = out[0], p[1] = out[1];
        __syncthreads();
        bf16x8 fd[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) fd[j] = fragment(at_d + j * 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16x8 fy = fragment(at_y + i * 32);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fy, fd[j], acc[i][j], 0, 0, 0);
        }
    }
    // accumulator v of a lane is element (4 (lane / 16) + v, lane % 16)
    float* const out = split > 1 ? a.partial + int64_t(blockIdx.x) * a.n_in * a.n_out : a.dh;
    const int64_t ldo = split > 1 ? a.n_out : a.ldh;
    const bool add = split == 1 && a.accumulate;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int32_t ri = i0 + wi + 16 * i + 4 * (lane >> 4) + v, cj = j0 + wj + 16 * j + (lane & 15);
                if (ri < a.n_in && cj < a.n_out) {
                    float* const p = out + int64_t(ri) * ldo + cj;
                    *p = add ? *p + acc[i][j][v] : acc[i][j][v];
                }
            }
}

// dh (+)= the slabs' sums, slab 0 first.
__global__ __launch_bounds__(kThreads) void slab_sum_kernel(const float* __restrict__ partial, int32_t split, int32_t n_in, int32_t n_out, float* dh,
                                                            int64_t ldh, int32_t accumulate) {
    const int64_t n = int64_t(n_in) * n_out;
    for (int64_t e = int64_t(blockIdx.x) * kThreads + threadIdx.x; e < n; e += int64_t(gridDim.x) * kThreads) {
        float x = 0.f;
        for (int32_t s = 0; s < split; ++s) x += partial[s * n + e];
        const int64_t i = e / n_out;
        float* const p = dh + i * ldh + (e - i * n_out);
        *p = accumulate ? *p + x : x;
    }
}

int64_t slab_rows(int64_t n_rows, int64_t split) { return std::max<int64_t>(1, ((n_rows + split - 1) / split + BK - 1) / BK) * BK; }

}  // namespace

int32_t varco_scaled_weight_split(int64_t n_rows, int32_t n_in, int32_t n_out) {
    const int64_t tiles = int64_t((n_in + kTile - 1) / kTile) * ((n_out + kTile - 1) / kTile);
    const int64_t split = std::max<int64_t>(1, std::min<int64_t>(512 / tiles, n_rows / 256));
    const int64_t rows = slab_rows(n_rows, split);
    return int32_t(std::max<int64_t>(1, (n_rows + rows - 1) / rows));
}

hipError_t varco_launch_scaled_bwd_weight(const ScaledWeightArgs& a, hipStream_t stream) {
    const int32_t split = varco_scaled_weight_split(a.n_rows, a.n_in, a.n_out);
    const int64_t rows = slab_rows(a.n_rows, split);
    const dim3 grid{unsigned(split), unsigned((a.n_in + kTile - 1) / kTile), unsigned((a.n_out + kTile - 1) / kTile)};
    hipLaunchKernelGGL(scaled_tn_kernel, grid, dim3(kThreads), 0, stream, a, split, rows);
    if (split > 1) {
        const int64_t n = int64_t(a.n_in) * a.n_out;
        hipLaunchKernelGGL(slab_sum_kernel, dim3(unsigned(std::min<int64_t>((n + kThreads - 1) / kThreads, 2048))), dim3(kThreads), 0, stream, a.partial, split,
                           a.n_in, a.n_out, a.dh, a.ldh, a.accumulate);
    }
    return hipGetLastError();
}
