// Rows and weight matrices as 8-bit codes with a power of two as scale for each 128 columns (128 x 128 elements of a weight
// matrix). Elementwise but for the largest size of a block: bound by reading the values once and writing a byte for each.
#include <algorithm>

#include "codes_device.h"
#include "varco_scaled.h"

namespace {

constexpr int kThreads = 256;

// A group of 16 (bf16) or 32 (fp32) lanes takes a block of 128 columns, a piece of 16 bytes per lane, so the block's
// largest element is found without leaving registers. The blocks of a row are numbered through all rows.
template <typename T, bool GATE>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(int64_t n_rows, int32_t width, const T* x, int64_t ldx, const T* gate, int64_t ldg,
                                                                 uint8_t* codes, uint8_t* scales) {
    using Row = RowPiece<T>;
    constexpr int P = Row::P, G = kCodeBlock / P;
    const int32_t blocks = (width + kCodeBlock - 1) / kCodeBlock, slots = int32_t(scale_ld(width));
    const int64_t ldc = code_ld(width), total = n_rows * slots;
    const int t = threadIdx.x & (G - 1);
    for (int64_t i = int64_t(blockIdx.x) * (kThreads / G) + threadIdx.x / G; i < total; i += int64_t(gridDim.x) * (kThreads / G)) {
        const int64_t row = i / slots;
        const int32_t b = int32_t(i - row * slots);
        if (b >= blocks) {                             // the padding of the scales
            if (t == 0) scales[i] = kOneScale;
            continue;
        }
        const int32_t at = b * kCodeBlock + t * P;
        float v[P];
        Row::load(x + row * ldx, at, width, v);
        if constexpr (GATE) {
            float g[P];
            Row::load(gate + row * ldg, at, width, g);
#pragma unroll
            for (int j = 0; j < P; ++j) v[j] = g[j] > 0.f ? v[j] : 0.f;
        }
        float a = 0.f;
#pragma unroll
        for (int j = 0; j < P; ++j) a = fmaxf(a, finite_size(v[j]));
        const int e = code_exponent(lanes_max<G>(a));
        if (at < ldc) Row::store_codes(codes + row * ldc, at, v, code_inverse(e));
        if (t == 0) scales[i] = uint8_t(e + 127);
    }
}

// A workgroup takes 128 x 128 weights: read once, kept in registers until the largest is known, written row-wise and, through LDS, column-wise.
__global__ __launch_bounds__(kThreads) void quantize_weights_kernel(int32_t n_in, int32_t n_out, const float* h, int64_t ldh, uint8_t* turned,
                                                                    uint8_t* turned_scales, uint8_t* codes, uint8_t* scales) {
    __shared__ float largest[kThreads / 64];
    __shared__ uint32_t tile[kCodeBlock][kCodeBlock / 4 + 1];
    const int32_t i0 = int32_t(blockIdx.y) * kCodeBlock, j0 = int32_t(blockIdx.x) * kCodeBlock;
    const int lane = threadIdx.x & 31, first = threadIdx.x >> 5;       // 32 lanes of 4 columns, 8 rows at a time
    float v[16][4];
    float a = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int32_t i = i0 + first + 8 * r;
        if (i < n_in)
            RowPiece<float>::load(h + i * ldh, j0 + 4 * lane, n_out, v[r]);
        else
#pragma unroll
            for (int j = 0; j < 4; ++j) v[r][j] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) a = fmaxf(a, finite_size(v[r][j]));
    }
    a = lanes_max<64>(a);
    if ((threadIdx.x & 63) == 0) largest[threadIdx.x >> 6] = a;
    __syncthreads();
    const int e = code_exponent(fmaxf(fmaxf(largest[0], largest[1]), fmaxf(largest[2], largest[3])));
    const float inverse = code_inverse(e);
    const int64_t ld_in = code_ld(n_in), ld_out = code_ld(n_out);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int32_t row = first + 8 * r;
        const uint32_t q = four_codes(v[r][0], v[r][1], v[r][2], v[r][3], inverse);
        tile[row][lane] = q;
        if (codes && i0 + row < n_in && j0 + 4 * lane < ld_out) *reinterpret_cast<uint32_t*>(codes + (i0 + row) * ld_out + j0 + 4 * lane) = q;
    }
    __syncthreads();
    if (turned) {
        const uint8_t* const bytes = reinterpret_cast<const uint8_t*>(tile);
        constexpr int kPitch = kCodeBlock + 4;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int32_t col = first + 8 * r;
            uint32_t q = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) q |= uint32_t(bytes[(4 * lane + j) * kPitch + col]) << (8 * j);
            if (j0 + col < n_out && i0 + 4 * lane < ld_in) *reinterpret_cast<uint32_t*>(turned + (j0 + col) * ld_in + i0 + 4 * lane) = q;
        }
    }
    if (threadIdx.x == 0) {
        const int64_t s_in = scale_ld(n_in), s_out = scale_ld(n_out);
        auto put = [e](uint8_t* s, int64_t ld, int64_t row, int64_t col, bool last) {
            s[row * ld + col] = uint8_t(e + 127);
            if (last)
                for (int64_t c = col + 1; c < ld; ++c) s[row * ld + c] = kOneScale;
        };
        if (codes) put(scales, s_out, blockIdx.y, blockIdx.x, blockIdx.x + 1 == gridDim.x);
        if (turned) put(turned_scales, s_in, blockIdx.x, blockIdx.y, blockIdx.y + 1 == gridDim.y);
    }
}

}  // namespace

hipError_t varco_launch_quantize_rows(int dtype, int64_t n_rows, int32_t width, const void* x, int64_t ldx, const void* gate, int64_t ldg,
                                      uint8_t* codes, uint8_t* scales, hipStream_t stream) {
    auto go = [&](auto type) {
        using T = decltype(type);
        const int64_t groups = n_rows * scale_ld(width), per = kThreads / (kCodeBlock / RowPiece<T>::P);
        const dim3 grid(unsigned(std::min<int64_t>((groups + per - 1) / per, 256 * 32)));
        if (gate)
            hipLaunchKernelGGL((quantize_rows_kernel<T, true>), grid, dim3(kThreads), 0, stream, n_rows, width, static_cast<const T*>(x), ldx,
                               static_cast<const T*>(gate), ldg, codes, scales);
        else
            hipLaunchKernelGGL((quantize_rows_kernel<T, false>), grid, dim3(kThreads), 0, stream, n_rows, width, static_cast<const T*>(x), ldx,
                               static_cast<const T*>(nullptr), 0, codes, scales);
    };
    if (dtype == VARCO_BF16)
        go(bf16_t{});
    else
        go(float{});
    return hipGetLastError();
}

hipError_t varco_launch_quantize_weights(int32_t n_in, int32_t n_out, const float* h, int64_t ldh, uint8_t* turned, uint8_t* turned_scales,
                                         uint8_t* codes, uint8_t* scales, hipStream_t stream) {
    const dim3 grid(unsigned((n_out + kCodeBlock - 1) / kCodeBlock), unsigned((n_in + kCodeBlock - 1) / kCodeBlock));
    hipLaunchKernelGGL(quantize_weights_kernel, grid, dim3(kThreads), 0, stream, n_in, n_out, h, ldh, turned, turned_scales, codes, scales);
    return hipGetLastError();
}
