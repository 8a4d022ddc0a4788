// Rows and weight matrices as 8-bit codes with a power of two as scale for each 128 columns (128 x 128 elements of a weight
// matrix). Elementwise but for the largest size of a block: bound by reading the values once and writing a byte for each.
// 2,449,029 x 512 bf16 rows with a gate 1,400 us, 4.5 TB/s; 410,003 x 47 fp32 17 us, 5.6 TB/s.
#include <algorithm>

#include "row_layout.h"
#include "varco_scaled.h"

namespace {

constexpr int kWeightThreads = 1024, kWeightRows = kCodeBlock * kCodeBlock / 4 / kWeightThreads;       // rows of a thread, four columns each

// Rows dealt to lanes as row_layout.h has it: no lane waits for more than the lanes of its scale.
template <typename T, int G, int E, bool GATE, bool ANY>
__global__ __launch_bounds__(row_threads(G)) void quantize_rows_kernel(int64_t n_rows, int32_t width, const T* x, int64_t ldx, const T* gate, int64_t ldg,
                                                                       uint8_t* codes, uint8_t* scales) {
    using Row = RowPiece<T>;
    constexpr int P = Row::P, kRows = row_threads(G) / G;
    const int64_t ldc = code_ld(width), lds = scale_ld(width);
    const int t = threadIdx.x & (G - 1);
    for (int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / G; row < n_rows; row += int64_t(gridDim.x) * kRows) {
        float v[E][P];
#pragma unroll
        for (int e = 0; e < E; ++e) Row::template load<ANY>(x + row * ldx, (t + e * G) * P, width, v[e]);
        if constexpr (GATE) {
            float g[E][P];
#pragma unroll
            for (int e = 0; e < E; ++e) Row::template load<ANY>(gate + row * ldg, (t + e * G) * P, width, g[e]);
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int j = 0; j < P; ++j) v[e][j] = g[e][j] > 0.f ? v[e][j] : 0.f;
        }
        store_row_codes<T, G, E>(v, t, width, codes + row * ldc, scales + row * lds);
    }
}

// A workgroup takes 128 x 128 weights: read once, kept in registers until the largest is known, written row-wise and, through LDS, column-wise.
__global__ __launch_bounds__(kWeightThreads) void quantize_weights_kernel(int32_t n_in, int32_t n_out, const float* h, int64_t ldh, uint8_t* turned,
                                                                    uint8_t* turned_scales, uint8_t* codes, uint8_t* scales) {
    __shared__ float largest[kWeightThreads / 64];
    __shared__ uint32_t tile[kCodeBlock][kCodeBlock / 4 + 1];
    const int32_t i0 = int32_t(blockIdx.y) * kCodeBlock, j0 = int32_t(blockIdx.x) * kCodeBlock;
    const int lane = threadIdx.x & 31, first = threadIdx.x >> 5;       // 32 lanes of 4 columns
    constexpr int kStep = kWeightThreads / 32;
    float v[kWeightRows][4];
    float a = 0.f;
#pragma unroll
    for (int r = 0; r < kWeightRows; ++r) {
        const int32_t i = i0 + first + kStep * r;
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
    a = largest[0];
#pragma unroll
    for (int i = 1; i < kWeightThreads / 64; ++i) a = fmaxf(a, largest[i]);
    const int e = code_exponent(a);
    const float inverse = code_inverse(e);
    const int64_t ld_in = code_ld(n_in), ld_out = code_ld(n_out);
#pragma unroll
    for (int r = 0; r < kWeightRows; ++r) {
        const int32_t row = first + kStep * r;
        const uint32_t q = four_codes(v[r][0], v[r][1], v[r][2], v[r][3], inverse);
        tile[row][lane] = q;
        if (codes && i0 + row < n_in && j0 + 4 * lane < ld_out) *reinterpret_cast<uint32_t*>(codes + (i0 + row) * ld_out + j0 + 4 * lane) = q;
    }
    __syncthreads();
    if (turned) {
        const uint8_t* const bytes = reinterpret_cast<const uint8_t*>(tile);
        constexpr int kPitch = kCodeBlock + 4;
#pragma unroll
        for (int r = 0; r < kWeightRows; ++r) {
            const int32_t col = first + kStep * r;
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
    with_type(dtype, [&](auto type) {
        using T = decltype(type);
        with_row_layout<T>(width, [&](auto g, auto e) {
            constexpr int G = decltype(g)::value, E = decltype(e)::value, kRows = row_threads(G) / G;
            const dim3 grid(unsigned(std::min<int64_t>((n_rows + kRows - 1) / kRows, 256 * 32)));
            with_bool(gate, [&](auto gated) {
                with_bool(width % RowPiece<T>::P, [&](auto any) {
                    hipLaunchKernelGGL((quantize_rows_kernel<T, G, E, decltype(gated)::value, decltype(any)::value>), grid, dim3(row_threads(G)), 0, stream,
                                       n_rows, width, static_cast<const T*>(x), ldx, static_cast<const T*>(gate), ldg, codes, scales);
                });
            });
        });
    });
    return hipGetLastError();
}

hipError_t varco_launch_quantize_weights(int32_t n_in, int32_t n_out, const float* h, int64_t ldh, uint8_t* turned, uint8_t* turned_scales,
                                         uint8_t* codes, uint8_t* scales, hipStream_t stream) {
    const dim3 grid(unsigned((n_out + kCodeBlock - 1) / kCodeBlock), unsigned((n_in + kCodeBlock - 1) / kCodeBlock));
    hipLaunchKernelGGL(quantize_weights_kernel, grid, dim3(kWeightThreads), 0, stream, n_in, n_out, h, ldh, turned, turned_scales, codes, scales);
    return hipGetLastError();
}
