// Root-mean-square norm of rows with a residual's addition, and its backward pass.
//   u = x + r (rounded to the storage type, which is what the backward pass reads)    s = 1 / sqrt(mean u^2 + eps)    y = u s g
//   h = dy g    xh = u s    dx = s (h - xh mean(h xh)) + du    dg = sum over rows of dy xh
// One pass: a row's elements stay in registers between the sum and their use. G lanes take a row, E pieces of 16 bytes per lane;
// rows above 2,048 elements are taken by 512 lanes, which meet in LDS.
// Bound by reading and writing each row once: 169,343 x 256 fp32 with a residual 125 to 131 us, 5.5 TB/s (132 with stores that the caches keep), its
// backward pass 125 us (130); 2,449,029 x 512 bf16 with a residual and codes 1,955 us (2,005), 4.5 TB/s; 1,000,003 x 1000 bf16 backward 1,650 us
// (1,625), 4.9 TB/s.
#include <algorithm>
#include <cfloat>

#include "row_layout.h"
#include "varco_scaled.h"

namespace {

// Sum over the G lanes of a row, in all of them, in one order.
template <int G, typename S>
__device__ __forceinline__ S row_sum(S x, S* shared) {
    if constexpr (G <= 64) {
        return lanes_sum<G>(x);
    } else {
        x = lanes_sum<64>(x);
        __syncthreads();             // (the previous row's sums have been read)
        if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
        __syncthreads();
        S s = S(0);
#pragma unroll
        for (int i = 0; i < G / 64; ++i) s += shared[i];
        return s;
    }
}

// 1 / sqrt(m), rounded once: a Newton step from the unit's root (off by a step), with its residual 1 - m h^2 in twice the bits. Where m is no normal
// number of fp32 the root is one of fp32 throughout (infinite, 0, NaN, of few bits). The lanes' sums are added in fp64 before it: of the roundings of
// a sum in fp32 the last few additions' count most, and with those, the root's and the division's 1 / rms was off by 0.71 2^-24 on average, 0.43 so (rounding
// alone: 0.43), and every value made of it, codes next to a rounding's border among them.
__device__ __forceinline__ float inverse_root(double m) {
    const float hi = float(m);
    if (!(hi >= FLT_MIN && hi < INFINITY)) return 1.f / sqrtf(hi);
    const float lo = float(m - double(hi)), h = __builtin_amdgcn_rsqf(hi);
    const float p = hi * h, q = fmaf(lo, h, fmaf(hi, h, -p));        // m h = p + q
    return fmaf(0.5f * h, fmaf(-q, h, fmaf(-p, h, 1.f)), h);
}

template <typename T, int G, int E, bool CODES, bool ANY>
__global__ __launch_bounds__(row_threads(G)) void rms_norm_kernel(NormFwdArgs a) {
    using Row = RowPiece<T>;
    constexpr int P = Row::P, kRows = row_threads(G) / G;
    __shared__ double shared[G > 64 ? G / 64 : 1];
    const int t = threadIdx.x & (G - 1);
    float gain[E][P];
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int32_t c = (t + e * G) * P + j;
            gain[e][j] = c < a.width && a.gain ? a.gain[c] : 1.f;
        }
    const double share = 1.0 / double(a.width);
    for (int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / G; row < a.n_rows; row += int64_t(gridDim.x) * kRows) {
        float v[E][P];
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) Row::template load<ANY>(static_cast<const T*>(a.x) + row * a.ldx, (t + e * G) * P, a.width, v[e]);
        if (a.residual) {
            float r[E][P];
#pragma unroll
            for (int e = 0; e < E; ++e) Row::template load<ANY>(static_cast<const T*>(a.residual) + row * a.ldr, (t + e * G) * P, a.width, r[e]);
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int j = 0; j < P; ++j) v[e][j] = Row::rounded(v[e][j] + r[e][j]);
        }
        if (a.total)
#pragma unroll
            for (int e = 0; e < E; ++e) Row::template store<ANY, true>(static_cast<T*>(a.total) + row * a.ldt, (t + e * G) * P, a.width, v[e]);
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int j = 0; j < P; ++j) sum = fmaf(v[e][j], v[e][j], sum);
        const float s = inverse_root(fma(row_sum<G>(double(sum), shared), share, double(a.eps)));
        if (t == 0 && a.inv_rms) a.inv_rms[row] = s;
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int j = 0; j < P; ++j) v[e][j] = v[e][j] * s * gain[e][j];
        if (a.y)
#pragma unroll
            for (int e = 0; e < E; ++e) Row::template store<ANY, true>(static_cast<T*>(a.y) + row * a.ldy, (t + e * G) * P, a.width, v[e]);
        if constexpr (CODES) store_row_codes<T, G, E>(v, t, a.width, a.codes + row * code_ld(a.width), a.scales + row * scale_ld(a.width));
    }
}

// dg: every lane sums its own columns over the rows that its group takes; the groups of a workgroup are joined in LDS, the workgroups'
// sums by a second launch, each in one order. With one workgroup dgain is written at once.
template <typename T, int G, int E, bool ANY>
__global__ __launch_bounds__(row_threads(G)) void rms_norm_bwd_kernel(NormBwdArgs a) {
    using Row = RowPiece<T>;
    constexpr int P = Row::P, kThreads = row_threads(G), kRows = kThreads / G;
    __shared__ float shared[G > 64 ? G / 64 : 1];
    __shared__ float joined[kRows > 1 ? kThreads * E * P : 1];
    const int t = threadIdx.x & (G - 1);
    float gain[E][P], dg[E][P];
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int32_t c = (t + e * G) * P + j;
            gain[e][j] = c < a.width && a.gain ? a.gain[c] : 1.f;
            dg[e][j] = 0.f;
        }
    const float share = 1.f / float(a.width);
    for (int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / G; row < a.n_rows; row += int64_t(gridDim.x) * kRows) {
        float dy[E][P], u[E][P];
        const float s = a.inv_rms[row];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            Row::template load<ANY>(static_cast<const T*>(a.dy) + row * a.lddy, (t + e * G) * P, a.width, dy[e]);
            Row::template load<ANY>(static_cast<const T*>(a.u) + row * a.ldu, (t + e * G) * P, a.width, u[e]);
        }
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int j = 0; j < P; ++j) {
                u[e][j] *= s;
                dg[e][j] = fmaf(dy[e][j], u[e][j], dg[e][j]);
                dy[e][j] *= gain[e][j];
                sum = fmaf(dy[e][j], u[e][j], sum);
            }
        if (!a.dx) continue;
        const float mean = row_sum<G>(sum, shared) * share;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float du[P];
            if (a.dtotal) Row::template load<ANY>(static_cast<const T*>(a.dtotal) + row * a.lddt, (t + e * G) * P, a.width, du);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const float d = s * fmaf(-u[e][j], mean, dy[e][j]);
                dy[e][j] = a.dtotal ? d + du[j] : d;
            }
            Row::template store<ANY, true>(static_cast<T*>(a.dx) + row * a.lddx, (t + e * G) * P, a.width, dy[e]);
        }
    }
    if (!a.dgain) return;
    if constexpr (kRows > 1) {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int j = 0; j < P; ++j) joined[(threadIdx.x / G) * (G * E * P) + (t + e * G) * P + j] = dg[e][j];
        __syncthreads();
        for (int32_t c = threadIdx.x; c < a.width; c += kThreads) {
            float x = 0.f;
            for (int r = 0; r < kRows; ++r) x += joined[r * (G * E * P) + c];
            if (gridDim.x > 1)
                a.partial[int64_t(blockIdx.x) * a.width + c] = x;
            else
                a.dgain[c] = a.accumulate ? a.dgain[c] + x : x;
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const int32_t c = (t + e * G) * P + j;
                if (c >= a.width) continue;
                if (gridDim.x > 1)
                    a.partial[int64_t(blockIdx.x) * a.width + c] = dg[e][j];
                else
                    a.dgain[c] = a.accumulate ? a.dgain[c] + dg[e][j] : dg[e][j];
            }
    }
}

// dgain (+)= the sum of `n` rows of `partial`: 16 columns per workgroup, 64 shares of the rows, in fp64.
constexpr int kShares = 64;
__global__ __launch_bounds__(16 * kShares) void gain_sum_kernel(const float* __restrict__ partial, int32_t n, int32_t width, float* dgain, int32_t accumulate) {
    __shared__ double shares[kShares][16];
    const int32_t c = int32_t(blockIdx.x) * 16 + (threadIdx.x & 15);
    const int part = threadIdx.x >> 4;
    double x = 0.0;
    if (c < width)
#pragma unroll 4
        for (int32_t r = part; r < n; r += kShares) x += double(partial[int64_t(r) * width + c]);
    shares[part][threadIdx.x & 15] = x;
    __syncthreads();
    for (int s = kShares / 2; s > 0; s >>= 1) {
        if (part < s) shares[part][threadIdx.x & 15] += shares[part + s][threadIdx.x & 15];
        __syncthreads();
    }
    if (part == 0 && c < width) dgain[c] = float(accumulate ? double(dgain[c]) + shares[0][threadIdx.x] : shares[0][threadIdx.x]);
}

}  // namespace

hipError_t varco_launch_rms_norm_fwd(int dtype, const NormFwdArgs& a, hipStream_t stream) {
    with_type(dtype, [&](auto type) {
        using T = decltype(type);
        with_row_layout<T>(a.width, [&](auto g, auto e) {
            constexpr int G = decltype(g)::value, E = decltype(e)::value, kRows = row_threads(G) / G;
            const dim3 grid(unsigned(std::min<int64_t>((a.n_rows + kRows - 1) / kRows, 256 * 16)));
            with_bool(a.codes, [&](auto codes) {
                with_bool(a.width % RowPiece<T>::P, [&](auto any) {
                    hipLaunchKernelGGL((rms_norm_kernel<T, G, E, decltype(codes)::value, decltype(any)::value>), grid, dim3(row_threads(G)), 0, stream, a);
                });
            });
        });
    });
    return hipGetLastError();
}

int32_t varco_norm_blocks(int dtype, int64_t n_rows, int32_t width) {
    int64_t blocks = 1;
    with_type(dtype, [&](auto type) {
        with_row_layout<decltype(type)>(width, [&](auto g, auto) {
            constexpr int G = decltype(g)::value, kRows = row_threads(G) / G;
            blocks = std::max<int64_t>(1, std::min<int64_t>((n_rows + kRows - 1) / kRows, 1024));
        });
    });
    return int32_t(blocks);
}

hipError_t varco_launch_rms_norm_bwd(int dtype, const NormBwdArgs& a, hipStream_t stream) {
    const int32_t blocks = varco_norm_blocks(dtype, a.n_rows, a.width);
    with_type(dtype, [&](auto type) {
        using T = decltype(type);
        with_row_layout<T>(a.width, [&](auto g, auto e) {
            constexpr int G = decltype(g)::value, E = decltype(e)::value;
            with_bool(a.width % RowPiece<T>::P, [&](auto any) {
                hipLaunchKernelGGL((rms_norm_bwd_kernel<T, G, E, decltype(any)::value>), dim3(unsigned(blocks)), dim3(row_threads(G)), 0, stream, a);
            });
        });
    });
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || !a.dgain || blocks == 1) return err;
    hipLaunchKernelGGL(gain_sum_kernel, dim3(unsigned((a.width + 15) / 16)), dim3(16 * kShares), 0, stream, a.partial, blocks, a.width, a.dgain, a.accumulate);
    return hipGetLastError();
}
