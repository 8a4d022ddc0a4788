// c = act((c +) X W) for rows X and weights W of 8-bit codes with a power of two as scale for each 128 elements of the reduction
// (rows of X: per row; W: per 128 outputs).
// bf16 results: v_mfma_scale_f32_16x16x128_f8f6f4 takes 128 steps of the reduction at once and applies the scales itself, as exponents, so
// the sums stay in its fp32 accumulators from the first block to the last. That unit adds products in groups of eight consecutive
// ones and drops, of each, what lies below 2^-13 of the group's largest power of two (measured: one product beside two larger
// ones that cancel; between groups 24 bits and more are kept). Over rows of normal numbers that is 1.5e-4 of the result's norm where
// the rounding to bf16 is 1.7e-3.
// fp32 results, which would lose ten bits to that, come from the bf16 units at half the rate: a code times its scale is a bf16
// number exactly, made of the fragment when it has been read (v_cvt_scalef32_pk_bf16_fp8).
// W lies with the reduction consecutive, as X does: a lane's 32 bytes of a fragment are two pieces of 16 bytes, taken as pieces g and
// g + 4 of the 8 of a block, g = lane / 16, in both operands. (The order inside a block of 128 is free as long as both have the same.)
// The weights are the first operand: a lane then holds four consecutive outputs of one row.
#include <algorithm>

#include "codes_device.h"
#include "varco_scaled.h"

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kTile = 128;           // rows and outputs of a tile; a wavefront takes 64 x 64
constexpr int BK = kCodeBlock;

// 16-byte piece p of row r of a tile: 128 bytes per row, pieces moved so that eight rows read at one piece use all banks.
__device__ __forceinline__ int piece_at(int r, int p) { return r * BK + ((p ^ (r & 7)) << 4); }

// A fragment's 32 codes as four fragments of the bf16 unit.
struct Bf16Fragment {
    bf16x8 f[4];
    __device__ __forceinline__ Bf16Fragment(const intx8& q, int scale) {
        const float x = __uint_as_float(scale ? uint32_t(scale) << 23 : 0x400000u);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uintx4 u;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                u[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(uint32_t(q[2 * i + j]), x, false));
                u[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(uint32_t(q[2 * i + j]), x, true));
            }
            f[i] = __builtin_bit_cast(bf16x8, u);
        }
    }
};

template <typename T>
__global__ __launch_bounds__(kThreads) void scaled_kernel(ScaledArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t lx[kTile * BK];
    __shared__ __attribute__((aligned(16))) uint8_t lw[kTile * BK];
    const int64_t m0 = int64_t(blockIdx.x) * kTile;
    const int32_t n0 = int32_t(blockIdx.y) * kTile;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, l = lane & 15;
    const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
    const int64_t ld = code_ld(a.n_in), lds = scale_ld(a.n_in);
    const int32_t steps = (a.n_in + BK - 1) / BK;
    floatx4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = floatx4(0.f);
    for (int32_t s = 0; s < steps; ++s) {
        uint4 vx[4], vw[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int e = threadIdx.x + h * kThreads, r = e >> 3, p = e & 7;
            const int64_t k = int64_t(s) * BK + p * 16;
            vx[h] = vw[h] = make_uint4(0u, 0u, 0u, 0u);
            if (k < ld && m0 + r < a.n_rows) vx[h] = *reinterpret_cast<const uint4*>(a.x + (m0 + r) * ld + k);
            if (k < ld && n0 + r < a.n_out) vw[h] = *reinterpret_cast<const uint4*>(a.w + (n0 + r) * ld + k);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int e = threadIdx.x + h * kThreads, r = e >> 3, p = e & 7;
            *reinterpret_cast<uint4*>(lx + piece_at(r, p)) = vx[h];
            *reinterpret_cast<uint4*>(lw + piece_at(r, p)) = vw[h];
        }
        __syncthreads();
        const int scale_w = a.w_scales[(n0 / kCodeBlock) * lds + s];
        auto fragment = [&](const uint8_t* t, int r) {
            const uint4 lo = *reinterpret_cast<const uint4*>(t + piece_at(r + l, g)), hi = *reinterpret_cast<const uint4*>(t + piece_at(r + l, g + 4));
            return intx8{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
        };
        if constexpr (sizeof(T) == 2) {
            intx8 fw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) fw[i] = fragment(lw, wn + 16 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const intx8 fx = fragment(lx, wm + 16 * j);
                const int scale_x = a.x_scales[min(m0 + wm + 16 * j + l, a.n_rows - 1) * lds + s];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[i], fx, acc[i][j], 0, 0, 0, scale_w, 0, scale_x);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Bf16Fragment fx(fragment(lx, wm + 16 * j), a.x_scales[min(m0 + wm + 16 * j + l, a.n_rows - 1) * lds + s]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const Bf16Fragment fw(fragment(lw, wn + 16 * i), scale_w);
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw.f[q], fx.f[q], acc[i][j], 0, 0, 0);
                }
            }
        }
    }
    // accumulator v of a lane: output 4 (lane / 16) + v, row lane % 16
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t row = m0 + wm + 16 * j + l;
        if (row >= a.n_rows) continue;
        T* const c = static_cast<T*>(a.c) + row * a.ldc;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int32_t n = n0 + wn + 16 * i + 4 * g + v;
                if (n >= a.n_out) continue;
                float x = acc[i][j][v];
                if (a.accumulate) x += Elem<T>::load(c + n);
                if (a.relu) x = x < 0.f ? 0.f : x;         // (NaN stays)
                Elem<T>::store(c + n, x);
            }
    }
}

}  // namespace

hipError_t varco_launch_scaled_transform(int dtype, const ScaledArgs& a, hipStream_t stream) {
    const dim3 grid(unsigned((a.n_rows + kTile - 1) / kTile), unsigned((a.n_out + kTile - 1) / kTile));
    if (dtype == VARCO_BF16)
        hipLaunchKernelGGL(scaled_kernel<bf16_t>, grid, dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL(scaled_kernel<float>, grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}
