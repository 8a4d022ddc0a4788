// Weight gradients from codes: dh (+)= sum over rows r of y[r, i] d[r, j]. The scales of both operands change along the reduction (a
// scale belongs to a row), so they cannot be applied to sums; code times scale is a bf16 number exactly (scales 2^-124 .. 2^119; what
// lies beyond is in kernels_scaled.hip), and the products are formed on the bf16 matrix units from those: nothing is rounded before the fp32 accumulators.
// Codes are turned into bf16 on their way into LDS (v_cvt_scalef32_pk_bf16_fp8, which applies the scale), where they lie as in memory, and
// are transposed when they are read (ds_read_b64_tr_b16 hands lane i of a group of 16 the i-th column of a 4 x 16 block). Row pitch: 64
// bytes more than a multiple of 256, so that the four rows of such a block start in four different quarters of the banks.
// The rows are cut into slabs, one workgroup per slab and tile, which leaves its sums as they lie in its accumulators; they are added by a second
// launch in one order. (410,003 rows, 100 x 47: 26 us, 41 with the sums as matrices; 169,343 rows, 256 x 256: 49, 52.)
// 2,449,029 rows, 512 x 512: 1,140 to 1,300 us, 990 to 1,130 TFLOP/s: the matrix units work 44 % of the time, the vector ALU (conversion, addresses) a third, and the
// two wavefronts of a SIMD do the one and the other mostly at the same time. (Codes requested when they are needed, one buffer, tiles of 128 x 128: 3,260 us.
// LDS layouts without the bank conflicts, a quarter of the cycles: 1,260 to 1,280; conversion between the products: 1,235, and 3 % slower over 256 x 256.)
// 169,343 rows, 256 x 256: 49 us, half of it the sums of the 256 slabs, 64 MB written and read.
#include <algorithm>

#include "codes_device.h"
#include "varco_scaled.h"

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));

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
template <int PITCH>
__device__ __forceinline__ bf16x8 fragment(uint32_t at) {
    using P = __attribute__((address_space(3))) shortx4*;
    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)at);
    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(at + 4 * PITCH));
    return __builtin_bit_cast(bf16x8, shortx8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
}

// One operand's share of a stage: BK rows of W columns in pieces of 16 codes, dealt to the threads row by row.
template <int W, int BK, int THREADS>
struct Slab {
    static constexpr int PER_ROW = W / 16, N = PER_ROW * BK / THREADS, ROWS = THREADS / PER_ROW, PITCH = W * 2 + 64;
    static_assert(N * THREADS == PER_ROW * BK && ROWS * PER_ROW == THREADS, "every thread takes as many pieces, of the same columns");
    const uint8_t* codes;                              // this thread's first piece of the next stage, and its scale
    const uint8_t* scales;
    int64_t ld, lds;
    int first;                                         // its row in a stage
    uint4 q[N];
    uint32_t s[N];
    // (pieces behind the last column repeat the one before; what comes of them is not stored)
    __device__ __forceinline__ void start(const uint8_t* c, const uint8_t* sc, int32_t width, int32_t c0, int64_t r0) {
        const int32_t col = c0 + 16 * int32_t(threadIdx.x % PER_ROW);
        ld = code_ld(width), lds = scale_ld(width), first = int(threadIdx.x / PER_ROW);
        codes = c + (r0 + first) * ld + min(int64_t(col), ld - 16), scales = sc + (r0 + first) * lds + min(col, width - 1) / kCodeBlock;
    }
    // a stage of `left` rows: those that there are not are the last one again
    __device__ __forceinline__ void load(int64_t left) {
        const int last = int(min(left, int64_t(BK))) - 1 - first;
#pragma unroll
        for (int h = 0; h < N; ++h) {
            const int row = min(h * ROWS, last);
            q[h] = *reinterpret_cast<const uint4*>(codes + __mul24(row, int(ld)));
            s[h] = scales[__mul24(row, int(lds))];
        }
        codes += BK * ld, scales += BK * lds;
    }
    // ... and zeros in one of the operands
    template <bool ZEROS>
    __device__ __forceinline__ void store(uint8_t* to, int64_t left) const {
#pragma unroll
        for (int h = 0; h < N; ++h) {
            const int row = first + h * ROWS;
            uint4 out[2];
            to_bf16(!ZEROS || row < left ? q[h] : make_uint4(0u, 0u, 0u, 0u), __uint_as_float(s[h] ? s[h] << 23 : 0x400000u), out);
            uint4* const p = reinterpret_cast<uint4*>(to + row * PITCH + (threadIdx.x % PER_ROW) * 32);
            p[0] = out[0], p[1] = out[1];
        }
    }
};

template <int WI_, int WJ_, int MI_, int NJ_, int BK>
struct Tile {
    static constexpr int WI = WI_, WJ = WJ_, MI = MI_, NJ = NJ_;
    static constexpr int BI = 16 * MI * WI, BJ = 16 * NJ * WJ, THREADS = 64 * WI * WJ, STAGE = BK;
    using Y = Slab<BI, BK, THREADS>;
    using D = Slab<BJ, BK, THREADS>;
    static constexpr int BYTES = 2 * BK * (Y::PITCH + D::PITCH);
};

// Four elements of a row, added to what it holds if `add`.
__device__ __forceinline__ void store_four(float* row, int32_t at, int32_t width, floatx4 v, bool add) {
    float x[4] = {v[0], v[1], v[2], v[3]};
    if (add) {
        float c[4];
        RowPiece<float>::load(row, at, width, c);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += c[i];
    }
    RowPiece<float>::store(row, at, width, x);
}

// Work is numbered slab after slab and dealt to the 8 XCDs in runs, so that the tiles of a slab share its rows in the L2 of one (or two). While a stage is multiplied the next one is
// on its way to registers; it goes to the other of two buffers when the products have been issued.
template <int WI, int WJ, int MI, int NJ, int BK>
__global__ __launch_bounds__(64 * WI * WJ, 2) void scaled_tn_kernel(ScaledWeightArgs a, int32_t split, int64_t rows_per_split, int32_t tiles_j, int32_t tiles) {
    using L = Tile<WI, WJ, MI, NJ, BK>;
    constexpr int PY = L::Y::PITCH, PD = L::D::PITCH;
    __shared__ __attribute__((aligned(16))) uint8_t lds[L::BYTES];
    const int32_t run = (split * tiles + 7) / 8, work = int32_t(blockIdx.x & 7) * run + int32_t(blockIdx.x >> 3);
    if (work >= split * tiles) return;                  // whole workgroup
    const int32_t slab = work / tiles, tile = work % tiles;
    const int32_t i0 = tile / tiles_j * L::BI, j0 = tile % tiles_j * L::BJ;
    const int64_t r0 = slab * rows_per_split, r1 = min(a.n_rows, r0 + rows_per_split);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wi = wave / WJ * (16 * MI), wj = wave % WJ * (16 * NJ);
    floatx4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = floatx4(0.f);
    const uint32_t base = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)lds));
    const uint32_t row = 8 * (lane >> 4) + ((lane >> 2) & 3), sub = 8 * (lane & 3);
    constexpr int kY = BK * PY, kD = BK * PD;
    const uint32_t at_y = base + row * PY + sub + wi * 2, at_d = base + 2 * kY + row * PD + sub + wj * 2;

    typename L::Y y;
    typename L::D d;
    y.start(a.y, a.y_scales, a.n_in, i0, r0);
    d.start(a.d, a.d_scales, a.n_out, j0, r0);
    if (r0 < r1) {
        y.load(r1 - r0), d.load(r1 - r0);
        y.template store<false>(lds, r1 - r0), d.template store<true>(lds + 2 * kY, r1 - r0);
    }
    __syncthreads();
    uint32_t buf = 0;
    for (int64_t r = r0; r < r1; r += BK, buf ^= 1u) {
        const int64_t left = r1 - r - BK;
        if (left > 0) y.load(left), d.load(left);
#pragma unroll
        for (int h = 0; h < BK / 32; ++h) {
            bf16x8 fd[NJ];
#pragma unroll
            for (int j = 0; j < NJ; ++j) fd[j] = fragment<PD>(at_d + buf * kD + h * 32 * PD + j * 32);
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const bf16x8 fy = fragment<PY>(at_y + buf * kY + h * 32 * PY + i * 32);
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fd[j], fy, acc[i][j], 0, 0, 0);
            }
        }
        if (left > 0) y.template store<false>(lds + (buf ^ 1u) * kY, left), d.template store<true>(lds + 2 * kY + (buf ^ 1u) * kD, left);
        __syncthreads();
    }
    // accumulator v of a lane is element (lane % 16, 4 (lane / 16) + v)
    if (split > 1) {
        // in the order of the accumulators, a kilobyte by an instruction
        floatx4* const out = reinterpret_cast<floatx4*>(a.partial) + (int64_t(slab) * tiles + tile) * (L::BI * L::BJ / 4) + wave * (MI * NJ * 64) + lane;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                if (i0 + wi + 16 * i < a.n_in && j0 + wj + 16 * j < a.n_out) out[(i * NJ + j) * 64] = acc[i][j];
        return;
    }
    const int g = lane >> 4, l = lane & 15;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const int32_t ri = i0 + wi + 16 * i + l, cj = j0 + wj + 16 * j + 4 * g;
            if (ri < a.n_in) store_four(a.dh + ri * a.ldh, cj, a.n_out, acc[i][j], a.accumulate);
        }
}

// dh (+)= the slabs' sums, in the order in which the tiles were stored: a fragment of 16 x 16 by 64 threads of four elements, kShares shares of the slabs,
// each from its first slab on, then the shares in turn.
constexpr int kShares = 8;
template <typename L>
__global__ __launch_bounds__(64 * kShares) void slab_sum_kernel(const float* __restrict__ partial, int32_t split, int32_t tiles_j, int32_t tiles, int32_t n_in, int32_t n_out,
                                                                float* dh, int64_t ldh, int32_t accumulate) {
    __shared__ floatx4 shares[kShares][64];
    const int lane = threadIdx.x & 63, share = threadIdx.x >> 6;
    const int32_t tile = int32_t(blockIdx.y), f = int32_t(blockIdx.x);           // fragment of the tile
    const int32_t wave = f / (L::MI * L::NJ), i = f % (L::MI * L::NJ) / L::NJ, j = f % L::NJ;
    const int32_t r0 = tile / tiles_j * L::BI + wave / L::WJ * (16 * L::MI) + 16 * i, c0 = tile % tiles_j * L::BJ + wave % L::WJ * (16 * L::NJ) + 16 * j;
    if (r0 >= n_in || c0 >= n_out) return;              // whole workgroup
    const floatx4* const from = reinterpret_cast<const floatx4*>(partial) + int64_t(tile) * (L::BI * L::BJ / 4) + f * 64 + lane;
    const int64_t step = int64_t(tiles) * (L::BI * L::BJ / 4);
    floatx4 x = floatx4(0.f);
#pragma unroll 8
    for (int32_t s = share; s < split; s += kShares) x += from[s * step];
    shares[share][lane] = x;
    __syncthreads();
    if (share) return;
#pragma unroll
    for (int i = 1; i < kShares; ++i) x += shares[i][lane];
    const int32_t ri = r0 + (lane & 15);
    if (ri < n_in) store_four(dh + ri * ldh, c0 + 4 * (lane >> 4), n_out, x, accumulate);
}

template <int WI, int WJ, int MI, int NJ, int BK>
void launch(Tile<WI, WJ, MI, NJ, BK>, const ScaledWeightArgs& a, int32_t split, int64_t rows, int32_t tiles_j, int32_t tiles, hipStream_t stream) {
    hipLaunchKernelGGL((scaled_tn_kernel<WI, WJ, MI, NJ, BK>), dim3(unsigned((int64_t(split) * tiles + 7) / 8 * 8)), dim3(64 * WI * WJ), 0, stream, a, split, rows,
                       tiles_j, tiles);
}

// Tiles of 256 x 256 where the weights have more than 128 rows and columns and a workgroup per compute unit gets 512 rows or more, 128 x 256 or 256 x 128
// where one side has 65 to 128; else 128 x 128, and 64 on a side of at most 64. (512 x 512 weights, tiles of 256 / of 128: 20,000 rows, 313 each, 36.9 /
// 30.8 us; 169,343 rows, 2,646 each, 114 / 168; 256 x 256 over 169,343 rows, 661 each, 49.5 / 58; tiles of 128 x 256, half the sums, there 47.9, over 410,003
// rows 93, 87 so. Tiles of 128 x 256 / 128 x 128 in turn: 500,000 rows 128 x 512 106 / 132, 125,702 rows 96 x 914 52 / 54, 1,000,000 rows 120 x 300 175 / 178,
// 200,000 rows 128 x 2048 146 / 188, 131,101 rows 65 x 256 23.9 / 23.6; 256 x 128 / 128 x 128 for the same turned round: 106 / 135, 52 / 56, 168 / 181, 145 / 193,
// 23.5 / 23.9.)
using Big = Tile<2, 4, 8, 4, 64>;
using Wide = Tile<2, 4, 4, 4, 64>;
using Tall = Tile<4, 2, 4, 4, 64>;
using Middle = Tile<2, 2, 4, 4, 32>;
using Narrow = Tile<2, 2, 4, 2, 64>;
using Flat = Tile<2, 2, 2, 4, 64>;
using Small = Tile<2, 2, 2, 2, 64>;

// Calls f(tile, workgroups that are wanted).
template <typename F>
void with_tile(int64_t n_rows, int32_t n_in, int32_t n_out, F f) {
    const bool many = n_rows * int64_t((n_in + 255) / 256) * ((n_out + 255) / 256) >= int64_t(256) * 512;
    if (many && n_in > 128 && n_out > 128)
        f(Big{}, 256);
    else if (many && n_in > 64 && n_out > 128)
        f(Wide{}, 256);
    else if (many && n_in > 128 && n_out > 64)
        f(Tall{}, 256);
    else if (n_in > 64 && n_out > 64)
        f(Middle{}, 512);
    else if (n_in > 64)
        f(Narrow{}, 512);
    else if (n_out > 64)
        f(Flat{}, 512);
    else
        f(Small{}, 512);
}
template <typename L>
int64_t tiles_of(int32_t n_in, int32_t n_out) { return int64_t((n_in + L::BI - 1) / L::BI) * ((n_out + L::BJ - 1) / L::BJ); }
int64_t slab_rows(int64_t n_rows, int64_t split, int64_t stage) { return std::max<int64_t>(1, ((n_rows + split - 1) / split + stage - 1) / stage) * stage; }
template <typename L>
int32_t split_of(int64_t n_rows, int32_t n_in, int32_t n_out, int64_t wanted) {
    const int64_t rows = slab_rows(n_rows, std::max<int64_t>(1, std::min<int64_t>(wanted / tiles_of<L>(n_in, n_out), n_rows / 256)), L::STAGE);
    return int32_t(std::max<int64_t>(1, (n_rows + rows - 1) / rows));
}

}  // namespace

int64_t varco_scaled_weight_floats(int64_t n_rows, int32_t n_in, int32_t n_out) {
    int64_t floats = 0;
    with_tile(n_rows, n_in, n_out, [&](auto tile, int64_t wanted) {
        using L = decltype(tile);
        const int64_t split = split_of<L>(n_rows, n_in, n_out, wanted);
        floats = split > 1 ? split * tiles_of<L>(n_in, n_out) * (L::BI * L::BJ) : 0;
    });
    return floats;
}

hipError_t varco_launch_scaled_bwd_weight(const ScaledWeightArgs& a, hipStream_t stream) {
    with_tile(a.n_rows, a.n_in, a.n_out, [&](auto tile, int64_t wanted) {
        using L = decltype(tile);
        const int32_t split = split_of<L>(a.n_rows, a.n_in, a.n_out, wanted);
        const int32_t tiles_j = int32_t((a.n_out + L::BJ - 1) / L::BJ), tiles = int32_t(tiles_of<L>(a.n_in, a.n_out));
        launch(L{}, a, split, slab_rows(a.n_rows, split, L::STAGE), tiles_j, tiles, stream);
        if (split > 1)
            hipLaunchKernelGGL(slab_sum_kernel<L>, dim3(L::BI * L::BJ / 256, tiles), dim3(64 * kShares), 0, stream, a.partial, split, tiles_j, tiles, a.n_in,
                               a.n_out, a.dh, a.ldh, a.accumulate);
    });
    return hipGetLastError();
}
