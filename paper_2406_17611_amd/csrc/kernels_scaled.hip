// c = act((c +) X W) for rows X and weights W of 8-bit codes with a power of two as scale for each 128 elements of the reduction
// (rows of X: per row; W: per 128 outputs).
// bf16 results: v_mfma_scale_f32_16x16x128_f8f6f4 takes 128 steps of the reduction at once and applies the scales itself, as exponents, so
// the sums stay in its fp32 accumulators from the first block to the last. That unit adds products in groups of eight consecutive
// ones and drops, of each, what lies below 2^-13 of the group's largest power of two (measured: one product beside two larger
// ones that cancel; between groups 24 bits and more are kept). Over rows of normal numbers that is 1.5e-4 of the result's norm where
// the rounding to bf16 is 1.7e-3.
// fp32 results, which would lose ten bits to that, come from the bf16 units at half the rate: a code times its scale, made of the fragment
// when it has been read (v_cvt_scalef32_pk_bf16_fp8), is a bf16 number exactly under scales from 2^-124 (its smallest code is 2^-133, the last
// step of bf16; below, the conversion rounds to that) to 2^119 (256 2^120, the only number beyond, is 2^128 and becomes an infinity, as in fp32).
// W lies with the reduction consecutive, as X does: a lane's 32 bytes of a fragment are two pieces of 16 bytes, taken as pieces g and
// g + 4 of the 8 of a block, g = lane / 16, in both operands. (The order inside a block of 128 is free as long as both have the same.)
// The weights are the first operand: a lane then holds four consecutive outputs of one row.
#include <algorithm>
#include <type_traits>

#include "codes_device.h"
#include "varco_scaled.h"

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int BK = kCodeBlock;

// Two pieces of 16 bytes as a fragment of the 8-bit unit.
__device__ __forceinline__ intx8 joined(const uint4& lo, const uint4& hi) {
    return intx8{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
}

// A fragment's 32 codes as four fragments of the bf16 unit. The scale's exponent + 127 are the upper bits of the fp32 number 2^e; 2^-127 is 0x400000 (the
// conversion reads the exponent bits, 0 as 2^-127: measured for all 255 scales and all codes).
struct Bf16Fragment {
    bf16x8 f[4];
    Bf16Fragment() = default;
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

// Which output (of the 16 NI of a wavefront) row `at` of weight fragment f is. Accumulator v of a lane is row 4 (lane / 16) + v of its
// fragment; with this order the accumulators of one fragment (fp32) or of two (bf16) are the 16 consecutive bytes of a store, and the four
// lanes of a row fill 64 bytes with it. (64 consecutive bytes per lane, stored in quarters, fill 64 bytes of a row in four instructions: fp32, 169,343 x
// 1000 x 1000 546 us against 458.)
template <typename T>
__device__ __forceinline__ constexpr int output_of(int f, int at) {
    return sizeof(T) == 2 ? 32 * (f >> 1) + 8 * (at >> 2) + 4 * (f & 1) + (at & 3) : 16 * f + at;
}

// A lane's outputs of a row: acc[f] the accumulators of fragment f, n0 the wavefront's first output.
template <typename T, int NI>
__device__ __forceinline__ void store_outputs(T* row, int32_t n0, int g, const ScaledArgs& a, const floatx4 (&acc)[NI]) {
    constexpr int P = RowPiece<T>::P, F = P / 4;
#pragma unroll
    for (int i = 0; i < NI / F; ++i) {
        const int32_t n = n0 + output_of<T>(F * i, 4 * g);
        float x[P];
        if (a.accumulate)
            RowPiece<T>::load(row, n, a.n_out, x);
        else
#pragma unroll
            for (int j = 0; j < P; ++j) x[j] = 0.f;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            x[j] += acc[F * i + j / 4][j % 4];
            if (a.relu) x[j] = x[j] < 0.f ? 0.f : x[j];         // (NaN stays)
        }
        RowPiece<T>::store(row, n, a.n_out, x);
    }
}

// Values as the 16 bytes of a piece.
template <typename T>
__device__ __forceinline__ void pack(const float (&x)[RowPiece<T>::P], uint32_t (&w)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 2)
            w[j] = bf16_pair(x[2 * j], x[2 * j + 1]);
        else
            w[j] = __float_as_uint(x[j]);
    }
}

// ONCE: lines that the caches need not keep.
template <bool ONCE>
__device__ __forceinline__ void store_16(void* to, const uint32_t (&w)[4]) {
    typedef uint32_t any4 __attribute__((ext_vector_type(4), aligned(2)));
    const any4 v = {w[0], w[1], w[2], w[3]};
    if constexpr (ONCE)
        __builtin_nontemporal_store(v, static_cast<any4*>(to));
    else
        *static_cast<any4*>(to) = v;
}
// Of two lanes, one `odd`, that CTRL pairs: the odd one gives its a for the other's b.
template <int CTRL>
__device__ __forceinline__ void swap_pieces(bool odd, uint32_t (&a)[4], uint32_t (&b)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t mine = odd ? a[j] : b[j];
        const uint32_t other = uint32_t(__builtin_amdgcn_update_dpp(int(mine), int(mine), CTRL, 0xF, 0xF, false));
        a[j] = odd ? other : a[j];
        b[j] = odd ? b[j] : other;
    }
}

// store_outputs for 16 rows where all the wavefront's outputs are there, nothing is added to and rows lie in whole cache lines: lanes l and l + 8
// of 16 exchange a piece, so that an instruction stores 128 consecutive bytes of 8 rows; the lines need not be kept. c: row 0, `at`: whole_at, rows: from
// row 0 to the last. (bf16, us, so / by 64 bytes / by 64 bytes and not kept: 169,343 x 256 -> 256 25 / 36 / 31, -> 2048 145 / 245 / 211; 2,449,029 x 512
// -> 512 805 / 845 / 1,040; 1,000,000 x 200 -> 136, rows that share lines, by 64 bytes 114, not kept 192. fp32 169,343 x 256 -> 256 42 / 54 / 52.)
template <typename T>
__device__ __forceinline__ int64_t whole_at(int32_t n0, int g, int l, int64_t ldc) {
    return (l & 7) * ldc + n0 + output_of<T>(l < 8 ? 0 : RowPiece<T>::P / 4, 4 * g);
}
template <typename T, int NI>
__device__ __forceinline__ void store_whole_outputs(T* c, int64_t at, int64_t rows, int l, const ScaledArgs& a, const floatx4 (&acc)[NI]) {
    constexpr int P = RowPiece<T>::P, F = P / 4;
    const int left = int(min(rows, int64_t(16)));
    c += at;
#pragma unroll
    for (int k = 0; k < NI / F; k += 2) {
        __builtin_amdgcn_sched_barrier(0);             // (not all pieces at once)
        uint32_t w[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float x[P];
#pragma unroll
            for (int j = 0; j < P; ++j) {
                x[j] = acc[F * (k + h) + j / 4][j % 4];
                if (a.relu) x[j] = x[j] < 0.f ? 0.f : x[j];
            }
            pack<T>(x, w[h]);
        }
        swap_pieces<0x128>(l >= 8, w[0], w[1]);        // row_ror 8
        T* const to = c + output_of<T>(F * k, 0);
        if ((l & 7) < left) store_16<true>(to, w[0]);
        if ((l & 7) + 8 < left) store_16<true>(to + 8 * a.ldc, w[1]);
    }
}

// What the pieces behind the last column of a row are loaded from.
__device__ __attribute__((aligned(16))) const uint8_t zero_piece[16] = {};

// 16 bytes per lane from memory to LDS, lane after lane from `to` on, without a register between (waited for by vmcnt).
__device__ __forceinline__ void copy_to_lds(const uint8_t* from, uint8_t* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
// p or q without a branch: a copy under a branch would count for the lanes that take it only.
__device__ __forceinline__ const uint8_t* either(bool first, const uint8_t* p, const uint8_t* q) {
    uintptr_t x = first ? reinterpret_cast<uintptr_t>(p) : reinterpret_cast<uintptr_t>(q);
    asm volatile("" : "+v"(x));
    return reinterpret_cast<const uint8_t*>(x);
}
// This thread's copies and LDS reads are done, then everybody's.
__device__ __forceinline__ void copies_done() {
    __builtin_amdgcn_s_waitcnt(0x0070);        // vmcnt(0) lgkmcnt(0)
    __syncthreads();
}

// The same with N of the youngest loads, stores and copies still under way (they end in order).
template <int N>
__device__ __forceinline__ void copies_done_but() {
    static_assert(N < 64, "six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Order of a row's 16-byte pieces in LDS: the 16 rows that a fragment takes meet all eight places of a row's 128 bytes. Rows of X are
// consecutive, those of W as output_of has them.
__device__ __forceinline__ int place_x(int row) { return row & 7; }
template <typename T>
__device__ __forceinline__ int place_w(int row) { return sizeof(T) == 2 ? (row & 3) | ((row >> 1) & 4) : row & 7; }

// Long reductions over fewer tiles, and what scaled_big_kernel does not take: tiles of 16 MI WM rows x 64 WN outputs, a block of 128 of the
// reduction at a time through LDS, copied there while the block before is multiplied (two buffers). 128 x 128, two workgroups per compute unit;
// fp32 128 x 256 where that makes 256 tiles and no more padding; 128 x 64 for at most 64 outputs. (us, 128 x 256 / 128 x 128: bf16 300,000 rows 640 -> 128 110 / 65,
// 100,000 rows 1000 -> 1000 231 / 213, 94,484 rows 1024 -> 600 106 / 110; fp32 94,484 rows 1024 -> 512 116 / 125, 100,000 rows 1025 -> 512 157 / 150.)
template <typename T, int WM, int WN, int MI>
__global__ __launch_bounds__(64 * WM * WN, 2) void scaled_tile_kernel(ScaledArgs a, int32_t tiles_n, int32_t tiles, bool whole_lines) {
    constexpr int WAVES = WM * WN, BM = 16 * MI * WM, BN = 64 * WN, NX = BM / 8 / WAVES, NW = BN / 8 / WAVES;
    static_assert(NX * 8 * WAVES == BM && NW * 8 * WAVES == BN, "every wavefront copies as many rows");
    __shared__ __attribute__((aligned(16))) uint8_t x0[BM * BK], w0[BN * BK], x1[BM * BK], w1[BN * BK];       // (apart, so that copies to one pair are not taken to alias reads of the other)
    // tiles are dealt to the 8 XCDs in runs, the tiles of the same rows one after the other: they share X in the L2 of their XCD
    const int32_t run = (tiles + 7) / 8, tile = int32_t(blockIdx.x & 7) * run + int32_t(blockIdx.x >> 3);
    if (int32_t(blockIdx.x >> 3) >= run || tile >= tiles) return;       // whole workgroup
    const int64_t m0 = int64_t(tile / tiles_n) * BM;
    const int32_t n0 = tile % tiles_n * BN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, l = lane & 15;
    const int wm = wave / WN * (16 * MI), wn = wave % WN * 64;
    const int64_t ld = code_ld(a.n_in), lds = scale_ld(a.n_in);
    const int32_t steps = (a.n_in + BK - 1) / BK;
    const int32_t tail = ld % BK == 0 ? BK : int32_t(ld % BK);         // bytes of the last block that there are

    // what a lane copies: piece (lane % 8) of LDS row 8 h' + lane / 8, as bytes from the tile's first row
    const uint8_t* const base_x = a.x + m0 * ld;
    const uint8_t* const base_w = a.w + int64_t(n0) * ld;
    const int last_m = int(min(int64_t(BM), a.n_rows - m0)) - 1, last_n = min(BN, a.n_out - n0) - 1;
    const int sub = lane >> 3, piece_x = 16 * ((lane & 7) ^ sub);
    uint32_t at_x[NX], at_w[NW];
#pragma unroll
    for (int h = 0; h < NX; ++h) at_x[h] = uint32_t(min((wave * NX + h) * 8 + sub, last_m)) * uint32_t(ld) + piece_x;
#pragma unroll
    for (int h = 0; h < NW; ++h) {
        const int r = (wave * NW + h) * 8 + sub;
        at_w[h] = uint32_t(min(r, last_n)) * uint32_t(ld) + 16 * ((lane & 7) ^ place_w<T>(r));
    }
    auto copy = [&](int32_t s, uint8_t* lx, uint8_t* lw) {
        const uint8_t* const x = base_x + int64_t(s) * BK;
        const uint8_t* const w = base_w + int64_t(s) * BK;
        if (s + 1 < steps || tail == BK) {
#pragma unroll
            for (int h = 0; h < NX; ++h) copy_to_lds(x + at_x[h], lx + (wave * NX + h) * 1024);
#pragma unroll
            for (int h = 0; h < NW; ++h) copy_to_lds(w + at_w[h], lw + (wave * NW + h) * 1024);
        } else {
#pragma unroll
            for (int h = 0; h < NX; ++h) copy_to_lds(either(piece_x < tail, x + at_x[h], zero_piece), lx + (wave * NX + h) * 1024);
#pragma unroll
            for (int h = 0; h < NW; ++h)
                copy_to_lds(either(16 * ((lane & 7) ^ place_w<T>((wave * NW + h) * 8 + sub)) < tail, w + at_w[h], zero_piece), lw + (wave * NW + h) * 1024);
        }
    };
    // the scales of four blocks at a time
    const uint8_t* const base_sx = a.x_scales + m0 * lds;
    const int* const from_sw = reinterpret_cast<const int*>(a.w_scales + int64_t(min(n0 + wn, a.n_out - 1) / kCodeBlock) * lds);
    int sx[MI], next_sx[MI], sw = 0;
    auto scales = [&](int32_t s) {
#pragma unroll
        for (int j = 0; j < MI; ++j) next_sx[j] = *reinterpret_cast<const int*>(base_sx + s + uint32_t(min(wm + 16 * j + l, last_m)) * uint32_t(lds));
    };

    floatx4 acc[MI][4];
#pragma unroll
    for (int j = 0; j < MI; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = floatx4(0.f);
    auto fragment = [&](const uint8_t* t, int r, int place) {
        return joined(*reinterpret_cast<const uint4*>(t + r * BK + ((g ^ place) << 4)), *reinterpret_cast<const uint4*>(t + r * BK + (((g + 4) ^ place) << 4)));
    };
    auto multiply = [&](const uint8_t* lx, const uint8_t* lw) {
        if constexpr (sizeof(T) == 2) {
            intx8 fw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) fw[i] = fragment(lw, wn + output_of<T>(i, l), place_w<T>(output_of<T>(i, l)));
            intx8 fx = fragment(lx, wm + l, place_x(l));
#pragma unroll
            for (int j = 0; j < MI; ++j) {
                intx8 next = fx;
                if (j + 1 < MI) next = fragment(lx, wm + 16 * (j + 1) + l, place_x(l));
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[i], fx, acc[j][i], 0, 0, 0, sw, 0, sx[j]);
                fx = next;
                __builtin_amdgcn_sched_barrier(0);         // (one fragment ahead: all of them at once do not fit the registers)
            }
        } else {
            Bf16Fragment fw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) fw[i] = Bf16Fragment(fragment(lw, wn + output_of<T>(i, l), place_w<T>(output_of<T>(i, l))), sw & 255);
            intx8 fx = fragment(lx, wm + l, place_x(l));
#pragma unroll
            for (int j = 0; j < MI; ++j) {
                const Bf16Fragment x(fx, sx[j] & 255);
                if (j + 1 < MI) fx = fragment(lx, wm + 16 * (j + 1) + l, place_x(l));
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[i].f[q], x.f[q], acc[j][i], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    auto block = [&](int32_t s, const uint8_t* lx, const uint8_t* lw, uint8_t* next_x, uint8_t* next_w) {
        copies_done();
        if ((s & 3) == 0) {
            sw = from_sw[s >> 2];
#pragma unroll
            for (int j = 0; j < MI; ++j) sx[j] = next_sx[j];
        } else {
            sw = int(uint32_t(sw) >> 8);
#pragma unroll
            for (int j = 0; j < MI; ++j) sx[j] = int(uint32_t(sx[j]) >> 8);
        }
        if (s + 1 < steps) {
            if ((s & 3) == 3) scales(s + 1);
            copy(s + 1, next_x, next_w);
        }
        multiply(lx, lw);
    };
    scales(0);
    copy(0, x0, w0);
    for (int32_t s = 0; s < steps; s += 2) {
        block(s, x0, w0, x1, w1);
        if (s + 1 < steps) block(s + 1, x1, w1, x0, w0);
    }
    const int64_t at_c = whole_at<T>(n0 + wn, g, l, a.ldc);
#pragma unroll
    for (int j = 0; j < MI; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(acc[j][i]));
        const int64_t row = m0 + wm + 16 * j;
        if (whole_lines) {
            if (n0 + wn < a.n_out) store_whole_outputs(static_cast<T*>(a.c) + row * a.ldc, at_c, a.n_rows - row, l, a, acc[j]);
        } else if (row + l < a.n_rows) {
            store_outputs(static_cast<T*>(a.c) + (row + l) * a.ldc, n0 + wn, g, a, acc[j]);
        }
    }
}

// Long reductions over many tiles, bf16 results: 256 x 256 outputs per workgroup, 128 x 128 per wavefront (one per SIMD, so that a
// fragment from LDS is used four times), v_mfma_scale_f32_32x32x64_f8f6f4. A workgroup takes tile after tile and never stops in between:
// a block of 128 of the reduction is copied while the one before is multiplied, also into the next tile, most fragments of the next 64 are
// read while the second half of the present 64 is multiplied, and the stores of a tile are under way during the next one's first block.
// The last tiles are moved back to end with the last row and output, so nothing is masked; elements in two tiles are stored twice, the same
// value. (Hence not where c is added to. Reductions are whole 256: two buffers.)
// Weight row [q1 h q0 v1 v0] (bits) of a fragment's 32 is output [q1 q0 h v1 v0] of it: accumulators 4 q + v, q = 0, 1 and 2, 3, of a lane are
// then 8 consecutive outputs.
// 262,181 x 2048 -> 2048: 1,110 to 1,250 us, 1,760 to 1,980 TFLOP/s (it varies with what is multiplied: 1,130 over rows of normal numbers, 1,205 over random
// codes); 131,072 x 8192 -> 2048 1,805 to 1,995 us, 2,430 TFLOP/s at best. Tiles that start anew (scaled_tile_kernel, 8 wavefronts of 128 x 64): 1,305 and
// 2,160. With all copies of a block in a row 1,310: a wavefront that issues
// a copy waits until the one before is taken, and issues no product meanwhile. Without copies 900: what bounds it is the L2, 8.5 TB/s.
typedef float floatx16 __attribute__((ext_vector_type(16)));
constexpr int kBigTile = 256, kBigBuffer = 2 * kBigTile * BK;

__global__ __launch_bounds__(kThreads, 1) void scaled_big_kernel(ScaledArgs a, int32_t tiles_n, int32_t tiles, bool whole_lines) {
    using T = bf16_t;
    __shared__ __attribute__((aligned(16))) uint8_t b0[kBigBuffer], b1[kBigBuffer];      // (apart: see scaled_tile_kernel)
    // runs of tiles for the 8 XCDs; the workgroups of an XCD take them in turn, so that those at work together lie side by side
    const int32_t run = (tiles + 7) / 8, stride = int32_t(gridDim.x >> 3);
    const int32_t end = min(tiles, (int32_t(blockIdx.x & 7) + 1) * run);
    int32_t tile = int32_t(blockIdx.x & 7) * run + int32_t(blockIdx.x >> 3);
    if (tile >= end) return;                            // whole workgroup
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 31, half = lane >> 5;
    const int wm = (wave >> 1) * 128, wn = (wave & 1) * 128;
    const int64_t ld = code_ld(a.n_in), lds = scale_ld(a.n_in);
    const int32_t blocks = a.n_in / BK;
    auto first_row = [&](int32_t t) { return min(int64_t(t / tiles_n) * kBigTile, a.n_rows - kBigTile); };
    auto first_output = [&](int32_t t) { return min(t % tiles_n * kBigTile, a.n_out - kBigTile); };

    // copies, 8 rows by an instruction: piece (lane % 8) of row lane / 8, in the order of place_x
    int32_t copy_tile = tile, copy_block = 0;
    const uint8_t* copy_x = a.x + first_row(tile) * ld;
    const uint8_t* copy_w = a.w + int64_t(first_output(tile)) * ld;
    const uint32_t at = uint32_t(wave * 64 + (lane >> 3)) * uint32_t(ld) + 16 * ((lane & 7) ^ (lane >> 3));
    auto copy_x_rows = [&](uint8_t* to, int h) { copy_to_lds(copy_x + h * 8 * ld + at, to + wave * 8192 + h * 1024); };
    auto copy_w_rows = [&](uint8_t* to, int h) { copy_to_lds(copy_w + h * 8 * ld + at, to + kBigTile * BK + wave * 8192 + h * 1024); };
    auto copied = [&]() {                               // (behind the last tile: that one again)
        copy_x += BK, copy_w += BK;
        if (++copy_block == blocks) {
            copy_tile = min(copy_tile + stride, end - 1), copy_block = 0;
            copy_x = a.x + first_row(copy_tile) * ld, copy_w = a.w + int64_t(first_output(copy_tile)) * ld;
        }
    };
    const int row_w = (l & 0x13) | ((l & 4) << 1) | ((l & 8) >> 1);
    auto fragment = [&](const uint8_t* row, int part, int place) {
        return joined(*reinterpret_cast<const uint4*>(row + (((4 * part + half) ^ place) << 4)), *reinterpret_cast<const uint4*>(row + (((4 * part + half + 2) ^ place) << 4)));
    };
    auto read_w = [&](const uint8_t* b, int part, int i) { return fragment(b + (kBigTile + wn + 32 * i + row_w) * BK, part, row_w & 7); };
    auto read_x = [&](const uint8_t* b, int part, int j) { return fragment(b + (wm + 32 * j + l) * BK, part, l & 7); };
    // the scales of four blocks, of the present one on (in the low byte) and of the next four
    int sx[4], next_sx[4], sw[4], next_sw[4];
    auto scales = [&](int32_t t, int32_t block) {
        const uint8_t* const x = a.x_scales + first_row(t) * lds + block;
        const uint8_t* const w = a.w_scales + block;
        const int32_t n0 = first_output(t) + wn + row_w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            next_sx[j] = *reinterpret_cast<const int*>(x + uint32_t(wm + 32 * j + l) * uint32_t(lds));
            next_sw[j] = *reinterpret_cast<const int*>(w + uint32_t((n0 + 32 * j) / kCodeBlock) * uint32_t(lds));
        }
    };

    const float least = a.relu ? 0.f : -INFINITY;
    floatx16 acc[4][4];
    intx8 w[4], x0[4], x1[4];
    auto multiply = [&](int i, const intx8 (&x)[4], auto after) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[i], x[j], acc[i][j], 0, 0, 0, sw[i], 0, sx[j]);
            asm volatile("" : "+a"(acc[i][j]));         // (here and not further down, where the fragments would have to be kept for it)
            after(j);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // A lane holds four of the eight pieces of 64 outputs of a row, lane + 32 the others; four neighbours exchange them, so that an instruction stores
    // 128 consecutive bytes of 8 rows. (32 bytes of 32 rows, as the accumulators lie: 16,384 x 4096 -> 4096 257 us, 235 so.)
    const int64_t c_lane = int64_t(l & ~3) * a.ldc + 16 * (l & 3) + 8 * half;
    auto store_tile = [&](T* c) __attribute__((always_inline)) {
        c += c_lane;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                uint32_t p[4][4];                           // pieces of the row
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[e] = acc[i + (h >> 1)][j][8 * (h & 1) + e];
                        v[e] = v[e] < least ? least : v[e];               // (NaN stays)
                    }
                    pack<T>(v, p[h]);
                }
                swap_pieces<0xB1>(l & 1, p[0], p[1]), swap_pieces<0xB1>(l & 1, p[2], p[3]);
                swap_pieces<0x4E>(l & 2, p[0], p[2]), swap_pieces<0x4E>(l & 2, p[1], p[3]);
                auto store = [&](auto once) {
#pragma unroll
                    for (int h = 0; h < 4; ++h) store_16<decltype(once)::value>(c + 32 * i + h * a.ldc, p[h]);
                };
                if (whole_lines)
                    store(std::true_type{});
                else
                    store(std::false_type{});
                __builtin_amdgcn_sched_barrier(0);
            }
            c += 32 * a.ldc;
        }
    };
    auto nothing = [](int) {};
    // The copies of the block after the next go where this one lay, once everybody has read it: its X behind the products of the last
    // quarter, its W behind those of the next block's first, one each, so that no product waits for a row of copies to be taken.
    auto block = [&](int32_t s, uint8_t* from, uint8_t* other) __attribute__((always_inline)) {
        if ((s & 3) == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) sx[j] = next_sx[j], sw[j] = next_sw[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) sx[j] = int(uint32_t(sx[j]) >> 8), sw[j] = int(uint32_t(sw[j]) >> 8);
        }
        const bool last = s + 1 == blocks;
        if (last || (s & 3) == 3) scales(last ? min(tile + stride, end - 1) : tile, last ? 0 : s + 1);
        multiply(0, x0, [&](int j) { copy_w_rows(other, j); });
        w[2] = read_w(from, 0, 2), w[3] = read_w(from, 0, 3);
        __builtin_amdgcn_sched_barrier(0);
        multiply(1, x0, [&](int j) { copy_w_rows(other, 4 + j); });
        copied();
        w[0] = read_w(from, 1, 0), w[1] = read_w(from, 1, 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) x1[j] = read_x(from, 1, j);
        __builtin_amdgcn_sched_barrier(0);
        multiply(2, x0, nothing);
        multiply(3, x0, nothing);
        multiply(0, x1, nothing);
        w[2] = read_w(from, 1, 2), w[3] = read_w(from, 1, 3);
        __builtin_amdgcn_sched_barrier(0);
        multiply(1, x1, nothing);
        copies_done_but<0>();                           // the next block's; and everybody has read this one
        w[0] = read_w(other, 0, 0), w[1] = read_w(other, 0, 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) x0[j] = read_x(other, 0, j);
        __builtin_amdgcn_sched_barrier(0);
        multiply(2, x1, [&](int j) { copy_x_rows(from, j); });
        multiply(3, x1, [&](int j) { copy_x_rows(from, 4 + j); });
    };
    scales(tile, 0);
#pragma unroll
    for (int h = 0; h < 8; ++h) copy_x_rows(b0, h), copy_w_rows(b0, h);
    copied();
#pragma unroll
    for (int h = 0; h < 8; ++h) copy_x_rows(b1, h);
    copies_done_but<0>();
    w[0] = read_w(b0, 0, 0), w[1] = read_w(b0, 0, 1);
#pragma unroll
    for (int j = 0; j < 4; ++j) x0[j] = read_x(b0, 0, j);
    for (; tile < end; tile += stride) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = floatx16(0.f);
#pragma clang loop unroll(disable)
        for (int32_t s = 0; s < blocks; s += 2) {
            block(s, b0, b1);
            block(s + 1, b1, b0);
        }
        store_tile(static_cast<T*>(a.c) + (first_row(tile) + wm) * a.ldc + first_output(tile) + wn);
    }
}

// Long reductions over few rows, where the tiles above would leave most compute units idle and each of theirs would wait for one block of the reduction
// after the other: 16 M rows x 16 N outputs per workgroup, its eight wavefronts take every eighth block of 128, fragments straight from memory, and
// join their sums in LDS in one order. Every workgroup reads its rows and weights anew: tiles of 32 x 32 up to 512 workgroups, of 64 x 64 up to 256. (us, 32 /
// 64 / the tiles above: 1 row 2048 -> 2048 7.9 / 11.6 / 13.5, fp32 7.9 / 12.3 / 19.6; 1 row 16,384 -> 4096 26 / - / 92; 200 rows 2048 -> 2048 11.1 / 11.8 /
// 14; 300 14.8 / 11.7 / 16.5; 500 19.3 / 12.0 / 16.7; 1,000, 512 workgroups of 64 x 64, 36 / 22.6 / 17.5; 1,000 rows 8192 -> 1000 - / 39 / 54.)
template <typename T, int M, int N>
__global__ __launch_bounds__(512) void scaled_few_kernel(ScaledArgs a) {
    constexpr int WAVES = 8, F = RowPiece<T>::P / 4;
    __shared__ floatx4 sums[WAVES][M][N][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, l = lane & 15;
    const int64_t m0 = int64_t(blockIdx.y) * (16 * M), ld = code_ld(a.n_in), lds = scale_ld(a.n_in);
    const int32_t n0 = int32_t(blockIdx.x) * (16 * N), steps = (a.n_in + BK - 1) / BK;
    const uint8_t *x[M], *w[N], *sx[M];
#pragma unroll
    for (int j = 0; j < M; ++j) {
        const int64_t row = min(m0 + 16 * j + l, a.n_rows - 1);
        x[j] = a.x + row * ld, sx[j] = a.x_scales + row * lds;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = a.w + int64_t(min(n0 + output_of<T>(i, l), a.n_out - 1)) * ld;
    const uint8_t* const sw = a.w_scales + int64_t(n0 / kCodeBlock) * lds;
    floatx4 acc[M][N];
#pragma unroll
    for (int j = 0; j < M; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) acc[j][i] = floatx4(0.f);
    auto fragment = [&](const uint8_t* row, int32_t s) {
        const int64_t k = int64_t(s) * BK + 16 * g;
        uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
        if (k < ld) lo = *reinterpret_cast<const uint4*>(row + k);
        if (k + 64 < ld) hi = *reinterpret_cast<const uint4*>(row + k + 64);
        return joined(lo, hi);
    };
#pragma unroll 2
    for (int32_t s = wave; s < steps; s += WAVES) {
        intx8 fx[M], fw[N];
        int scale_x[M];
#pragma unroll
        for (int i = 0; i < N; ++i) fw[i] = fragment(w[i], s);
#pragma unroll
        for (int j = 0; j < M; ++j) fx[j] = fragment(x[j], s), scale_x[j] = sx[j][s];
        const int scale_w = sw[s];
#pragma unroll
        for (int j = 0; j < M; ++j)
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int i = 0; i < N; ++i) acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[i], fx[j], acc[j][i], 0, 0, 0, scale_w, 0, scale_x[j]);
            } else {
                const Bf16Fragment bx(fx[j], scale_x[j]);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const Bf16Fragment bw(fw[i], scale_w);
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw.f[q], bx.f[q], acc[j][i], 0, 0, 0);
                }
            }
    }
#pragma unroll
    for (int j = 0; j < M; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) sums[wave][j][i][lane] = acc[j][i];
    __syncthreads();
    for (int piece = wave; piece < M * N / F; piece += WAVES) {
        const int j = piece / (N / F), i = piece % (N / F) * F;
        floatx4 sum[F];
#pragma unroll
        for (int f = 0; f < F; ++f) {
            sum[f] = sums[0][j][i + f][lane];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) sum[f] += sums[v][j][i + f][lane];
        }
        const int64_t row = m0 + 16 * j + l;
        if (row < a.n_rows) store_outputs(static_cast<T*>(a.c) + row * a.ldc, n0 + 16 * i, g, a, sum);
    }
}

// Short reductions (512 at most): bound by reading X and writing c. A wavefront keeps the weights of 16 NI outputs in registers
// and the workgroup walks over rows, 16 R WR at a time, which are copied to LDS D - 1 steps ahead. WN wavefronts take the same rows, their
// other outputs. (NI: 4; 2 where fp32 results take more than 256 columns, whose weights are kept as bf16, twice the registers.)
// Loads and stores are counted together and end in order: a wavefront waits until no more of them are under way than were
// started after the copies it needs, (D - 2) steps' copies and (D - 1) steps' stores; less may be under way than that only
// in the first steps and in wavefronts that store by elements, or nothing, which wait until their stores are through as well. Every step starts
// copies, of the last rows again where there are no more, so that the count holds to the end.
// (The empty assembly keeps the products in front of the stores' branches: under a branch the lanes that do not take it would
// supply nothing to the matrix instruction.)
// 2,449,029 x 512 -> 512 bf16: 805 us, 4.7 TB/s (rows requested into registers one step ahead 1,588; 128 x 128 tiles 1,446); 169,343 x 256 -> 256
// bf16 25 us (51; 41), fp32 42 us (82; 64). WHOLE: the rows of c are what store_whole_outputs takes.
template <typename T, int KB, int NI, int WN, int R>
struct RowsLayout {
    static constexpr int WR = kThreads / 64 / WN, ROWS = 16 * R * WR, COPIES = KB * ROWS * BK / 1024 / 4 + 1, STORES = R * NI * 4 / RowPiece<T>::P;
    static constexpr int BYTES = KB * ROWS * BK + 4 * 256;
    static constexpr int D = BYTES > 24 * 1024 ? 3 : 4;
    static constexpr int BUSY = (D - 2) * COPIES + (D - 1) * STORES;
    static_assert(BUSY < 64 && ROWS <= 64 && KB * ROWS % 32 == 0, "");
};
template <typename T, int KB, int NI, int WN, int R, bool WHOLE>
__global__ __launch_bounds__(kThreads, (RowsLayout<T, KB, NI, WN, R>::D * RowsLayout<T, KB, NI, WN, R>::BYTES > 80 * 1024 ? 1 : 2)) void scaled_rows_kernel(ScaledArgs a) {
    using L = RowsLayout<T, KB, NI, WN, R>;
    constexpr int WR = L::WR, ROWS = L::ROWS, D = L::D, PER_WAVE = L::COPIES - 1;
    __shared__ __attribute__((aligned(16))) uint8_t b0[L::BYTES], b1[L::BYTES], b2[L::BYTES], b3[D > 3 ? L::BYTES : 16];       // (apart: see scaled_tile_kernel)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, l = lane & 15;
    const int32_t n0 = (int32_t(blockIdx.y) * WN + wave % WN) * (16 * NI);
    const int wr = wave / WN * (16 * R);
    const uint32_t ld = uint32_t(code_ld(a.n_in));
    const int64_t step = int64_t(gridDim.x) * ROWS, first = int64_t(blockIdx.x) * ROWS;

    // a kilobyte of copies is eight rows of one block of 128 columns: rows 8 (q % (ROWS / 8)) + lane / 8 of block q / (ROWS / 8)
    const int sub = lane >> 3, piece = 16 * ((lane & 7) ^ sub);
    auto copy = [&](int64_t r0, uint8_t* to) {
        const int64_t base = min(r0, a.n_rows - 1);
        const int last = int(min(int64_t(ROWS), a.n_rows - base)) - 1;
        const uint8_t* const x = a.x + base * ld;
#pragma unroll
        for (int h = 0; h < PER_WAVE; ++h) {
            const int q = wave * PER_WAVE + h, kb = q / (ROWS / 8), row = q % (ROWS / 8) * 8 + sub;
            const uint32_t k = kb * kCodeBlock + piece;
            copy_to_lds(either(k < ld, x + (uint32_t(min(row, last)) * ld + k), zero_piece), to + q * 1024);
        }
        const uint8_t* const sc = a.x_scales + (base + min(lane, last)) * 4;         // (a scale row is 4 bytes: 512 columns at most)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)sc,
                                         (__attribute__((address_space(3))) void*)(to + KB * ROWS * BK + wave * 256), 4, 0, 0);
    };
    copy(first, b0);
    copy(first + step, b1);
    if constexpr (D > 3) copy(first + 2 * step, b2);

    intx8 fw[NI][KB];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const uint8_t* const row = a.w + int64_t(min(n0 + output_of<T>(i, l), a.n_out - 1)) * ld;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const uint32_t k = kb * kCodeBlock + g * 16;
            uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
            if (k < ld) lo = *reinterpret_cast<const uint4*>(row + k);
            if (k + 64 < ld) hi = *reinterpret_cast<const uint4*>(row + k + 64);
            fw[i][kb] = joined(lo, hi);
        }
    }
    const int scale_w = *reinterpret_cast<const int*>(a.w_scales + int64_t(min(n0, a.n_out - 1) / kCodeBlock) * 4);
    const bool regular = n0 + 16 * NI <= a.n_out;
    int filled = 0;                                     // steps that have stored
    const int64_t at = whole_at<T>(n0, g, l, a.ldc);

    auto walk = [&](int64_t r0, const uint8_t* now, uint8_t* next) {
        if (regular && filled >= D - 1)
            copies_done_but<L::BUSY>();
        else
            copies_done_but<(D - 2) * L::COPIES>();
        ++filled;
        copy(r0 + (D - 1) * step, next);
        floatx4 acc[R][NI];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < NI; ++i) acc[r][i] = floatx4(0.f);
        int scale_x[R];
#pragma unroll
        for (int r = 0; r < R; ++r) scale_x[r] = *reinterpret_cast<const int*>(now + KB * ROWS * BK + wave * 256 + (wr + 16 * r + l) * 4);
        auto multiply = [&](auto block) {
            constexpr int kb = decltype(block)::value;
            auto fragment = [&](int r) {
                const uint8_t* const row = now + kb * ROWS * BK + (wr + 16 * r + l) * BK;
                return joined(*reinterpret_cast<const uint4*>(row + ((g ^ place_x(l)) << 4)), *reinterpret_cast<const uint4*>(row + (((g + 4) ^ place_x(l)) << 4)));
            };
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if constexpr (sizeof(T) == 2) {
                    const intx8 fx = fragment(r);
#pragma unroll
                    for (int i = 0; i < NI; ++i)
                        acc[r][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[i][kb], fx, acc[r][i], 0, 0, kb, scale_w, kb, scale_x[r]);
                } else {
                    const Bf16Fragment x(fragment(r), (scale_x[r] >> (8 * kb)) & 255);
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        const Bf16Fragment w(fw[i][kb], (scale_w >> (8 * kb)) & 255);
#pragma unroll
                        for (int q = 0; q < 4; ++q) acc[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.f[q], x.f[q], acc[r][i], 0, 0, 0);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        multiply(std::integral_constant<int, 0>{});
        if constexpr (KB > 1) multiply(std::integral_constant<int, 1>{});
        if constexpr (KB > 2) multiply(std::integral_constant<int, 2>{});
        if constexpr (KB > 3) multiply(std::integral_constant<int, 3>{});
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int i = 0; i < NI; ++i) asm volatile("" : "+v"(acc[r][i]));
            if constexpr (WHOLE) {
                __builtin_amdgcn_sched_barrier(0);
                const int64_t row = r0 + wr + 16 * r;
                if (regular) store_whole_outputs(static_cast<T*>(a.c) + row * a.ldc, at, a.n_rows - row, l, a, acc[r]);
                __builtin_amdgcn_sched_barrier(0);
            } else {
                const int64_t row = r0 + wr + 16 * r + l;
                if (row < a.n_rows) store_outputs(static_cast<T*>(a.c) + row * a.ldc, n0, g, a, acc[r]);
            }
        }
    };
    for (int64_t r0 = first; r0 < a.n_rows;) {
        walk(r0, b0, D > 3 ? b3 : b2);
        if ((r0 += step) >= a.n_rows) break;
        walk(r0, b1, b0);
        if ((r0 += step) >= a.n_rows) break;
        walk(r0, b2, b1);
        if constexpr (D > 3) {
            if ((r0 += step) >= a.n_rows) break;
            walk(r0, b3, b2);
        }
        r0 += step;
    }
}

}  // namespace

hipError_t varco_launch_scaled_transform(int dtype, const ScaledArgs& a, hipStream_t stream) {
    auto with_type = [&](auto type) {
        using T = decltype(type);
        const int32_t blocks = (a.n_in + kCodeBlock - 1) / kCodeBlock;
        const bool whole_lines = !a.accumulate && a.ldc * int64_t(sizeof(T)) % 128 == 0 && reinterpret_cast<uintptr_t>(a.c) % 128 == 0;
        if (blocks > 4) {
            auto tile = [&](auto wm, auto wn, auto mi) {
                constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, MI = decltype(mi)::value;
                const int64_t tiles_n = (a.n_out + 64 * WN - 1) / (64 * WN), tiles = (a.n_rows + 16 * MI * WM - 1) / (16 * MI * WM) * tiles_n;
                hipLaunchKernelGGL((scaled_tile_kernel<T, WM, WN, MI>), dim3(unsigned((tiles + 7) / 8 * 8)), dim3(64 * WM * WN), 0, stream, a, int32_t(tiles_n),
                                   int32_t(tiles), whole_lines && a.n_out % 64 == 0);
            };
            using std::integral_constant;
            const int64_t big_n = (a.n_out + kBigTile - 1) / kBigTile, big = (a.n_rows + kBigTile - 1) / kBigTile * big_n;
            auto few = [&](auto m, int64_t most) {
                constexpr int M = decltype(m)::value;
                const int64_t few_n = (a.n_out + 16 * M - 1) / (16 * M), few_m = (a.n_rows + 16 * M - 1) / (16 * M);
                if (few_n * few_m > most) return false;
                hipLaunchKernelGGL((scaled_few_kernel<T, M, M>), dim3(unsigned(few_n), unsigned(few_m)), dim3(512), 0, stream, a);
                return true;
            };
            if (few(integral_constant<int, 2>{}, 512) || few(integral_constant<int, 4>{}, 256)) return;
            if (a.n_out <= 64)
                tile(integral_constant<int, 4>{}, integral_constant<int, 1>{}, integral_constant<int, 2>{});
            else if (sizeof(T) == 2 && big >= 256 && a.n_rows >= kBigTile && a.n_out >= kBigTile && a.n_in % (2 * BK) == 0 && !a.accumulate)
                hipLaunchKernelGGL(scaled_big_kernel, dim3(256), dim3(kThreads), 0, stream, a, int32_t(big_n), int32_t(big), whole_lines && a.n_out % 64 == 0);
            else if (sizeof(T) == 4 && 2 * big >= 256 && (a.n_out + 127) / 128 % 2 == 0)
                tile(integral_constant<int, 2>{}, integral_constant<int, sizeof(T) == 4 ? 4 : 2>{}, integral_constant<int, 4>{});
            else
                tile(integral_constant<int, 2>{}, integral_constant<int, 2>{}, integral_constant<int, 4>{});
            return;
        }
        auto launch = [&](auto kb, auto wn) {
            constexpr int KB = decltype(kb)::value, WN = decltype(wn)::value, R = WN == 4 ? 2 : 1;
            constexpr int NI = sizeof(T) == 4 && KB > 2 ? 2 : 4;
            using L = RowsLayout<T, KB, NI, WN, R>;
            const int64_t columns = (a.n_out + 16 * NI * WN - 1) / (16 * NI * WN), steps = (a.n_rows + L::ROWS - 1) / L::ROWS;
            // workgroups that are resident together, all columns of the same rows on one XCD (a multiple of 8 in a row of the grid)
            constexpr int kResident = std::max(1, std::min(KB <= 2 && sizeof(T) == 2 ? 3 : 2, 160 * 1024 / (L::D * L::BYTES)));
            const int64_t groups = std::min(steps, std::max<int64_t>(8, 256 * kResident / columns / 8 * 8));
            const dim3 grid{unsigned(groups), unsigned(columns)};
            if (whole_lines && a.n_out % (16 * NI) == 0)
                hipLaunchKernelGGL((scaled_rows_kernel<T, KB, NI, WN, R, true>), grid, dim3(kThreads), 0, stream, a);
            else
                hipLaunchKernelGGL((scaled_rows_kernel<T, KB, NI, WN, R, false>), grid, dim3(kThreads), 0, stream, a);
        };
        auto with_outputs = [&](auto kb) {
            if (a.n_out <= 64)
                launch(kb, std::integral_constant<int, 1>{});
            else if (a.n_out <= 128)
                launch(kb, std::integral_constant<int, 2>{});
            else
                launch(kb, std::integral_constant<int, 4>{});
        };
        if (blocks == 1)
            with_outputs(std::integral_constant<int, 1>{});
        else if (blocks == 2)
            with_outputs(std::integral_constant<int, 2>{});
        else if (blocks == 3)
            with_outputs(std::integral_constant<int, 3>{});
        else
            with_outputs(std::integral_constant<int, 4>{});
    };
    if (dtype == VARCO_BF16)
        with_type(bf16_t{});
    else
        with_type(float{});
    return hipGetLastError();
}
