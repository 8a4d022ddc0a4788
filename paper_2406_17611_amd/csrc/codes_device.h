// Rows of 8-bit codes: numbers of 4 exponent and 3 fraction bits (e4m3: no infinity, one NaN, largest 448), and a power of
// two for each 128 columns of a row as their scale, stored as its exponent + 127 in a byte. A power of two costs no bits
// of a floating number inside its range, and it is the form of scale that the matrix units apply by themselves.
#pragma once

#include "elem.h"

constexpr int kCodeBlock = 128;                        // columns (of weights: rows and columns) of a scale
constexpr int kOneScale = 127;                         // the byte of scale 1
inline __host__ __device__ int64_t code_ld(int64_t width) { return (width + 15) / 16 * 16; }        // VARCO_CODE_LD
inline __host__ __device__ int64_t scale_ld(int64_t width) { return (width + 511) / 512 * 4; }      // VARCO_SCALE_LD

// Smallest e with a 2^-e <= 448 = 1.75 2^8, at least -127, for finite a >= 0; 0 for a = 0. (Numbers below 2^-126 have a
// zero exponent field: the limit is theirs whatever it says.)
__device__ __forceinline__ int code_exponent(float a) {
    const int bits = int(__float_as_uint(a));
    const int e = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0);
    return bits == 0 ? 0 : max(e, -127);
}
// 2^-e for -127 <= e <= 126.
__device__ __forceinline__ float code_inverse(int e) { return __uint_as_float(uint32_t(127 - e) << 23); }

__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }
// |x|, 0 for what is not finite: one such element does not take the other 127 of its block along.
__device__ __forceinline__ float finite_size(float x) { return is_finite(x) ? fabsf(x) : 0.f; }

// Four codes of values that `inverse` brings to 448 at most; infinities and NaN become the code of NaN.
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d, float inverse) {
    auto in = [inverse](float x) { return is_finite(x) ? x * inverse : __uint_as_float(0x7FC00000u); };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(in(a), in(b), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(in(c), in(d), w, true);
    return uint32_t(w);
}

// Lanes of a wavefront combined by data paths of the vector ALU: every lane gets the result over its group of N lanes
// (N = 1, 2, 4, .., 64, groups aligned), the same bits in all of them.
template <int CTRL>
__device__ __forceinline__ float other_lane(float x) {
    const int u = int(__float_as_uint(x));
    return __uint_as_float(uint32_t(__builtin_amdgcn_update_dpp(u, u, CTRL, 0xF, 0xF, false)));
}
template <int CTRL>
__device__ __forceinline__ double other_lane(double x) {
    const auto u = __builtin_bit_cast(uint64_t, x);
    const auto half = [](uint32_t v) { return uint32_t(__builtin_amdgcn_update_dpp(int(v), int(v), CTRL, 0xF, 0xF, false)); };
    return __builtin_bit_cast(double, uint64_t(half(uint32_t(u >> 32))) << 32 | half(uint32_t(u)));
}
// f of the numbers that the two halves of 32 (WIDE: of 64) lanes hold.
template <bool WIDE, typename F>
__device__ __forceinline__ float over_halves(float x, F f) {
    const uint32_t u = __float_as_uint(x);
    const auto r = WIDE ? __builtin_amdgcn_permlane32_swap(u, u, false, false) : __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <bool WIDE, typename F>
__device__ __forceinline__ double over_halves(double x, F f) {
    const auto u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = uint32_t(u), hi = uint32_t(u >> 32);
    const auto r = WIDE ? __builtin_amdgcn_permlane32_swap(lo, lo, false, false) : __builtin_amdgcn_permlane16_swap(lo, lo, false, false);
    const auto s = WIDE ? __builtin_amdgcn_permlane32_swap(hi, hi, false, false) : __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
    return f(__builtin_bit_cast(double, uint64_t(s[0]) << 32 | r[0]), __builtin_bit_cast(double, uint64_t(s[1]) << 32 | r[1]));
}
template <int N, typename S, typename F>
__device__ __forceinline__ S over_lanes(S x, F f) {
    if (N >= 2) x = f(x, other_lane<0xB1>(x));          // quad_perm 1 0 3 2
    if (N >= 4) x = f(x, other_lane<0x4E>(x));          // quad_perm 2 3 0 1
    if (N >= 8) x = f(x, other_lane<0x141>(x));         // row_half_mirror: the other four lanes of eight
    if (N >= 16) x = f(x, other_lane<0x140>(x));        // row_mirror: the other eight of sixteen
    if (N >= 32) x = over_halves<false>(x, f);
    if (N >= 64) x = over_halves<true>(x, f);
    return x;
}
template <int N, typename S>
__device__ __forceinline__ S lanes_sum(S x) {
    return over_lanes<N>(x, [](S a, S b) { return a + b; });
}
template <int N>
__device__ __forceinline__ float lanes_max(float x) {
    return over_lanes<N>(x, [](float a, float b) { return fmaxf(a, b); });
}

// A row in pieces of 16 bytes of its storage type, converted to fp32, from any address of an element. ANY: of any length; the piece that
// the last column ends in is loaded from before it, so that it does not leave the row, and moved down; by how much is the same in
// all lanes. (1,000,000 bf16 rows of 47, norm and codes 91 us; 160 with the last piece by elements.) Else of whole pieces. ONCE: with the hint that
// the caches need not keep it, where a kernel reads or writes far more than they hold (kernels_clip.hip, kernels_norm.hip have the figures).
template <typename T>
struct RowPiece {
    static constexpr int P = 16 / int(sizeof(T));
    template <bool ANY = true, bool ONCE = false>
    static __device__ __forceinline__ void load(const T* row, int32_t at, int32_t width, float (&v)[P]) {
        if constexpr (!ANY) {
            const uint4 u = at < width ? load_16<ONCE>(row + at) : make_uint4(0u, 0u, 0u, 0u);
            convert(u.x, u.y, u.z, u.w, v);
            return;
        }
        if (width < P) {
#pragma unroll
            for (int i = 0; i < P; ++i) v[i] = at + i < width ? Elem<T>::load(row + at + i) : 0.f;
            return;
        }
        const uint4 u = load_16<ONCE>(row + min(at, width - P));
        uint32_t w[4] = {u.x, u.y, u.z, u.w};
        const int by = width % P ? P - width % P : 0;
        if (by) {
            if constexpr (sizeof(T) == 2) {
                const uint4 m = moved_up8(u, by);
                const bool ends = at + P > width;
                w[0] = ends ? m.x : w[0], w[1] = ends ? m.y : w[1], w[2] = ends ? m.z : w[2], w[3] = ends ? m.w : w[3];
            } else {
                if (at + P > width) {
                    w[0] = by == 1 ? w[1] : by == 2 ? w[2] : w[3];
                    w[1] = by == 1 ? w[2] : by == 2 ? w[3] : 0u;
                    w[2] = by == 1 ? w[3] : 0u;
                    w[3] = 0u;
                }
            }
        }
        const bool none = at >= width;
        convert(none ? 0u : w[0], none ? 0u : w[1], none ? 0u : w[2], none ? 0u : w[3], v);
    }
    static __device__ __forceinline__ void convert(uint32_t x, uint32_t y, uint32_t z, uint32_t t, float (&v)[P]) {
        const uint32_t w[4] = {x, y, z, t};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 2)
                v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            else
                v[i] = __uint_as_float(w[i]);
        }
    }
    template <bool ONCE>
    static __device__ __forceinline__ uint4 load_16(const T* p) {
        typedef uint32_t any4 __attribute__((ext_vector_type(4), aligned(2)));
        const any4 u = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const any4*>(p)) : *reinterpret_cast<const any4*>(p);
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
    template <bool ANY = true, bool ONCE = false>
    static __device__ __forceinline__ void store(T* row, int32_t at, int32_t width, const float (&v)[P]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 2)
                w[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
            else
                w[i] = __float_as_uint(v[i]);
        }
        if (at + P <= width) {
            typedef uint32_t any4 __attribute__((ext_vector_type(4), aligned(2)));
            if constexpr (ONCE)
                __builtin_nontemporal_store(any4{w[0], w[1], w[2], w[3]}, reinterpret_cast<any4*>(row + at));
            else
                *reinterpret_cast<any4*>(row + at) = any4{w[0], w[1], w[2], w[3]};
        } else if (ANY && at < width) {                // what is left, by its binary digits (the same in all lanes)
            typedef uint32_t any2 __attribute__((ext_vector_type(2), aligned(2)));
            typedef uint32_t any1 __attribute__((aligned(2)));
            const int left = width % P;
            T* const p = row + at;
            if constexpr (sizeof(T) == 2) {
                if (left & 4) *reinterpret_cast<any2*>(p) = any2{w[0], w[1]};
                if (left & 2) *reinterpret_cast<any1*>(p + (left & 4)) = left & 4 ? w[2] : w[0];
                if (left & 1) p[left - 1].bits = uint16_t(left == 1 ? w[0] : left == 3 ? w[1] : left == 5 ? w[2] : w[3]);
            } else {
                if (left & 2) *reinterpret_cast<any2*>(p) = any2{w[0], w[1]};
                if (left & 1) *reinterpret_cast<any1*>(p + left - 1) = left == 1 ? w[0] : w[2];
            }
        }
    }
    // The value that a stored element holds.
    static __device__ __forceinline__ float rounded(float v) {
        if constexpr (sizeof(T) == 2)
            return bf16_to_float(float_to_bf16(v));
        else
            return v;
    }
    // This piece's codes, to `row` of code_ld(width) bytes.
    static __device__ __forceinline__ void store_codes(uint8_t* row, int32_t at, const float (&v)[P], float inverse) {
        if constexpr (P == 8)
            *reinterpret_cast<uint2*>(row + at) = make_uint2(four_codes(v[0], v[1], v[2], v[3], inverse), four_codes(v[4], v[5], v[6], v[7], inverse));
        else
            *reinterpret_cast<uint32_t*>(row + at) = four_codes(v[0], v[1], v[2], v[3], inverse);
    }
};
