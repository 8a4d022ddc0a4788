// How rows are dealt to lanes by the kernels that keep a row in registers: G lanes take a row, E pieces of 16 bytes each (piece t + e G
// of lane t), so that the 128 columns of a scale are in lanes of one wavefront and every lane keeps its columns from row to row.
#pragma once

#include <type_traits>

#include "codes_device.h"
#include "varco.h"

constexpr int kWideRow = 512;        // lanes of a row above 2,048 elements: a workgroup
constexpr int row_threads(int g) { return g > 64 ? g : 256; }       // of a workgroup

template <int N>
using Int = std::integral_constant<int, N>;

// Calls f(lanes of a row, pieces per lane) for rows of `width` elements, the columns up to whole 16 included.
template <typename T, typename F>
void with_row_layout(int32_t width, F f) {
    const int64_t pieces = code_ld(width) / RowPiece<T>::P;
    if (pieces <= 4)
        f(Int<4>{}, Int<1>{});
    else if (pieces <= 8)
        f(Int<8>{}, Int<1>{});
    else if (pieces <= 16)
        f(Int<16>{}, Int<1>{});
    else if (pieces <= 32)
        f(Int<32>{}, Int<1>{});
    else if (pieces <= 64)
        f(Int<64>{}, Int<1>{});
    else if (pieces <= 128)
        f(Int<64>{}, Int<2>{});
    else if (pieces <= 256)
        f(Int<64>{}, Int<4>{});
    else if (pieces <= 512 && sizeof(T) == 4)
        f(Int<64>{}, Int<8>{});
    else if (pieces <= kWideRow)
        f(Int<kWideRow>{}, Int<1>{});
    else if (pieces <= 2 * kWideRow)
        f(Int<kWideRow>{}, Int<2>{});
    else if (pieces <= 4 * kWideRow)
        f(Int<kWideRow>{}, Int<4>{});
    else if constexpr (sizeof(T) == 4)
        f(Int<kWideRow>{}, Int<8>{});
}

template <typename F>
void with_bool(bool b, F f) {
    if (b)
        f(std::true_type{});
    else
        f(std::false_type{});
}
template <typename F>
void with_type(int dtype, F f) {
    if (dtype == VARCO_BF16)
        f(bf16_t{});
    else
        f(float{});
}

// Codes and scales of a row that G lanes hold, v[e] the values of piece t + e G; what lies behind the last column is taken as 0.
template <typename T, int G, int E>
__device__ __forceinline__ void store_row_codes(const float (&v)[E][RowPiece<T>::P], int t, int32_t width, uint8_t* codes, uint8_t* scales) {
    using Row = RowPiece<T>;
    constexpr int P = Row::P, kLanes = kCodeBlock / P < G ? kCodeBlock / P : G;        // of a scale
    const int32_t ldc = int32_t(code_ld(width)), lds = int32_t(scale_ld(width)), blocks = (width + kCodeBlock - 1) / kCodeBlock;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int32_t at = (t + e * G) * P;
        float q[P], m = 0.f;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            q[j] = at + j < width ? v[e][j] : 0.f;
            m = fmaxf(m, finite_size(q[j]));
        }
        const int x = code_exponent(lanes_max<kLanes>(m));
        if (at < ldc) Row::store_codes(codes, at, q, code_inverse(x));
        if (at % kCodeBlock == 0 && at < width) scales[at / kCodeBlock] = uint8_t(x + 127);
    }
    if (t < lds - blocks) scales[blocks + t] = kOneScale;
}
