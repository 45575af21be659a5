// Activations in kernels that read and write them piece by piece (act.hip, norm.hip, expert.hip, head.hip), and the values of 8-bit checkpoints.
#pragma once
#include "psgd_dev.h"

#include <type_traits>

namespace psgd {

// An activation is loaded and stored 16 bytes at a time, with the non-temporal hint or without.
template <bool STREAM, class V> __device__ __forceinline__ V ld_act(const PSGD_GLOBAL V* p) {
    if constexpr (STREAM) return __builtin_nontemporal_load(p); else return *p;
}
template <bool STREAM, class V> __device__ __forceinline__ void st_act(PSGD_GLOBAL V* p, V v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, p); else *p = v;
}
template <class T> constexpr int kPiece = 16 / (int)sizeof(T);      // columns of a piece
struct ActPlace { int64_t row; int col; bool in; };

// A piece as it is stored; zeros beyond cols.  A piece that begins inside the row is read as a whole.
template <bool STREAM, class T>
__device__ __forceinline__ uintx4 load_raw(const T* x, int64_t ld, const ActPlace& p) {
    uintx4 w = {0u, 0u, 0u, 0u};
    if (p.in) w = ld_act<STREAM>(reinterpret_cast<const PSGD_GLOBAL uintx4*>(as_global(x) + p.row * ld + p.col));
    return w;
}
template <class T>
__device__ __forceinline__ void clear_beyond(uintx4& w, const ActPlace& p, int cols) {
    if (p.col + kPiece<T> > cols) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if constexpr (sizeof(T) == 4) w[u] = p.col + u < cols ? w[u] : 0u;
            else w[u] &= (p.col + 2 * u < cols ? 0xffffu : 0u) | (p.col + 2 * u + 1 < cols ? 0xffff0000u : 0u);
        }
    }
}
template <class T, int N = kPiece<T>>
__device__ __forceinline__ void widen(const uintx4& w, float (&v)[N]) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if constexpr (N == 4) v[u] = __uint_as_float(w[u]);
        else { v[2 * u] = __uint_as_float(w[u] << 16); v[2 * u + 1] = __uint_as_float(w[u] & 0xffff0000u); }
    }
}
// nothing beyond cols is written
template <bool STREAM, class T, int N = kPiece<T>>
__device__ __forceinline__ void store_piece(T* x, int64_t ld, const ActPlace& p, int cols, const float (&v)[N]) {
    if (!p.in) return;
    PSGD_GLOBAL T* at = as_global(x) + p.row * ld + p.col;
    if (p.col + N <= cols) {
        typedef __attribute__((__vector_size__(16))) T piece;
        piece q;
#pragma unroll
        for (int u = 0; u < N; ++u) q[u] = (T)v[u];
        st_act<STREAM>(reinterpret_cast<PSGD_GLOBAL uintx4*>(at), __builtin_bit_cast(uintx4, q));
    } else {
#pragma unroll
        for (int u = 0; u < N; ++u)
            if (p.col + u < cols) at[u] = (T)v[u];
    }
}

// What join makes of LANES lanes next to each other, in all of them: lane ^ 1, lane ^ 2, the other four of eight, the other eight of sixteen, the other row
// of two, the other half.  (In registers; by way of LDS each step waits for it: 60000 rows of 512 in bf16 normalised, 27.1 us in place of 24.2.)
template <int LANES, class F>
__device__ __forceinline__ float lanes_join(float v, F join) {
    auto from = [](float x, auto ctrl) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true)); };
    v = join(v, from(v, std::integral_constant<int, 0xB1>{}));
    v = join(v, from(v, std::integral_constant<int, 0x4E>{}));
    if constexpr (LANES > 4) v = join(v, from(v, std::integral_constant<int, 0x141>{}));
    if constexpr (LANES > 8) v = join(v, from(v, std::integral_constant<int, 0x140>{}));
    if constexpr (LANES > 16) {
        const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = join(__uint_as_float(two[0]), __uint_as_float(two[1]));
    }
    if constexpr (LANES > 32) {
        const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = join(__uint_as_float(two[0]), __uint_as_float(two[1]));
    }
    return v;
}
template <int LANES> __device__ __forceinline__ float lanes_sum(float v) { return lanes_join<LANES>(v, [](float a, float b) { return a + b; }); }
template <int LANES> __device__ __forceinline__ float lanes_max(float v) { return lanes_join<LANES>(v, [](float a, float b) { return fmaxf(a, b); }); }

// four codes to a word, and their group's scale
template <int W> struct ActCodes { unsigned w[W]; float scale; };
template <int W>
__device__ __forceinline__ void values(const ActCodes<W>& c, float (&x)[4 * W]) {
    bool any = c.scale > 0x1p120f;       // (128 times the largest scale is infinite)
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const unsigned w = c.w[i] ^ 0x80808080u;        // code + 128
        any |= ((w - 0x01010101u) & ~w & 0x80808080u) != 0;         // a byte that is zero
#pragma unroll
        for (int k = 0; k < 4; ++k) x[4 * i + k] = fmaf((float)((w >> (8 * k)) & 0xffu), c.scale, -128.f * c.scale);
    }
    if (__any(any)) {
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const signed char code = (signed char)(c.w[i] >> (8 * k));
                x[4 * i + k] = code == -128 ? __builtin_nanf("") : (float)code * c.scale;
            }
    }
}

}  // namespace psgd
