// Values of 8-bit checkpoints (act.hip) in kernels that read them.
#pragma once
#include "psgd_dev.h"

namespace psgd {

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
