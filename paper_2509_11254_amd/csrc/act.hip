// Activations kept in 8 bits for the backward pass.
//
// A row is cut into groups of 32 columns.  A group's scale is the smallest power of two 2^e with max|x| <= 127 * 2^e (kept as
// e + 127 in a byte, 0 for a group of zeros), an element's code round(x / 2^e) to even in a signed byte; -128 stands for what
// is not finite and comes back as NaN.  With a power of two neither the division nor the way back rounds, and a value has at most
// seven significant bits: it is a bf16 number, so that matrix products take it as it is.
//
// A thread has 16 columns, two threads a group: one to four 16-byte loads, a 16-byte store of codes, one exchange for the
// maximum.  All kernels here read and write each byte once and are bound by HBM.
#include "tile_dev.h"

namespace psgd {

constexpr int kGroup = 32;
typedef signed char codex16 __attribute__((ext_vector_type(16)));

// item of 16 columns: row and first column.  `per` items per row.
struct ActPlace { int64_t row; int col; bool in; };
__device__ __forceinline__ ActPlace act_place(int64_t rows, int per) {
    const int64_t first = (int64_t)blockIdx.x * kThreads;
    const int64_t row0 = first / per;
    const unsigned at = (unsigned)(first - row0 * per) + threadIdx.x, down = at / (unsigned)per;
    ActPlace p;
    p.row = row0 + down;
    p.col = 16 * (int)(at - down * per);
    p.in = p.row < rows;
    return p;
}

// 16 elements from column c on of a row; zeros beyond cols.  Whole 16-byte pieces that begin inside the row are read.
__device__ __forceinline__ void load16(const PSGD_GLOBAL bf16_t* p, int c, int cols, float (&x)[16]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        bf16x8 v;
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = (bf16_t)0.f;
        if (c + 8 * h < cols) v = *reinterpret_cast<const PSGD_GLOBAL bf16x8*>(p + c + 8 * h);
#pragma unroll
        for (int u = 0; u < 8; ++u) x[8 * h + u] = c + 8 * h + u < cols ? (float)v[u] : 0.f;
    }
}
__device__ __forceinline__ void load16(const PSGD_GLOBAL float* p, int c, int cols, float (&x)[16]) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        floatx4 v = {0.f, 0.f, 0.f, 0.f};
        if (c + 4 * h < cols) v = *reinterpret_cast<const PSGD_GLOBAL floatx4*>(p + c + 4 * h);
#pragma unroll
        for (int u = 0; u < 4; ++u) x[4 * h + u] = c + 4 * h + u < cols ? v[u] : 0.f;
    }
}
// nothing beyond cols is written
__device__ __forceinline__ void store16(PSGD_GLOBAL bf16_t* p, int c, int cols, const float (&x)[16]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (c + 8 * h + 8 <= cols) {
            bf16x8 v;
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = (bf16_t)x[8 * h + u];
            *reinterpret_cast<PSGD_GLOBAL bf16x8*>(p + c + 8 * h) = v;
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (c + 8 * h + u < cols) p[c + 8 * h + u] = (bf16_t)x[8 * h + u];
        }
    }
}
__device__ __forceinline__ void store16(PSGD_GLOBAL float* p, int c, int cols, const float (&x)[16]) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        if (c + 4 * h + 4 <= cols) {
            const floatx4 v = {x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
            *reinterpret_cast<PSGD_GLOBAL floatx4*>(p + c + 4 * h) = v;
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c + 4 * h + u < cols) p[c + 4 * h + u] = x[4 * h + u];
        }
    }
}

// codes of this thread's half of a group, and the group's scale byte (the other half is lane ^ 1's: all lanes come here)
__device__ __forceinline__ int quantise16(const float (&x)[16], codex16& code) {
    unsigned most = 0;
#pragma unroll
    for (int u = 0; u < 16; ++u) {
        const unsigned a = __float_as_uint(x[u]) & 0x7fffffffu;
        most = max(most, a < 0x7f800000u ? a : 0u);
    }
    most = max(most, (unsigned)__shfl_xor((int)most, 1));
    // 127 * 2^e reaches 1.f * 2^E for e = E - 6 where 1.f <= 127 / 64, else for E - 5
    const int e = (int)(most >> 23) - 6 + ((most & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    const int scale = most == 0 ? 0 : min(max(e, 1), 248);
    const float inverse = __uint_as_float((unsigned)(254 - scale) << 23);
#pragma unroll
    for (int u = 0; u < 16; ++u) {
        const bool finite = (__float_as_uint(x[u]) & 0x7f800000u) != 0x7f800000u;
        const int q = (int)rintf(fminf(fmaxf(x[u] * inverse, -127.f), 127.f));
        code[u] = (signed char)(finite ? (scale ? q : 0) : -128);
    }
    return scale;
}
__device__ __forceinline__ float act_scale(unsigned byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float act_value(signed char code, float scale) {
    return code == -128 ? __builtin_nanf("") : (float)code * scale;
}

struct ActOut { signed char* codes; unsigned char* scales; };

__device__ __forceinline__ void store_codes(const ActOut& k, const ActPlace& p, int64_t ldc, int groups, const codex16& code, int scale) {
    if (!p.in) return;
    *reinterpret_cast<PSGD_GLOBAL codex16*>(as_global(k.codes) + p.row * ldc + p.col) = code;
    if ((p.col & (kGroup - 1)) == 0) as_global(k.scales)[p.row * groups + p.col / kGroup] = (unsigned char)scale;
}
__device__ __forceinline__ void load_values(const signed char* codes, const unsigned char* scales, const ActPlace& p, int64_t ldc, int groups,
                                            float (&x)[16]) {
    const codex16 code = *reinterpret_cast<const PSGD_GLOBAL codex16*>(as_global(codes) + p.row * ldc + p.col);
    const float scale = act_scale(as_global(scales)[p.row * groups + p.col / kGroup]);
#pragma unroll
    for (int u = 0; u < 16; ++u) x[u] = act_value(code[u], scale);
}

// The two threads of a group are neighbours: `per` counts whole groups' halves (an even number of items per row).
template <class T>
__global__ __launch_bounds__(kThreads) void act_store_kernel(int64_t rows, int cols, int per, const T* x, int64_t ld, ActOut out, int64_t ldc, int groups) {
    const ActPlace p = act_place(rows, per);
    float v[16];
    load16(as_global(x) + (p.in ? p.row : 0) * ld, p.in ? p.col : cols, cols, v);
    codex16 code;
    const int scale = quantise16(v, code);
    if (p.col < (cols + 15) / 16 * 16) store_codes(out, p, ldc, groups, code, scale);
}

template <class T>
__global__ __launch_bounds__(kThreads) void act_restore_kernel(int64_t rows, int cols, int per, const signed char* codes, const unsigned char* scales,
                                                               int64_t ldc, int groups, T* x, int64_t ld) {
    const ActPlace p = act_place(rows, per);
    if (!p.in || p.col >= cols) return;
    float v[16];
    load_values(codes, scales, p, ldc, groups, v);
    store16(as_global(x) + p.row * ld, p.col, cols, v);
}

// act(x) and its derivative.  SiLU: x s, s (1 + x (1 - s)) with s = 1 / (1 + e^-x).  GELU: x F, F + x f with the normal
// distribution's F and f.  bf16 results take the hardware's exponential (1e-6 relative), fp32 ones the library's.
template <int ACT, bool FAST>
__device__ __forceinline__ float act_fn(float x, float& slope) {
    if constexpr (ACT == PSGD_SILU) {
        const float s = 1.f / (1.f + (FAST ? __expf(-x) : expf(-x)));
        slope = s * (1.f + x * (1.f - s));
        return x * s;
    } else {
        const float cdf = 0.5f * (1.f + erff(x * 0.70710678118654752f));
        slope = cdf + x * 0.39894228040143268f * (FAST ? __expf(-0.5f * x * x) : expf(-0.5f * x * x));
        return x * cdf;
    }
}

template <class T, int ACT, bool GATED>
__global__ __launch_bounds__(kThreads) void act_glu_kernel(int64_t rows, int cols, int per, const T* gate, const T* up, int64_t ld_in, T* h,
                                                           int64_t ld_h, ActOut kg, ActOut ku, int64_t ldc, int groups) {
    const ActPlace p = act_place(rows, per);
    const int64_t row = p.in ? p.row : 0;
    const int col = p.in ? p.col : cols;
    const bool kept = p.col < (cols + 15) / 16 * 16;
    float g[16], u[16], y[16];
    load16(as_global(gate) + row * ld_in, col, cols, g);
    if constexpr (GATED) load16(as_global(up) + row * ld_in, col, cols, u);
    codex16 code;
    int scale = quantise16(g, code);
    if (kept) store_codes(kg, p, ldc, groups, code, scale);
    if constexpr (GATED) {
        scale = quantise16(u, code);
        if (kept) store_codes(ku, p, ldc, groups, code, scale);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float slope;
        y[i] = act_fn<ACT, sizeof(T) == 2>(g[i], slope);
        if constexpr (GATED) y[i] *= u[i];
    }
    if (p.in) store16(as_global(h) + p.row * ld_h, p.col, cols, y);
}

template <class T, int ACT, bool GATED>
__global__ __launch_bounds__(kThreads) void act_glu_backward_kernel(int64_t rows, int cols, int per, const signed char* cg, const unsigned char* sg,
                                                                    const signed char* cu, const unsigned char* su, int64_t ldc, int groups,
                                                                    const T* dh, int64_t ld_h, T* dgate, T* dup, int64_t ld_out) {
    const ActPlace p = act_place(rows, per);
    if (!p.in || p.col >= cols) return;
    float g[16], u[16], d[16], y[16];
    load_values(cg, sg, p, ldc, groups, g);
    if constexpr (GATED) load_values(cu, su, p, ldc, groups, u);
    load16(as_global(dh) + p.row * ld_h, p.col, cols, d);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float slope;
        const float a = act_fn<ACT, sizeof(T) == 2>(g[i], slope);
        y[i] = d[i] * a;
        g[i] = (GATED ? d[i] * u[i] : d[i]) * slope;
    }
    store16(as_global(dgate) + p.row * ld_out, p.col, cols, g);
    if constexpr (GATED) store16(as_global(dup) + p.row * ld_out, p.col, cols, y);
}

struct ActGrid {
    dim3 grid;
    int per, groups;
};
static ActGrid act_grid(int64_t rows, int64_t cols) {
    ActGrid g;
    g.groups = (int)((cols + kGroup - 1) / kGroup);
    g.per = 2 * g.groups;
    g.grid = dim3((unsigned)((rows * g.per + kThreads - 1) / kThreads));
    return g;
}
static int act_shape(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1 || rows > kMaxExtent || cols > kMaxExtent) return PSGD_E_SHAPE;
    if (rows * (2 * ((cols + kGroup - 1) / kGroup)) > (int64_t)INT32_MAX * kThreads) return PSGD_E_SHAPE;
    return PSGD_OK;
}
static bool bad_codes(const void* codes, const void* scales) { return !codes || !scales; }
static bool bad_ldc(int64_t ldc, int64_t cols) { return ldc < cols || (ldc & 15) != 0; }

struct WgradPlan {
    size_t bytes = 0, x = 0, planes = 0, part = 0;
    int n_planes = 1;
    TilePlan tile = {};
    int64_t ldx = 0;
};
static WgradPlan wgrad_plan(int64_t tokens, int64_t out, int64_t in, int dtype) {
    WgradPlan w;
    auto take = [&](size_t bytes) { const size_t at = w.bytes; w.bytes += up256(bytes); return at; };
    w.ldx = up8(in);
    w.x = take((size_t)tokens * w.ldx * 2);
    if (dtype == PSGD_F32) {
        w.n_planes = 3;
        w.planes = take((size_t)tokens * up8(out) * 2 * 3);
    }
    w.tile = tile_plan(in, out, (tokens + kTileK - 1) / kTileK * w.n_planes, true);
    w.part = take(tile_part_bytes(in, out, w.tile));
    return w;
}
static int wgrad_shape(int64_t tokens, int64_t out, int64_t in) {
    if (tokens < 0 || out < 1 || in < 1 || tokens > kMaxExtent || out > kMaxExtent || in > kMaxExtent) return PSGD_E_SHAPE;
    if (up8(in) > kMaxLd || up8(out) > kMaxLd) return PSGD_E_SHAPE;
    return act_shape(tokens, in);
}

}  // namespace psgd

using namespace psgd;

extern "C" {

int psgd_act_store(void* stream, int64_t rows, int64_t cols, const void* x, int dtype, int64_t ld, int8_t* codes, int64_t ldc, uint8_t* scales) {
    if ((rows != 0 && (!x || bad_codes(codes, scales))) || bad_dtype(dtype)) return PSGD_E_INVALID_ARG;
    if (int rc = act_shape(rows, cols)) return rc;
    if (bad_ld(ld, cols) || bad_ldc(ldc, cols) || misaligned(x) || misaligned(codes)) return PSGD_E_ALIGN;
    if (rows == 0) return PSGD_OK;
    const ActGrid g = act_grid(rows, cols);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const ActOut out = {codes, scales};
    if (dtype == PSGD_F32) hipLaunchKernelGGL(act_store_kernel<float>, g.grid, dim3(kThreads), 0, st, rows, (int)cols, g.per, (const float*)x, ld, out, ldc, g.groups);
    else hipLaunchKernelGGL(act_store_kernel<bf16_t>, g.grid, dim3(kThreads), 0, st, rows, (int)cols, g.per, (const bf16_t*)x, ld, out, ldc, g.groups);
    return hipGetLastError() == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

int psgd_act_restore(void* stream, int64_t rows, int64_t cols, const int8_t* codes, int64_t ldc, const uint8_t* scales, void* x, int dtype, int64_t ld) {
    if ((rows != 0 && (!x || bad_codes(codes, scales))) || bad_dtype(dtype)) return PSGD_E_INVALID_ARG;
    if (int rc = act_shape(rows, cols)) return rc;
    if (bad_ld(ld, cols) || bad_ldc(ldc, cols) || misaligned(x) || misaligned(codes)) return PSGD_E_ALIGN;
    if (rows == 0) return PSGD_OK;
    const ActGrid g = act_grid(rows, cols);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (dtype == PSGD_F32) hipLaunchKernelGGL(act_restore_kernel<float>, g.grid, dim3(kThreads), 0, st, rows, (int)cols, g.per, codes, scales, ldc, g.groups, (float*)x, ld);
    else hipLaunchKernelGGL(act_restore_kernel<bf16_t>, g.grid, dim3(kThreads), 0, st, rows, (int)cols, g.per, codes, scales, ldc, g.groups, (bf16_t*)x, ld);
    return hipGetLastError() == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

int psgd_act_glu(void* stream, int64_t rows, int64_t cols, int act, int dtype, const void* gate, const void* up, int64_t ld_in, void* h, int64_t ld_h,
                 int8_t* gate_codes, uint8_t* gate_scales, int8_t* up_codes, uint8_t* up_scales, int64_t ldc) {
    if (bad_dtype(dtype) || (act != PSGD_SILU && act != PSGD_GELU)) return PSGD_E_INVALID_ARG;
    if (rows != 0 && (!gate || !h || bad_codes(gate_codes, gate_scales))) return PSGD_E_INVALID_ARG;
    if (rows != 0 && (up ? bad_codes(up_codes, up_scales) : (up_codes || up_scales))) return PSGD_E_INVALID_ARG;
    if (int rc = act_shape(rows, cols)) return rc;
    if (bad_ld(ld_in, cols) || bad_ld(ld_h, cols) || bad_ldc(ldc, cols) || misaligned(gate) || misaligned(up) || misaligned(h) ||
        misaligned(gate_codes) || misaligned(up_codes)) return PSGD_E_ALIGN;
    if (rows == 0) return PSGD_OK;
    const ActGrid g = act_grid(rows, cols);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const ActOut kg = {gate_codes, gate_scales}, ku = {up_codes, up_scales};
#define PSGD_GLU(T, ACT, GATED)                                                                                                       \
    hipLaunchKernelGGL((act_glu_kernel<T, ACT, GATED>), g.grid, dim3(kThreads), 0, st, rows, (int)cols, g.per, (const T*)gate, (const T*)up, \
                       ld_in, (T*)h, ld_h, kg, ku, ldc, g.groups)
#define PSGD_GLU_ACT(T, GATED) do { if (act == PSGD_SILU) PSGD_GLU(T, PSGD_SILU, GATED); else PSGD_GLU(T, PSGD_GELU, GATED); } while (0)
    if (dtype == PSGD_F32) { if (up) PSGD_GLU_ACT(float, true); else PSGD_GLU_ACT(float, false); }
    else                   { if (up) PSGD_GLU_ACT(bf16_t, true); else PSGD_GLU_ACT(bf16_t, false); }
#undef PSGD_GLU
#undef PSGD_GLU_ACT
    return hipGetLastError() == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

int psgd_act_glu_backward(void* stream, int64_t rows, int64_t cols, int act, int dtype, const int8_t* gate_codes, const uint8_t* gate_scales,
                          const int8_t* up_codes, const uint8_t* up_scales, int64_t ldc, const void* dh, int64_t ld_h, void* dgate, void* dup,
                          int64_t ld_out) {
    if (bad_dtype(dtype) || (act != PSGD_SILU && act != PSGD_GELU)) return PSGD_E_INVALID_ARG;
    const bool gated = up_codes != nullptr;
    if (rows != 0 && (!dh || !dgate || bad_codes(gate_codes, gate_scales))) return PSGD_E_INVALID_ARG;
    if (rows != 0 && (gated ? (!up_scales || !dup) : (up_scales || dup))) return PSGD_E_INVALID_ARG;
    if (int rc = act_shape(rows, cols)) return rc;
    if (bad_ld(ld_h, cols) || bad_ld(ld_out, cols) || bad_ldc(ldc, cols) || misaligned(dh) || misaligned(dgate) || misaligned(dup) ||
        misaligned(gate_codes) || misaligned(up_codes)) return PSGD_E_ALIGN;
    if (rows == 0) return PSGD_OK;
    const ActGrid g = act_grid(rows, cols);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
#define PSGD_GLU(T, ACT, GATED)                                                                                                       \
    hipLaunchKernelGGL((act_glu_backward_kernel<T, ACT, GATED>), g.grid, dim3(kThreads), 0, st, rows, (int)cols, g.per, gate_codes,    \
                       gate_scales, up_codes, up_scales, ldc, g.groups, (const T*)dh, ld_h, (T*)dgate, (T*)dup, ld_out)
#define PSGD_GLU_ACT(T, GATED) do { if (act == PSGD_SILU) PSGD_GLU(T, PSGD_SILU, GATED); else PSGD_GLU(T, PSGD_GELU, GATED); } while (0)
    if (dtype == PSGD_F32) { if (gated) PSGD_GLU_ACT(float, true); else PSGD_GLU_ACT(float, false); }
    else                   { if (gated) PSGD_GLU_ACT(bf16_t, true); else PSGD_GLU_ACT(bf16_t, false); }
#undef PSGD_GLU
#undef PSGD_GLU_ACT
    return hipGetLastError() == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

size_t psgd_act_wgrad_workspace_bytes(int64_t tokens, int64_t out_features, int64_t in_features, int dtype) {
    if (wgrad_shape(tokens, out_features, in_features) || bad_dtype(dtype)) return 0;
    return std::max<size_t>(256, wgrad_plan(tokens, out_features, in_features, dtype).bytes);
}

int psgd_act_wgrad(void* workspace, void* stream, int64_t tokens, int64_t out_features, int64_t in_features, const void* dy, int dtype, int64_t ldy,
                   const int8_t* codes, int64_t ldc, const uint8_t* scales, void* g, int g_dtype, int64_t ldg, int accumulate) {
    if (!workspace || !g || (tokens != 0 && (!dy || bad_codes(codes, scales))) || bad_dtype(dtype) || bad_dtype(g_dtype)) return PSGD_E_INVALID_ARG;
    if (int rc = wgrad_shape(tokens, out_features, in_features)) return rc;
    if (ldy > kMaxLd || ldg > kMaxLd) return PSGD_E_SHAPE;
    if (bad_ld(ldy, out_features) || bad_ld(ldg, in_features) || bad_ldc(ldc, in_features) || misaligned(dy) || misaligned(g) ||
        misaligned(codes) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PSGD_E_ALIGN;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const WgradPlan w = wgrad_plan(tokens, out_features, in_features, dtype);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    bf16_t* x = reinterpret_cast<bf16_t*>(ws + w.x);
    bf16_t* planes = reinterpret_cast<bf16_t*>(ws + w.planes);
    if (tokens > 0) {
        if (int rc = psgd_act_restore(stream, tokens, in_features, codes, ldc, scales, x, PSGD_BF16, w.ldx)) return rc;
        if (dtype == PSGD_F32 && launch_planes(dy, dtype, tokens, out_features, ldy, planes, 3, st) != hipSuccess) return PSGD_E_HIP;
    }
    TileArgs t = {};
    t.P = {x, w.ldx, 0, (int)in_features};
    if (dtype == PSGD_F32) t.L = {planes, up8(out_features), tokens * up8(out_features), (int)out_features};
    else t.L = {static_cast<const bf16_t*>(dy), ldy, 0, (int)out_features};
    t.K = (int)tokens;
    t.pairs = w.n_planes == 3 ? kPairsL3 : kPairs1;
    t.n_pairs = w.n_planes;
    t.n_split = w.tile.n_split;
    TileOut o = {};
    o.ptr = g;
    o.ld = ldg;
    o.dtype = g_dtype;
    o.accumulate = accumulate != 0;
    o.part = reinterpret_cast<float*>(ws + w.part);
    return launch_product(false, w.tile.shape, t, o, st) == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

}  // extern "C"
