// Activations kept in 8 bits for the backward pass.
//
// A row is cut into groups of 32 columns.  A group's scale is the smallest power of two 2^e with max|x| <= 127 * 2^e (kept as
// e + 127 in a byte, 0 for a group of zeros), an element's code round(x / 2^e) to even in a signed byte; -128 stands for what
// is not finite and comes back as NaN.  With a power of two neither the division nor the way back rounds, and a value has at most
// seven significant bits: it is a bf16 number, so that matrix products take it as it is.
//
// A thread has 16 bytes of an activation at a time, 8 columns in bf16 and 4 in fp32, so that every load and store of a wavefront is one
// run of 1 KB (with two stores of 16 bytes side by side, each leaves half of every line to the other, and the non-temporal hint costs 40 %); four or eight threads next to each other have a group.  Each byte is read and written once, and HBM would bound all of it, were
// it not for the arithmetic: at 5 TB/s there are 24 vector instructions per element.  So the common case has few: rounding to a
// whole number is the addition of 1.5 * 2^23 (whose last bit is 1), the codes are the sums' low bytes; a code becomes a value by the
// conversion of an unsigned byte and one multiply-add; what is not finite or beyond the largest scale is sought once per group, and sends the
// wavefront the slow way.  16384 x 11008 in bf16, stored and restored: 201 -> 171 us, 6.4 TB/s; gated unit of 8192 x 11008, both ways: 293 -> 229, 6.4 TB/s.
#include "act_dev.h"
#include "train.h"

namespace psgd {

constexpr int kGroup = 32;
constexpr int kActItems = 2;        // pieces per thread, all of whose loads are sent off first (1: 225 us, 4: 202, where 2 take 200)
// From this many bytes of activations in a call on they are loaded and stored with the non-temporal hint (16384 x 11008 in bf16 and back 200 -> 180 us,
// gated unit of 8192 x 11008 forward and backward 260 -> 228); what is smaller, the next kernel may find in the caches.  Codes never have it (188, 240).
constexpr int64_t kActStream = 96 << 20;
constexpr unsigned kInfBits = 0x7f800000u;
constexpr unsigned kTopBits = 0x7f7e0000u;      // 127 * 2^121, the largest number that the largest scale holds
constexpr float kWhole = 12582912.f;            // 1.5 * 2^23

// piece i of this thread: row and first column.  `per`: pieces of a row, of whole groups; inv_per its reciprocal.
struct ActRows { int64_t rows; int cols, per; double inv_per; };
template <int N>
__device__ __forceinline__ ActPlace act_place(const ActRows& r, int i) {
    const int64_t first = ((int64_t)blockIdx.x * kActItems + i) * kThreads;
    int64_t row0 = (int64_t)((double)first * r.inv_per);        // off by one at most
    int64_t rest = first - row0 * r.per;
    if (rest < 0) { --row0; rest += r.per; }
    if (rest >= r.per) { ++row0; rest -= r.per; }
    unsigned at = (unsigned)rest + threadIdx.x, down = 0;
    if (r.per >= kThreads) {
        if (at >= (unsigned)r.per) { at -= r.per; down = 1; }
    } else {
        down = at / (unsigned)r.per;
        at -= down * r.per;
    }
    ActPlace p;
    p.row = row0 + down;
    p.col = N * (int)at;
    p.in = p.row < r.rows && p.col < r.cols;
    return p;
}

// the largest magnitude of a group as fp32 bits, what is not finite included (all lanes of the group come here)
template <class T>
__device__ __forceinline__ unsigned group_most(const uintx4& w) {
    typedef unsigned short ushortx2 __attribute__((ext_vector_type(2)));
    unsigned most;
    if constexpr (sizeof(T) == 4) {
        most = max(max(w[0] & 0x7fffffffu, w[1] & 0x7fffffffu), max(w[2] & 0x7fffffffu, w[3] & 0x7fffffffu));
    } else {
        ushortx2 m = __builtin_bit_cast(ushortx2, w[0] & 0x7fff7fffu);
#pragma unroll
        for (int u = 1; u < 4; ++u) m = __builtin_elementwise_max(m, __builtin_bit_cast(ushortx2, w[u] & 0x7fff7fffu));
        most = (unsigned)max(m[0], m[1]) << 16;
    }
    // lanes ^ 1, ^ 2 and, for eight lanes to a group, the other four
    most = max(most, (unsigned)__builtin_amdgcn_mov_dpp((int)most, 0xB1, 0xf, 0xf, true));
    most = max(most, (unsigned)__builtin_amdgcn_mov_dpp((int)most, 0x4E, 0xf, 0xf, true));
    if constexpr (sizeof(T) == 4) most = max(most, (unsigned)__builtin_amdgcn_mov_dpp((int)most, 0x141, 0xf, 0xf, true));
    return most;
}
// the scale byte for a largest magnitude that is finite: 127 * 2^e reaches 1.f * 2^E for e = E - 6 where 1.f <= 127 / 64, else for E - 5
__device__ __forceinline__ int scale_byte(unsigned most) {
    const int e = (int)((most + 0x1ffffu) >> 23) - 6;          // (a fraction above 0x7e0000 carries)
    return most == 0 ? 0 : min(max(e, 1), 248);
}

// four codes: the low bytes of four sums
__device__ __forceinline__ unsigned low_bytes(float a, float b, float c, float d) {
    const unsigned ab = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x0c0c0400u);
    const unsigned cd = __builtin_amdgcn_perm(__float_as_uint(d), __float_as_uint(c), 0x0c0c0400u);
    return __builtin_amdgcn_perm(cd, ab, 0x05040100u);
}

// codes of this thread's part of a group (kPiece / 4 words) and the group's scale byte; all lanes come here
template <class T, int N = kPiece<T>>
__device__ __forceinline__ int quantise(const uintx4& w, const float (&x)[N], unsigned (&code)[N / 4]) {
    unsigned most = group_most<T>(w);
    int scale = scale_byte(most);
    const float inverse = __uint_as_float((unsigned)(254 - scale) << 23);
    if (!__any(most > kTopBits)) {
#pragma unroll
        for (int u = 0; u < N; u += 4)
            code[u / 4] = low_bytes(fmaf(x[u], inverse, kWhole), fmaf(x[u + 1], inverse, kWhole), fmaf(x[u + 2], inverse, kWhole), fmaf(x[u + 3], inverse, kWhole));
        return scale;
    }
    most = 0;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const unsigned a = __float_as_uint(x[u]) & 0x7fffffffu;
        most = max(most, a < kInfBits ? a : 0u);
    }
#pragma unroll
    for (int d = 1; d < kGroup / N; d <<= 1) most = max(most, (unsigned)__shfl_xor((int)most, d));
    scale = scale_byte(most);
    const float inv = __uint_as_float((unsigned)(254 - scale) << 23);
#pragma unroll
    for (int u = 0; u < N; u += 4) {
        code[u / 4] = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool finite = (__float_as_uint(x[u + k]) & 0x7fffffffu) < kInfBits;
            const int q = finite ? (int)rintf(fminf(fmaxf(x[u + k] * inv, -127.f), 127.f)) : -128;
            code[u / 4] |= ((unsigned)q & 0xffu) << (8 * k);
        }
    }
    return scale;
}

struct ActOut { signed char* codes; unsigned char* scales; };

// (a row's codes reach to the next multiple of 16 columns)
template <int W>
__device__ __forceinline__ void store_codes(const ActOut& k, const ActPlace& p, const ActRows& r, int64_t ldc, const unsigned (&code)[W], int scale) {
    if (p.row < r.rows && p.col < (r.cols + 15) / 16 * 16) {
        PSGD_GLOBAL signed char* at = as_global(k.codes) + p.row * ldc + p.col;
        if constexpr (W == 2) *reinterpret_cast<PSGD_GLOBAL uintx2*>(at) = uintx2{code[0], code[1]};
        else *reinterpret_cast<PSGD_GLOBAL unsigned*>(at) = code[0];
    }
    if (p.in && (p.col & (kGroup - 1)) == 0) as_global(k.scales)[p.row * ((r.cols + kGroup - 1) / kGroup) + p.col / kGroup] = (unsigned char)scale;
}

template <int W>
__device__ __forceinline__ ActCodes<W> load_codes(const signed char* codes, const unsigned char* scales, const ActPlace& p, const ActRows& r, int64_t ldc) {
    ActCodes<W> c = {};
    if (p.in) {
        const PSGD_GLOBAL signed char* at = as_global(codes) + p.row * ldc + p.col;
        if constexpr (W == 2) {
            const uintx2 w = *reinterpret_cast<const PSGD_GLOBAL uintx2*>(at);
            c.w[0] = w[0], c.w[1] = w[1];
        } else {
            c.w[0] = *reinterpret_cast<const PSGD_GLOBAL unsigned*>(at);
        }
        c.scale = __uint_as_float((unsigned)as_global(scales)[p.row * ((r.cols + kGroup - 1) / kGroup) + p.col / kGroup] << 23);
    }
    return c;
}
template <class T, bool STREAM>
__global__ __launch_bounds__(kThreads) void act_store_kernel(ActRows r, const T* x, int64_t ld, ActOut out, int64_t ldc) {
    constexpr int N = kPiece<T>;
    ActPlace p[kActItems];
    uintx4 w[kActItems];
#pragma unroll
    for (int i = 0; i < kActItems; ++i) {
        p[i] = act_place<N>(r, i);
        w[i] = load_raw<STREAM>(x, ld, p[i]);
    }
#pragma unroll
    for (int i = 0; i < kActItems; ++i) {
        clear_beyond<T>(w[i], p[i], r.cols);
        float v[N];
        unsigned code[N / 4];
        widen<T>(w[i], v);
        const int scale = quantise<T>(w[i], v, code);
        store_codes(out, p[i], r, ldc, code, scale);
    }
}

template <class T, bool STREAM>
__global__ __launch_bounds__(kThreads) void act_restore_kernel(ActRows r, const signed char* codes, const unsigned char* scales, int64_t ldc, T* x, int64_t ld) {
    constexpr int N = kPiece<T>;
    ActPlace p[kActItems];
    ActCodes<N / 4> c[kActItems];
#pragma unroll
    for (int i = 0; i < kActItems; ++i) {
        p[i] = act_place<N>(r, i);
        c[i] = load_codes<N / 4>(codes, scales, p[i], r, ldc);
    }
#pragma unroll
    for (int i = 0; i < kActItems; ++i) {
        float v[N];
        values(c[i], v);
        store_piece<STREAM>(x, ld, p[i], r.cols, v);
    }
}

// act(x) and its derivative.  SiLU: x s, s (1 + x (1 - s)) with s = 1 / (1 + e^-x).  GELU: x F, F + x f with the normal
// distribution's F and f.  For bf16 results (FAST) the hardware's exponential and reciprocal, good to 1e-6, and F from f by formula
// 7.1.26 of Abramowitz and Stegun: one exponential serves both.  It is good to 1e-7 of 1, and relative to F to 0.05 % at -4, 0.16 % at -5, 0.4 % (a rounding to
// bf16) at -6, 2 % at -10, where F is 8e-24.  For fp32 the library's functions, F as a complement, which keeps its digits below zero.
template <int ACT, bool FAST>
__device__ __forceinline__ float act_fn(float x, float& slope) {
    if constexpr (ACT == PSGD_SILU) {
        const float s = FAST ? __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x)) : 1.f / (1.f + expf(-x));
        slope = s * fmaf(x, 1.f - s, 1.f);
        return x * s;
    } else if constexpr (FAST) {
        const float z = fabsf(x) * 0.70710678118654752f, k = __builtin_amdgcn_rcpf(fmaf(0.3275911f, z, 1.f));
        const float e = __builtin_amdgcn_exp2f(-0.72134752044448170f * x * x);
        const float poly = k * fmaf(k, fmaf(k, fmaf(k, fmaf(k, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
        const float tail = 0.5f * poly * e, cdf = x < 0.f ? tail : 1.f - tail;
        slope = fmaf(x * 0.39894228040143268f, e, cdf);
        return x * cdf;
    } else {
        const float cdf = 0.5f * erfcf(x * -0.70710678118654752f);
        slope = cdf + x * 0.39894228040143268f * expf(-0.5f * x * x);
        return x * cdf;
    }
}

template <class T, int ACT, bool GATED, bool STREAM>
__global__ __launch_bounds__(kThreads) void act_glu_kernel(ActRows r, const T* gate, const T* up, int64_t ld_in, T* h, int64_t ld_h, ActOut kg, ActOut ku,
                                                           int64_t ldc) {
    constexpr int N = kPiece<T>;
    ActPlace p[kActItems];
    uintx4 wg[kActItems], wu[kActItems];
#pragma unroll
    for (int i = 0; i < kActItems; ++i) {
        p[i] = act_place<N>(r, i);
        wg[i] = load_raw<STREAM>(gate, ld_in, p[i]);
        if constexpr (GATED) wu[i] = load_raw<STREAM>(up, ld_in, p[i]);
    }
#pragma unroll
    for (int i = 0; i < kActItems; ++i) {
        float g[N], u[N], y[N];
        unsigned code[N / 4];
        clear_beyond<T>(wg[i], p[i], r.cols);
        widen<T>(wg[i], g);
        int scale = quantise<T>(wg[i], g, code);
        store_codes(kg, p[i], r, ldc, code, scale);
        if constexpr (GATED) {
            clear_beyond<T>(wu[i], p[i], r.cols);
            widen<T>(wu[i], u);
            scale = quantise<T>(wu[i], u, code);
            store_codes(ku, p[i], r, ldc, code, scale);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float slope;
            y[k] = act_fn<ACT, sizeof(T) == 2>(g[k], slope);
            if constexpr (GATED) y[k] *= u[k];
        }
        store_piece<STREAM>(h, ld_h, p[i], r.cols, y);
    }
}

template <class T, int ACT, bool GATED, bool STREAM>
__global__ __launch_bounds__(kThreads) void act_glu_backward_kernel(ActRows r, const signed char* cg, const unsigned char* sg, const signed char* cu,
                                                                    const unsigned char* su, int64_t ldc, const T* dh, int64_t ld_h, T* dgate, T* dup,
                                                                    int64_t ld_out) {
    constexpr int N = kPiece<T>;
    ActPlace p[kActItems];
    ActCodes<N / 4> kg[kActItems], ku[kActItems];
    uintx4 wd[kActItems];
#pragma unroll
    for (int i = 0; i < kActItems; ++i) {
        p[i] = act_place<N>(r, i);
        kg[i] = load_codes<N / 4>(cg, sg, p[i], r, ldc);
        if constexpr (GATED) ku[i] = load_codes<N / 4>(cu, su, p[i], r, ldc);
        wd[i] = load_raw<STREAM>(dh, ld_h, p[i]);
    }
#pragma unroll
    for (int i = 0; i < kActItems; ++i) {
        float g[N], u[N], d[N], y[N];
        values(kg[i], g);
        if constexpr (GATED) values(ku[i], u);
        widen<T>(wd[i], d);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float slope;
            const float a = act_fn<ACT, sizeof(T) == 2>(g[k], slope);
            y[k] = d[k] * a;
            g[k] = (GATED ? d[k] * u[k] : d[k]) * slope;
        }
        store_piece<STREAM>(dgate, ld_out, p[i], r.cols, g);
        if constexpr (GATED) store_piece<STREAM>(dup, ld_out, p[i], r.cols, y);
    }
}

struct ActGrid {
    ActRows rows;
    dim3 grid;
};
static ActGrid act_grid(int64_t rows, int64_t cols, int dtype) {
    ActGrid g;
    const int n = dtype == PSGD_F32 ? kPiece<float> : kPiece<bf16_t>;
    g.rows.rows = rows, g.rows.cols = (int)cols;
    g.rows.per = (int)((cols + kGroup - 1) / kGroup * (kGroup / n));
    g.rows.inv_per = 1.0 / g.rows.per;
    g.grid = dim3((unsigned)((rows * g.rows.per + kThreads * kActItems - 1) / (kThreads * kActItems)));
    return g;
}
static int act_shape(int64_t rows, int64_t cols, int dtype) {
    if (rows < 0 || cols < 1 || rows > kMaxExtent || cols > kMaxExtent) return PSGD_E_SHAPE;
    const int64_t per = (cols + kGroup - 1) / kGroup * (kGroup / (dtype == PSGD_F32 ? kPiece<float> : kPiece<bf16_t>));
    if (rows * per >= ((int64_t)kActItems << 32) - kActItems * kThreads) return PSGD_E_SHAPE;      // a launch has fewer than 2^32 threads
    return PSGD_OK;
}
static bool bad_codes(const void* codes, const void* scales) { return !codes || !scales; }
static bool bad_ldc(int64_t ldc, int64_t cols) { return ldc < cols || (ldc & 15) != 0; }

static bool act_stream(int64_t rows, int64_t cols, int dtype, int matrices) {
    return rows * cols * (dtype == PSGD_F32 ? 4 : 2) * matrices >= kActStream;
}
static int act_restore(void* stream, int64_t rows, int64_t cols, const int8_t* codes, int64_t ldc, const uint8_t* scales, void* x, int dtype, int64_t ld,
                       bool stream_it) {
    if (rows == 0) return PSGD_OK;
    const ActGrid g = act_grid(rows, cols, dtype);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    forget_errors();
#define PSGD_RESTORE(T, STREAM) hipLaunchKernelGGL((act_restore_kernel<T, STREAM>), g.grid, dim3(kThreads), 0, st, g.rows, codes, scales, ldc, (T*)x, ld)
    if (dtype == PSGD_F32) { if (stream_it) PSGD_RESTORE(float, true); else PSGD_RESTORE(float, false); }
    else                   { if (stream_it) PSGD_RESTORE(bf16_t, true); else PSGD_RESTORE(bf16_t, false); }
#undef PSGD_RESTORE
    return hipGetLastError() == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

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
    w.n_planes = dtype == PSGD_F32 ? 3 : 1;
    // A launch of its own puts X's values into the workspace for all tiles, or each tile makes them of the codes as it goes, as often as there are tiles along
    // `out`.  (Tokens x out x in, in us, the first way with its best tiles and the second: 64 x 1000 x 1000 11.4, 8.1; 400 x 2000 x 1000 14.8, 12.9; 64 x 4096 x 4096
    // 16.1, 14.2; 300 x 11008 x 11008 112, 139; 2000 x 4096 x 4096 74, 100.)
    w.tile = tile_plan(in, out, (tokens + kTileK - 1) / kTileK * w.n_planes, true, 3 + tokens * (double)in * 3e-6 / 5);
    if (!w.tile.from_codes) w.x = take((size_t)tokens * w.ldx * 2);
    if (dtype == PSGD_F32) w.planes = take((size_t)tokens * up8(out) * 2 * 3);
    w.part = take(tile_part_bytes(in, out, w.tile));
    return w;
}
static int wgrad_shape(int64_t tokens, int64_t out, int64_t in) {
    if (tokens < 0 || out < 1 || in < 1 || tokens > kMaxExtent || out > kMaxExtent || in > kMaxExtent) return PSGD_E_SHAPE;
    if (up8(in) > kMaxLd || up8(out) > kMaxLd) return PSGD_E_SHAPE;
    return act_shape(tokens, in, PSGD_BF16);
}

}  // namespace psgd

using namespace psgd;

extern "C" {

int psgd_act_store(void* stream, int64_t rows, int64_t cols, const void* x, int dtype, int64_t ld, int8_t* codes, int64_t ldc, uint8_t* scales) {
    if ((rows != 0 && (!x || bad_codes(codes, scales))) || bad_dtype(dtype)) return PSGD_E_INVALID_ARG;
    if (int rc = act_shape(rows, cols, dtype)) return rc;
    if (bad_ld(ld, cols) || bad_ldc(ldc, cols) || misaligned(x) || misaligned(codes)) return PSGD_E_ALIGN;
    if (rows == 0) return PSGD_OK;
    const ActGrid g = act_grid(rows, cols, dtype);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    forget_errors();
    const ActOut out = {codes, scales};
#define PSGD_STORE(T, STREAM) hipLaunchKernelGGL((act_store_kernel<T, STREAM>), g.grid, dim3(kThreads), 0, st, g.rows, (const T*)x, ld, out, ldc)
    const bool stream_it = act_stream(rows, cols, dtype, 1);
    if (dtype == PSGD_F32) { if (stream_it) PSGD_STORE(float, true); else PSGD_STORE(float, false); }
    else                   { if (stream_it) PSGD_STORE(bf16_t, true); else PSGD_STORE(bf16_t, false); }
#undef PSGD_STORE
    return hipGetLastError() == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

int psgd_act_restore(void* stream, int64_t rows, int64_t cols, const int8_t* codes, int64_t ldc, const uint8_t* scales, void* x, int dtype, int64_t ld) {
    if ((rows != 0 && (!x || bad_codes(codes, scales))) || bad_dtype(dtype)) return PSGD_E_INVALID_ARG;
    if (int rc = act_shape(rows, cols, dtype)) return rc;
    if (bad_ld(ld, cols) || bad_ldc(ldc, cols) || misaligned(x) || misaligned(codes)) return PSGD_E_ALIGN;
    return act_restore(stream, rows, cols, codes, ldc, scales, x, dtype, ld, act_stream(rows, cols, dtype, 1));
}

int psgd_act_glu(void* stream, int64_t rows, int64_t cols, int act, int dtype, const void* gate, const void* up, int64_t ld_in, void* h, int64_t ld_h,
                 int8_t* gate_codes, uint8_t* gate_scales, int8_t* up_codes, uint8_t* up_scales, int64_t ldc) {
    if (bad_dtype(dtype) || (act != PSGD_SILU && act != PSGD_GELU)) return PSGD_E_INVALID_ARG;
    if (rows != 0 && (!gate || !h || bad_codes(gate_codes, gate_scales))) return PSGD_E_INVALID_ARG;
    if (rows != 0 && (up ? bad_codes(up_codes, up_scales) : (up_codes || up_scales))) return PSGD_E_INVALID_ARG;
    if (int rc = act_shape(rows, cols, dtype)) return rc;
    if (bad_ld(ld_in, cols) || bad_ld(ld_h, cols) || bad_ldc(ldc, cols) || misaligned(gate) || misaligned(up) || misaligned(h) ||
        misaligned(gate_codes) || misaligned(up_codes)) return PSGD_E_ALIGN;
    if (rows == 0) return PSGD_OK;
    const ActGrid g = act_grid(rows, cols, dtype);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    forget_errors();
    const ActOut kg = {gate_codes, gate_scales}, ku = {up_codes, up_scales};
    const bool stream_it = act_stream(rows, cols, dtype, up ? 3 : 2);
#define PSGD_GLU(T, ACT, GATED, STREAM)                                                                                                       \
    hipLaunchKernelGGL((act_glu_kernel<T, ACT, GATED, STREAM>), g.grid, dim3(kThreads), 0, st, g.rows, (const T*)gate, (const T*)up, \
                       ld_in, (T*)h, ld_h, kg, ku, ldc)
#define PSGD_GLU_STREAM(T, ACT, GATED) do { if (stream_it) PSGD_GLU(T, ACT, GATED, true); else PSGD_GLU(T, ACT, GATED, false); } while (0)
#define PSGD_GLU_ACT(T, GATED) do { if (act == PSGD_SILU) PSGD_GLU_STREAM(T, PSGD_SILU, GATED); else PSGD_GLU_STREAM(T, PSGD_GELU, GATED); } while (0)
    if (dtype == PSGD_F32) { if (up) PSGD_GLU_ACT(float, true); else PSGD_GLU_ACT(float, false); }
    else                   { if (up) PSGD_GLU_ACT(bf16_t, true); else PSGD_GLU_ACT(bf16_t, false); }
#undef PSGD_GLU
#undef PSGD_GLU_STREAM
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
    if (int rc = act_shape(rows, cols, dtype)) return rc;
    if (bad_ld(ld_h, cols) || bad_ld(ld_out, cols) || bad_ldc(ldc, cols) || misaligned(dh) || misaligned(dgate) || misaligned(dup) ||
        misaligned(gate_codes) || misaligned(up_codes)) return PSGD_E_ALIGN;
    if (rows == 0) return PSGD_OK;
    const ActGrid g = act_grid(rows, cols, dtype);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    forget_errors();
    const bool stream_it = act_stream(rows, cols, dtype, gated ? 3 : 2);
#define PSGD_GLU(T, ACT, GATED, STREAM)                                                                                                       \
    hipLaunchKernelGGL((act_glu_backward_kernel<T, ACT, GATED, STREAM>), g.grid, dim3(kThreads), 0, st, g.rows, gate_codes,    \
                       gate_scales, up_codes, up_scales, ldc, (const T*)dh, ld_h, (T*)dgate, (T*)dup, ld_out)
#define PSGD_GLU_STREAM(T, ACT, GATED) do { if (stream_it) PSGD_GLU(T, ACT, GATED, true); else PSGD_GLU(T, ACT, GATED, false); } while (0)
#define PSGD_GLU_ACT(T, GATED) do { if (act == PSGD_SILU) PSGD_GLU_STREAM(T, PSGD_SILU, GATED); else PSGD_GLU_STREAM(T, PSGD_GELU, GATED); } while (0)
    if (dtype == PSGD_F32) { if (gated) PSGD_GLU_ACT(float, true); else PSGD_GLU_ACT(float, false); }
    else                   { if (gated) PSGD_GLU_ACT(bf16_t, true); else PSGD_GLU_ACT(bf16_t, false); }
#undef PSGD_GLU
#undef PSGD_GLU_STREAM
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
    forget_errors();
    const WgradPlan w = wgrad_plan(tokens, out_features, in_features, dtype);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    bf16_t* x = reinterpret_cast<bf16_t*>(ws + w.x);
    bf16_t* planes = reinterpret_cast<bf16_t*>(ws + w.planes);
    const bool restore = !w.tile.from_codes;
    if (tokens > 0) {
        if (restore)
            if (int rc = act_restore(stream, tokens, in_features, codes, ldc, scales, x, PSGD_BF16, w.ldx, false)) return rc;
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
    const TileCodes from = {codes, ldc, scales, (int)((in_features + kGroup - 1) / kGroup)};
    return (restore ? launch_product(false, w.tile.shape, t, o, st) : launch_code_product(from, t, o, st)) == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

}  // extern "C"
