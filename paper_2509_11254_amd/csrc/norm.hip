// Layer normalisation and its gradients.
//
//   s = x, or x + add rounded to the type it is kept in;  mean = sum_c s / n,  var = sum_c (s - mean)^2 / n,  r = 1 / sqrt(var + eps)
//   u = (s - mean) r,  y = u w + b
//   g = dy w,  ds = r (g - sum_c g / n - u sum_c(g u) / n) (+ the gradient that comes past the norm),  dw = sum_rows dy u,  db = sum_rows dy
//
// A row is in the registers of one wavefront (several narrow ones are) or of four to sixteen, 16 bytes to a lane and piece; it is read once.  The variance is taken of what is left when a
// first mean is subtracted, and corrected by what is left of the mean in that: a row far from zero loses nothing to it.  The backward pass is given the sum of both, rounded:
// of rows far from zero it takes the mean of its u's and subtracts that as well.
//
// Backward, a workgroup goes through rows that are the grid apart and keeps its columns' sums of dy u and dy in registers, in fp32; it
// writes them once at its end, and a second launch adds up the workgroups' sums in their order.
#include "act_dev.h"
#include "train.h"

#include <algorithm>
#include <type_traits>

namespace psgd {

typedef float floatx2 __attribute__((ext_vector_type(2)));

constexpr int64_t kNormMaxCols = 16384;

struct NormParam { const void* ptr; int dtype; };
struct NormDev {
    int64_t rows;
    int cols;
    float eps;
    const void *x, *add;
    int64_t ld_x, ld_add;
    void *total, *y;
    int64_t ld_total, ld_y;
    NormParam w, b;
    floatx2* stats;
};
struct NormGradDev {
    int64_t rows;
    int cols;
    const void *dy, *x, *past;      // past: the gradient that comes past the norm
    int64_t ld_dy, ld_x, ld_past, ld_dx;
    void* dx;
    NormParam w;
    const floatx2* stats;
    float* part;                    // nullable; [workgroup][2][ldp]: sums of dy u and of dy
    int64_t ldp;
    // where the rows are few: workgroups from `row_blocks` on add up columns
    int row_blocks;
    void *dw, *db;
    int g_dtype, accumulate;
};

// N columns of a vector that ends at `cols`; `otherwise` where there is no vector, zeros beyond cols
template <int N>
__device__ __forceinline__ void load_param(const NormParam& p, int col, int cols, float otherwise, float (&v)[N]) {
    if (!p.ptr) {
#pragma unroll
        for (int u = 0; u < N; ++u) v[u] = col + u < cols ? otherwise : 0.f;
    } else if (p.dtype == PSGD_F32) {
        const PSGD_GLOBAL float* at = as_global(static_cast<const float*>(p.ptr)) + col;
        if (col + N <= cols) {
#pragma unroll
            for (int u = 0; u < N; u += 4) {
                const floatx4 q = *reinterpret_cast<const PSGD_GLOBAL floatx4*>(at + u);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[u + k] = q[k];
            }
        } else {
#pragma unroll
            for (int u = 0; u < N; ++u) v[u] = col + u < cols ? at[u] : 0.f;
        }
    } else {
        const PSGD_GLOBAL bf16_t* at = as_global(static_cast<const bf16_t*>(p.ptr)) + col;
        if (col + N <= cols) {
#pragma unroll
            for (int u = 0; u < N; u += 4) {
                const bf16x4 q = *reinterpret_cast<const PSGD_GLOBAL bf16x4*>(at + u);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[u + k] = (float)q[k];
            }
        } else {
#pragma unroll
            for (int u = 0; u < N; ++u) v[u] = col + u < cols ? (float)at[u] : 0.f;
        }
    }
}

// Threads of a workgroup: WAVES to a row, and where that is one, four wavefronts with a row each, or with 64 / LANES rows.
template <int WAVES> constexpr int kNormThreads = WAVES == 1 ? 256 : 64 * WAVES;
template <int WAVES, int LANES> constexpr int kNormRows = WAVES == 1 ? 256 / LANES : 1;

// sums over a row's lanes; `shared`: two sets of [K][WAVES], used in turn, so that one barrier is enough
// REGISTERS: without LDS inside a wavefront.  (Not in the backward pass, where two sums hide each other's waits: 8192 x 11008 121 us in place of 98.)
template <int WAVES, int LANES, bool REGISTERS, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float* shared, int& turn) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if constexpr (REGISTERS) {
            v[k] = lanes_sum<LANES>(v[k]);
        } else {
#pragma unroll
            for (int d = LANES / 2; d > 0; d >>= 1) v[k] += __shfl_xor(v[k], d);
        }
    }
    if constexpr (WAVES > 1) {
        float* to = shared + turn * 2 * WAVES;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) to[k * WAVES + (threadIdx.x >> 6)] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = to[k * WAVES];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) v[k] += to[k * WAVES + w];
        }
    }
}

// A rounded product: fused into the subtraction in one place and not in another, the mean would not be the same for all columns.
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

// A mean is kept in 32 bits, off by up to 2^-24 of itself, and so are all u's of the row by that times r: of nearer rows by 2^-23 at most, the size of u's own
// roundings.  Of rows beyond this their mean is asked for (16384 x 4096 with addend, all rows beyond it: 118 us, otherwise 91.5; 8192 x 11008 112, 99.5).
constexpr float kNormFar = 2.f;
__device__ __forceinline__ bool far_from_zero(const floatx2& st) { return fabsf(st.x) * st.y > kNormFar; }

// `otherwise` in the place of a piece's elements beyond cols (of bf16 twice)
template <class T>
__device__ __forceinline__ void fill_beyond(uintx4& w, const ActPlace& p, int cols, unsigned otherwise) {
    if (p.col + kPiece<T> > cols) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if constexpr (sizeof(T) == 4) {
                w[u] = p.col + u < cols ? w[u] : otherwise;
            } else {
                const unsigned in = (p.col + 2 * u < cols ? 0xffffu : 0u) | (p.col + 2 * u + 1 < cols ? 0xffff0000u : 0u);
                w[u] = (w[u] & in) | (otherwise & ~in);
            }
        }
    }
}

template <class T, int WAVES, int PIECES, int LANES, bool ADD, bool STREAM>
__global__ __launch_bounds__(kNormThreads<WAVES>) void norm_kernel(NormDev a) {
    constexpr int N = kPiece<T>;
    __shared__ float shared[4 * WAVES];
    int turn = 0;
    const int at = WAVES == 1 ? threadIdx.x % LANES : threadIdx.x, group = WAVES == 1 ? threadIdx.x / LANES : 0;
    const float inv_n = 1.f / (float)a.cols;
    float w[PIECES][N], b[PIECES][N];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int col = N * (at + LANES * WAVES * i);
        load_param<N>(a.w, col, a.cols, 1.f, w[i]);
        load_param<N>(a.b, col, a.cols, 0.f, b[i]);
    }
    const int64_t step = (int64_t)gridDim.x * kNormRows<WAVES, LANES>;
    uintx4 raw[PIECES], raw_add[PIECES];
    ActPlace p[PIECES];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            p[i].row = row, p[i].col = N * (at + LANES * WAVES * i), p[i].in = p[i].col < a.cols;
            raw[i] = load_raw<STREAM>(static_cast<const T*>(a.x), a.ld_x, p[i]);
            if constexpr (ADD) raw_add[i] = load_raw<STREAM>(static_cast<const T*>(a.add), a.ld_add, p[i]);
        }
    };
    int64_t row = (int64_t)blockIdx.x * kNormRows<WAVES, LANES> + group;
    if (row < a.rows) fetch(row);
    for (; row < a.rows; row += step) {
        float v[PIECES][N], sum[1] = {0.f};
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            p[i].row = row;
            clear_beyond<T>(raw[i], p[i], a.cols);
            widen<T>(raw[i], v[i]);
            if constexpr (ADD) {
                float o[N];
                clear_beyond<T>(raw_add[i], p[i], a.cols);
                widen<T>(raw_add[i], o);
#pragma unroll
                for (int u = 0; u < N; ++u) v[i][u] = (float)(T)(v[i][u] + o[u]);       // (what is normalised is what is kept)
                store_piece<STREAM>(static_cast<T*>(a.total), a.ld_total, p[i], a.cols, v[i]);
            }
#pragma unroll
            for (int u = 0; u < N; ++u) sum[0] += v[i][u];
        }
        if (row + step < a.rows) fetch(row + step);     // (the next row is on its way while this one is added up)
#pragma unroll
        for (int i = 0; i < PIECES; ++i) p[i].row = row;
        row_sums<WAVES, LANES, true>(sum, shared, turn);
        const float first = rounded_product(sum[0], inv_n);
        float rest[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
#pragma unroll
            for (int u = 0; u < N; ++u) v[i][u] -= first;
            if (p[i].col + N > a.cols)
#pragma unroll
                for (int u = 0; u < N; ++u) v[i][u] = p[i].col + u < a.cols ? v[i][u] : 0.f;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                rest[0] += v[i][u];
                rest[1] = fmaf(v[i][u], v[i][u], rest[1]);
            }
        }
        row_sums<WAVES, LANES, true>(rest, shared, turn);
        const float more = rounded_product(rest[0], inv_n);
        float var = fmaf(rest[1], inv_n, -more * more);
        var = var < 0.f ? 0.f : var;
        const float r = 1.f / sqrtf(var + a.eps);
        if (a.stats && at == 0) as_global(a.stats)[row] = floatx2{first + more, r};
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
#pragma unroll
            for (int u = 0; u < N; ++u) v[i][u] = fmaf((v[i][u] - more) * r, w[i][u], b[i][u]);
            store_piece<STREAM>(static_cast<T*>(a.y), a.ld_y, p[i], a.cols, v[i]);
        }
    }
}

__device__ __forceinline__ void put_sum(void* out, int dtype, int accumulate, int c, float s) {
    if (dtype == PSGD_F32) {
        PSGD_GLOBAL float* to = as_global(static_cast<float*>(out)) + c;
        *to = accumulate ? *to + s : s;
    } else {
        PSGD_GLOBAL bf16_t* to = as_global(static_cast<bf16_t*>(out)) + c;
        *to = (bf16_t)(accumulate ? (float)*to + s : s);
    }
}

// The means of what the kept means of rows far from zero leave of their u's, 0 of others': shift[row], four rows of a wavefront at a time.
constexpr int64_t kNormFewRows = 1024;
template <class T, int THREADS>
__device__ __forceinline__ void far_shifts(const NormGradDev& a, float* shift) {
    constexpr int N = kPiece<T>, W = THREADS / 64, ROWS = 4, AHEAD = 4;
    const int lane = threadIdx.x & 63;
    for (int row0 = ROWS * (threadIdx.x >> 6); row0 < (int)a.rows; row0 += ROWS * W) {
        floatx2 st[ROWS];
        float rest[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) st[i] = as_global(a.stats)[min(row0 + i, (int)a.rows - 1)], rest[i] = 0.f;
#pragma unroll 1
        for (int c0 = 0; c0 < a.cols; c0 += AHEAD * 64 * N) {
            uintx4 raw[ROWS][AHEAD];
            ActPlace p[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    p[j].row = min(row0 + i, (int)a.rows - 1), p[j].col = c0 + N * (lane + 64 * j), p[j].in = p[j].col < a.cols;
                    raw[i][j] = load_raw<false>(static_cast<const T*>(a.x), a.ld_x, p[j]);
                }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    float x[N], sum = 0.f;
                    widen<T>(raw[i][j], x);
                    if (p[j].col + N > a.cols)
#pragma unroll
                        for (int k = 0; k < N; ++k) x[k] = p[j].col + k < a.cols ? x[k] : st[i].x;
#pragma unroll
                    for (int k = 0; k < N; ++k) sum += x[k] - st[i].x;
                    rest[i] += sum;
                }
        }
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            rest[i] = lanes_sum<64>(rest[i]);
            if (lane == 0 && row0 + i < (int)a.rows) shift[row0 + i] = far_from_zero(st[i]) ? rest[i] * st[i].y / (float)a.cols : 0.f;
        }
    }
}

// dw and db of four pieces of columns, all rows: a lane has a piece of every 16th row of its wavefront's.  Where rows are far from zero each workgroup reads all of
// them once more, and its pieces of dy: the calls on such rows take longer (1000 x 515 in fp32 112 us in place of 10, 64 x 8192 49 and 9.3), the others one launch less.
template <class T, int THREADS>
__device__ __forceinline__ void norm_columns(const NormGradDev& a, int block) {
    constexpr int N = kPiece<T>, W = THREADS / 64;
    __shared__ float joined[W][4][2 * N];
    __shared__ float shift[kNormFewRows];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    ActPlace p;
    p.col = N * (4 * block + (lane & 3)), p.in = p.col < a.cols;
    float s[2 * N];
#pragma unroll
    for (int k = 0; k < 2 * N; ++k) s[k] = 0.f;
    bool far = false;
#pragma unroll 4
    for (int row = 16 * wv + (lane >> 2); row < (int)a.rows; row += 16 * W) {
        p.row = row;
        const uintx4 raw_x = load_raw<false>(static_cast<const T*>(a.x), a.ld_x, p), raw_dy = load_raw<false>(static_cast<const T*>(a.dy), a.ld_dy, p);
        const floatx2 st = as_global(a.stats)[row];
        far |= far_from_zero(st);
        float u[N], g[N];
        widen<T>(raw_x, u);
        widen<T>(raw_dy, g);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            s[k] = fmaf(g[k], (u[k] - st[0]) * st[1], s[k]);
            s[N + k] += g[k];
        }
    }
    if (__syncthreads_or(far)) {
        far_shifts<T, THREADS>(a, shift);
        __syncthreads();
#pragma unroll 4
        for (int row = 16 * wv + (lane >> 2); row < (int)a.rows; row += 16 * W) {
            p.row = row;
            float g[N];
            widen<T>(load_raw<false>(static_cast<const T*>(a.dy), a.ld_dy, p), g);
#pragma unroll
            for (int k = 0; k < N; ++k) s[k] = fmaf(g[k], -shift[row], s[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < 2 * N; ++k) {
#pragma unroll
        for (int d = 32; d >= 4; d >>= 1) s[k] += __shfl_xor(s[k], d);
        if (lane < 4) joined[wv][lane][k] = s[k];
    }
    __syncthreads();
    if (threadIdx.x < 8 * N) {
        const int piece = threadIdx.x & 3, k = threadIdx.x >> 2, c = N * (4 * block + piece) + (k < N ? k : k - N);
        float sum = joined[0][piece][k];
#pragma unroll
        for (int w = 1; w < W; ++w) sum += joined[w][piece][k];
        void* out = k < N ? a.dw : a.db;
        if (out && c < a.cols) put_sum(out, a.g_dtype, a.accumulate, c, sum);
    }
}

enum NormMode { NORM_MANY, NORM_STREAM, NORM_FEW };     // NORM_STREAM: with the non-temporal hint; NORM_FEW: sums of columns beside the rows
template <class T, int WAVES, int PIECES, int LANES, bool PAST, NormMode MODE>
__global__ __launch_bounds__(kNormThreads<WAVES>) void norm_backward_kernel(NormGradDev a) {
    constexpr int N = kPiece<T>;
    constexpr bool STREAM = MODE == NORM_STREAM;
    if constexpr (MODE == NORM_FEW)
        if ((int)blockIdx.x >= a.row_blocks) {
            norm_columns<T, kNormThreads<WAVES>>(a, blockIdx.x - a.row_blocks);
            return;
        }
    __shared__ float shared[4 * WAVES];
    int turn = 0;
    const int at = WAVES == 1 ? threadIdx.x % LANES : threadIdx.x, group = WAVES == 1 ? threadIdx.x / LANES : 0;
    const float inv_n = 1.f / (float)a.cols;
    float w[PIECES][N], dw[PIECES][N], db[PIECES][N];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        load_param<N>(a.w, N * (at + LANES * WAVES * i), a.cols, 1.f, w[i]);
#pragma unroll
        for (int u = 0; u < N; ++u) dw[i][u] = db[i][u] = 0.f;
    }
    const int64_t step = (int64_t)a.row_blocks * kNormRows<WAVES, LANES>;
    uintx4 raw_x[PIECES], raw_dy[PIECES], raw_past[PIECES];
    floatx2 stats = {0.f, 0.f};
    ActPlace p[PIECES];
    auto fetch = [&](int64_t row) {
        stats = as_global(a.stats)[row];        // (asked about first)
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            p[i].row = row, p[i].col = N * (at + LANES * WAVES * i), p[i].in = p[i].col < a.cols;
            raw_x[i] = load_raw<STREAM>(static_cast<const T*>(a.x), a.ld_x, p[i]);
            raw_dy[i] = load_raw<STREAM>(static_cast<const T*>(a.dy), a.ld_dy, p[i]);
            if constexpr (PAST) raw_past[i] = load_raw<STREAM>(static_cast<const T*>(a.past), a.ld_past, p[i]);
        }
    };
    int64_t row = (int64_t)blockIdx.x * kNormRows<WAVES, LANES> + group;
    if (row < a.rows) fetch(row);
    for (; row < a.rows; row += step) {
        const floatx2 st = stats;
        uintx4 past[PIECES];
        float u[PIECES][N], g[PIECES][N], sums[2] = {0.f, 0.f};
        float shift = 0.f;          // the mean of what the kept mean leaves of the u's
        unsigned beyond = 0;        // (beyond the columns g is 0, and u finite where the row's elements are)
        if (far_from_zero(st)) {
            float rest[1] = {0.f};
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                float x[N];
                widen<T>(raw_x[i], x);
#pragma unroll
                for (int k = 0; k < N; ++k) rest[0] += p[i].col + k < a.cols ? (x[k] - st.x) * st.y : 0.f;
            }
            row_sums<WAVES, LANES, true>(rest, shared, turn);
            shift = rest[0] * inv_n;
            const PSGD_GLOBAL T* first = as_global(static_cast<const T*>(a.x)) + row * a.ld_x;
            if constexpr (sizeof(T) == 4) beyond = *reinterpret_cast<const PSGD_GLOBAL unsigned*>(first);
            else beyond = *reinterpret_cast<const PSGD_GLOBAL unsigned short*>(first) * 0x10001u;
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            fill_beyond<T>(raw_x[i], p[i], a.cols, beyond);
            clear_beyond<T>(raw_dy[i], p[i], a.cols);
            widen<T>(raw_x[i], u[i]);
            widen<T>(raw_dy[i], g[i]);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                u[i][k] = fmaf(u[i][k] - st.x, st.y, -shift);
                dw[i][k] = fmaf(g[i][k], u[i][k], dw[i][k]);
                db[i][k] += g[i][k];
                g[i][k] *= w[i][k];
                sums[0] += g[i][k];
                sums[1] = fmaf(g[i][k], u[i][k], sums[1]);
            }
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) past[i] = raw_past[i];
        if (row + step < a.rows) fetch(row + step);     // (the next row is on its way while this one is added up)
        row_sums<WAVES, LANES, false>(sums, shared, turn);
        const float c1 = sums[0] * inv_n, c2 = sums[1] * inv_n;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            float o[N];
            p[i].row = row;
            if constexpr (PAST) widen<T>(past[i], o);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float d = st.y * (g[i][k] - fmaf(u[i][k], c2, c1));
                g[i][k] = PAST ? o[k] + d : d;
            }
            store_piece<STREAM>(static_cast<T*>(a.dx), a.ld_dx, p[i], a.cols, g[i]);
        }
    }
    if (MODE == NORM_FEW || !a.part) return;
    constexpr int SPAN = LANES * WAVES * PIECES * N;
    if constexpr (WAVES == 1) {         // the sums of a wavefront's rows, and then the four wavefronts' in their order
        __shared__ float joined[2 * SPAN];
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k)
#pragma unroll
                for (int d = 32; d >= LANES; d >>= 1) dw[i][k] += __shfl_xor(dw[i][k], d), db[i][k] += __shfl_xor(db[i][k], d);
        for (int from = 0; from < 4; ++from) {
            if ((int)(threadIdx.x >> 6) == from && (threadIdx.x & 63) < LANES)
#pragma unroll
                for (int i = 0; i < PIECES; ++i)
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const int c = N * (at + LANES * i) + k;
                        joined[c] = from ? joined[c] + dw[i][k] : dw[i][k];
                        joined[SPAN + c] = from ? joined[SPAN + c] + db[i][k] : db[i][k];
                    }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < a.cols; c += 256) {
            as_global(a.part)[(int64_t)blockIdx.x * 2 * a.ldp + c] = joined[c];
            as_global(a.part)[((int64_t)blockIdx.x * 2 + 1) * a.ldp + c] = joined[SPAN + c];
        }
    } else {
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                const int c = N * (at + LANES * WAVES * i) + k;
                if (c >= a.cols) break;         // (the rows of `part` are a multiple of 8 long)
                PSGD_GLOBAL float* to = as_global(a.part) + (int64_t)blockIdx.x * 2 * a.ldp + c;
                *reinterpret_cast<PSGD_GLOBAL floatx4*>(to) = floatx4{dw[i][k], dw[i][k + 1], dw[i][k + 2], dw[i][k + 3]};
                *reinterpret_cast<PSGD_GLOBAL floatx4*>(to + a.ldp) = floatx4{db[i][k], db[i][k + 1], db[i][k + 2], db[i][k + 3]};
            }
    }
}

// sums of the workgroups' sums: 64 columns to a block, 16 threads to a column; blockIdx.y: the weight's or the bias's
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float* part, int64_t ldp, int n_parts, int cols, void* dw, void* db, int dtype, int accumulate) {
    __shared__ float shared[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
    void* out = blockIdx.y ? db : dw;
    if (!out) return;
    float s = 0.f;
    if (c < cols) {
#pragma unroll 4
        for (int i = slice; i < n_parts; i += 16) s += as_global(part)[((int64_t)i * 2 + blockIdx.y) * ldp + c];
    }
    shared[slice][threadIdx.x & 63] = s;
    __syncthreads();
    if (slice == 0 && c < cols) {
#pragma unroll
        for (int i = 1; i < 16; ++i) s += shared[i][threadIdx.x];
        put_sum(out, dtype, accumulate, c, s);
    }
}

// ---- host --------------------------------------------------------------------------------------------------------------

// Wavefronts to a row and pieces to a lane.  One wavefront needs no barrier, and has a row of up to four pieces to a lane; wider rows have four wavefronts
// or eight with as few pieces as do (16384 x 4096 with addend, in us, of (4, 2), (8, 1), (2, 4), each with its best grid: forward 90.0, 90.7, 92.9, backward 95.8, 90.8,
// 98.9; 8192 x 8192 of (4, 4), (8, 2), (16, 1): 93.8, 91.2, 106.4, 96.2, 93.3, 93.2; 8192 x 11008 without one of (8, 3), (16, 2): 65.9, 95.4, 99.0, 167;
// 16384 x 2048 of (1, 4), (2, 2), (4, 1): 46.2, 46.6, 47.2, 54.0, 54.7, 52.2, the last with a grid of its own, and 67.1 with the others').  Beyond 12288 columns
// in bf16 and 8192 in fp32 the backward pass keeps part of a row in scratch: 8192 x 16384 in bf16 322 us, 3.3 TB/s, 8192 x 11008 and 4096 x 16384 in fp32 404 and 525, 3.6 and 2.0, with
// what comes past the norm.  Rows of up to 512 bytes lie beside each other in a wavefront (60000 rows in bf16, forward and
// backward, in us, with a wavefront each and so: of 64 columns 21.7 and 32.8, 7.9 and 12.9; of 256 22.9 and 33.8, 13.0 and 23.7).
struct NormShape { int waves, pieces, lanes = 64; };
static NormShape norm_variant(int64_t cols, int dtype, bool backward) {
    const int n = (int)((cols + (dtype == PSGD_F32 ? 3 : 7)) / (dtype == PSGD_F32 ? 4 : 8));
    if (n <= 32) return {1, 1, n <= 8 ? 8 : n <= 16 ? 16 : 32};
    if (n <= 256) return {1, (n + 63) / 64};
    if (n <= 512) return backward ? NormShape{8, 1} : NormShape{4, 2};
    if (n <= 2048) return {8, (n + 511) / 512};
    return {16, (n + 1023) / 1024};
}
// Workgroups.  Forward, rows in flight: too many streams of addresses cost as much as too few loads (16384 x 4096, 512, 1024 and 2048 workgroups: with addend 90.0, 98.2 and
// 100.5 us, without 60.1, 47.1, 51.0).  Backward, one to a compute unit, or two of one wavefront to a row: each has its columns' sums written and read (16384 x 4096 with 256, 512 and
// 1024: 90.8, 98.4 and 102.8 us).
static int norm_blocks(int64_t rows, const NormShape& v, int most) {
    const int per = v.waves == 1 ? 256 / v.lanes : 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>((rows + per - 1) / per, most));
}
static int forward_blocks(const NormShape& v, bool add) { return add || v.waves >= 8 ? 512 : 1024; }
static int backward_blocks(const NormShape& v) { return v.waves == 1 && v.pieces < 4 ? 512 : 256; }
// Few rows: the sums of columns are made beside the rows, in one launch, from another reading of them.  (Calls of 1000 x 515 in fp32 9.8 us, with sums of workgroups and a
// second launch 12.3; 200 x 1000 in bf16 9.6, 12.6; of 1024 x 4096, 8 MB, 14.9 and 15.1, where nothing is gained that rows far from zero would not cost.)
constexpr int64_t kNormFewBytes = 9 << 18;
// From this many bytes in a call on activations have the non-temporal hint (as those of act.hip).
constexpr int64_t kNormStream = 96 << 20;

static int norm_shape(int64_t rows, int64_t cols) {
    return rows < 0 || cols < 1 || rows > kMaxExtent || cols > kNormMaxCols ? PSGD_E_SHAPE : PSGD_OK;
}
// an output may take the place of an input of the same layout
static bool bad_place(const RowArea& out, const RowArea& in) {
    return overlap(out, in) && !(out.ptr == in.ptr && (out.stride == in.stride || out.rows == 1) && out.width == in.width);
}

// launch(waves, pieces, lanes) with constants
template <class T, bool BACKWARD, class F>
static hipError_t norm_dispatch(const NormShape& v, F launch) {
#define PSGD_LANES(W, P, L) \
    if (v.waves == W && v.pieces == P && v.lanes == L) return launch(std::integral_constant<int, W>{}, std::integral_constant<int, P>{}, std::integral_constant<int, L>{})
#define PSGD_SHAPE(W, P) PSGD_LANES(W, P, 64)
    PSGD_LANES(1, 1, 8);
    PSGD_LANES(1, 1, 16);
    PSGD_LANES(1, 1, 32);
    PSGD_SHAPE(1, 1);
    PSGD_SHAPE(1, 2);
    PSGD_SHAPE(1, 3);
    PSGD_SHAPE(1, 4);
    if constexpr (BACKWARD) { PSGD_SHAPE(8, 1); }
    else { PSGD_SHAPE(4, 2); }
    PSGD_SHAPE(8, 2);
    PSGD_SHAPE(8, 3);
    PSGD_SHAPE(8, 4);
    if constexpr (sizeof(T) == 4) {
        PSGD_SHAPE(16, 3);
        PSGD_SHAPE(16, 4);
    }
#undef PSGD_SHAPE
#undef PSGD_LANES
    return hipErrorInvalidValue;
}

template <class T, bool ADD, bool STREAM>
static hipError_t launch_norm_as(const NormDev& a, const NormShape& v, hipStream_t st) {
    const int blocks = norm_blocks(a.rows, v, forward_blocks(v, ADD));
    return norm_dispatch<T, false>(v, [&](auto waves, auto pieces, auto lanes) {
        hipLaunchKernelGGL((norm_kernel<T, waves.value, pieces.value, lanes.value, ADD, STREAM>), dim3(blocks), dim3(kNormThreads<waves.value>), 0, st, a);
        return hipGetLastError();
    });
}
template <class T, bool PAST, NormMode MODE>
static hipError_t launch_backward_as(const NormGradDev& a, const NormShape& v, hipStream_t st) {
    const int per = 4 * kPiece<T>, blocks = a.row_blocks + (a.dw || a.db ? (a.cols + per - 1) / per : 0);
    return norm_dispatch<T, true>(v, [&](auto waves, auto pieces, auto lanes) {
        hipLaunchKernelGGL((norm_backward_kernel<T, waves.value, pieces.value, lanes.value, PAST, MODE>), dim3(blocks), dim3(kNormThreads<waves.value>), 0, st, a);
        return hipGetLastError();
    });
}

}  // namespace psgd

using namespace psgd;

extern "C" {

int psgd_norm(void* stream, int64_t rows, int64_t cols, int dtype, const void* x, int64_t ld_x, const void* add, int64_t ld_add, const void* weight,
              const void* bias, int w_dtype, float eps, void* total, int64_t ld_total, void* y, int64_t ld_y, float* stats) {
    if (bad_dtype(dtype) || bad_dtype(w_dtype) || !(eps >= 0.f && eps < __builtin_inff())) return PSGD_E_INVALID_ARG;
    if (rows != 0 && (!x || !y || (add == nullptr) != (total == nullptr))) return PSGD_E_INVALID_ARG;
    if (int rc = norm_shape(rows, cols)) return rc;
    if (bad_ld(ld_x, cols) || bad_ld(ld_y, cols) || (add && (bad_ld(ld_add, cols) || bad_ld(ld_total, cols))) || misaligned(x) || misaligned(add) || misaligned(weight) || misaligned(bias) || misaligned(total) ||
        misaligned(y) || misaligned(stats)) return PSGD_E_ALIGN;
    if (ld_x > kMaxLd || ld_y > kMaxLd || (add && (ld_add > kMaxLd || ld_total > kMaxLd))) return PSGD_E_SHAPE;
    if (rows == 0) return PSGD_OK;
    const int64_t size = dtype == PSGD_F32 ? 4 : 2, w_size = w_dtype == PSGD_F32 ? 4 : 2;
    const RowArea in[] = {{x, rows, ld_x * size, cols * size}, {add, rows, ld_add * size, cols * size}};
    const RowArea params[] = {{weight, 1, 0, cols * w_size}, {bias, 1, 0, cols * w_size}};
    const RowArea out[] = {{total, rows, ld_total * size, cols * size}, {y, rows, ld_y * size, cols * size}, {stats, 1, 0, rows * 8}};
    for (int i = 0; i < 3; ++i) {
        for (const RowArea& a : in)
            if (i == 2 ? overlap(out[i], a) : bad_place(out[i], a)) return PSGD_E_INVALID_ARG;
        for (const RowArea& a : params)
            if (overlap(out[i], a)) return PSGD_E_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return PSGD_E_INVALID_ARG;
    }
    const NormDev a = {rows, (int)cols, eps, x, add, ld_x, ld_add, total, y, ld_total, ld_y, {weight, w_dtype}, {bias, w_dtype}, reinterpret_cast<floatx2*>(stats)};
    const NormShape v = norm_variant(cols, dtype, false);
    const bool stream_it = rows * cols * size * (add ? 4 : 2) >= kNormStream;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    forget_errors();
    hipError_t e;
#define PSGD_NORM(T, ADD) (stream_it ? launch_norm_as<T, ADD, true>(a, v, st) : launch_norm_as<T, ADD, false>(a, v, st))
    if (dtype == PSGD_F32) e = add ? PSGD_NORM(float, true) : PSGD_NORM(float, false);
    else e = add ? PSGD_NORM(bf16_t, true) : PSGD_NORM(bf16_t, false);
#undef PSGD_NORM
    return e == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

size_t psgd_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int dtype) {
    if (bad_dtype(dtype) || norm_shape(rows, cols)) return 0;
    return up256((size_t)norm_blocks(rows, norm_variant(cols, dtype, true), backward_blocks(norm_variant(cols, dtype, true))) * 2 * up8(cols) * sizeof(float));
}

int psgd_norm_backward(void* workspace, void* stream, int64_t rows, int64_t cols, int dtype, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x,
                       const void* weight, int w_dtype, const float* stats, const void* dtotal, int64_t ld_dtotal, void* dx, int64_t ld_dx, void* dweight,
                       void* dbias, int g_dtype, int accumulate) {
    const bool sums = dweight || dbias;
    if (bad_dtype(dtype) || bad_dtype(w_dtype) || bad_dtype(g_dtype) || (sums && !workspace)) return PSGD_E_INVALID_ARG;
    if (rows != 0 && (!dy || !x || !stats || !dx)) return PSGD_E_INVALID_ARG;
    if (int rc = norm_shape(rows, cols)) return rc;
    if (bad_ld(ld_dy, cols) || bad_ld(ld_x, cols) || (dtotal && bad_ld(ld_dtotal, cols)) || bad_ld(ld_dx, cols) || misaligned(dy) || misaligned(x) || misaligned(weight) || misaligned(stats) ||
        misaligned(dtotal) || misaligned(dx) || misaligned(dweight) || misaligned(dbias) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PSGD_E_ALIGN;
    if (ld_dy > kMaxLd || ld_x > kMaxLd || (dtotal && ld_dtotal > kMaxLd) || ld_dx > kMaxLd) return PSGD_E_SHAPE;
    const int64_t size = dtype == PSGD_F32 ? 4 : 2, w_size = w_dtype == PSGD_F32 ? 4 : 2, g_size = g_dtype == PSGD_F32 ? 4 : 2;
    const RowArea in[] = {{dy, rows, ld_dy * size, cols * size}, {x, rows, ld_x * size, cols * size}, {dtotal, rows, ld_dtotal * size, cols * size},
                          {weight, 1, 0, cols * w_size}, {stats, 1, 0, rows * 8}};
    const RowArea out[] = {{dx, rows, ld_dx * size, cols * size}, {dweight, 1, 0, cols * g_size}, {dbias, 1, 0, cols * g_size}};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 5; ++j)
            if (i == 0 && j < 3 ? bad_place(out[i], in[j]) : overlap(out[i], in[j])) return PSGD_E_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return PSGD_E_INVALID_ARG;
    }
    if (rows == 0 && (!sums || accumulate)) return PSGD_OK;
    NormGradDev a = {rows, (int)cols, dy, x, dtotal, ld_dy, ld_x, ld_dtotal, ld_dx, dx, {weight, w_dtype}, reinterpret_cast<const floatx2*>(stats),
                     nullptr, up8(cols)};
    const NormShape v = norm_variant(cols, dtype, true);
    const bool few = rows <= kNormFewRows && rows * cols * size <= kNormFewBytes && dx != dy && dx != x;       // (where dx takes their place, the columns would find some rows written)
    if (sums && few) a.dw = dweight, a.db = dbias, a.g_dtype = g_dtype, a.accumulate = accumulate != 0;
    else if (sums) a.part = static_cast<float*>(workspace);
    a.row_blocks = norm_blocks(rows, v, few ? (int)kNormFewRows : backward_blocks(v));
    const bool stream_it = !few && rows * cols * size * (dtotal ? 4 : 3) >= kNormStream;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    forget_errors();
    if (rows != 0) {
        hipError_t e;
#define PSGD_NORM(T, PAST) \
    (few ? launch_backward_as<T, PAST, NORM_FEW>(a, v, st) : stream_it ? launch_backward_as<T, PAST, NORM_STREAM>(a, v, st) : launch_backward_as<T, PAST, NORM_MANY>(a, v, st))
        if (dtype == PSGD_F32) e = dtotal ? PSGD_NORM(float, true) : PSGD_NORM(float, false);
        else e = dtotal ? PSGD_NORM(bf16_t, true) : PSGD_NORM(bf16_t, false);
#undef PSGD_NORM
        if (e != hipSuccess) return PSGD_E_HIP;
    }
    if (!sums || (few && rows)) return PSGD_OK;
    hipLaunchKernelGGL(norm_sum_kernel, dim3((unsigned)((cols + 63) / 64), 2), dim3(1024), 0, st, a.part, a.ldp, rows ? a.row_blocks : 0, (int)cols, dweight, dbias,
                       g_dtype, accumulate != 0);
    return hipGetLastError() == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

}  // extern "C"
