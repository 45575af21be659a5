// Tokens sorted by the experts they chose, their rows in that order, and the experts' rows back at their tokens, added up with weights.
//
//   place[t, s]   the row of token t's choice s, counted through the experts in their order and within one through the choices in theirs; -1: it does not count
//   Xs[place[t, s]] = X[t],  Y[t] = sum_s w[t, s] Ys[place[t, s]]  (with w = 1 the gradient of X from Xs'),  dYs[place[t, s]] = w[t, s] dY[t],
//   dw[t, s] = dY[t] . Ys[place[t, s]]
//
// The sort counts: how often each expert is chosen before each choice.  A workgroup has a run of the choices, each wavefront a part of it.
// Of 64 choices next to each other, a ballot for every bit of the expert's number says which are the same.
// The rows' kernels move each row once; HBM bounds them.
#include "act_dev.h"
#include "train.h"

#include <algorithm>

namespace psgd {

constexpr int kMaxExperts = 1024;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
// Choices that one workgroup sorts alone (64 experts, us: 1600 choices 5.7, 4096 7.8; 8000 alone 11.7, 8200 by two launches 8.5; a launch takes the host 3).
constexpr int64_t kSortOneBlock = 4096;
constexpr int kSortBlocks = 256;            // workgroups at most, each of which reads all others' counts

struct SortDev {
    const int64_t* choice;
    int64_t n;
    int per;            // choices of a wavefront, a multiple of 64
    int experts, bits;
    int* counts;        // nullable (one workgroup); [workgroup][experts + 1], the last: choices that do not count
    int *place, *order, *offsets;
};

__device__ __forceinline__ int sort_class(const SortDev& a, int64_t i) {
    const int64_t e = as_global(a.choice)[i];
    return e >= 0 && e < a.experts ? (int)e : a.experts;
}

__global__ __launch_bounds__(kSortThreads) void expert_count_kernel(SortDev a) {
    extern __shared__ int count[];      // [experts + 1]
    for (int e = threadIdx.x; e <= a.experts; e += kSortThreads) count[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * a.per * kSortWaves, last = min(a.n, first + (int64_t)a.per * kSortWaves);
    for (int64_t i = first + threadIdx.x; i < last; i += kSortThreads) atomicAdd(&count[sort_class(a, i)], 1);
    __syncthreads();
    for (int e = threadIdx.x; e <= a.experts; e += kSortThreads) as_global(a.counts)[(int64_t)blockIdx.x * (a.experts + 1) + e] = count[e];
}

__global__ __launch_bounds__(kSortThreads) void expert_place_kernel(SortDev a) {
    extern __shared__ int shared[];
    const int classes = a.experts + 1, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    int* next = shared;                             // [wavefronts][classes]: where the wavefront's next choice of a class goes
    int* total = shared + kSortWaves * classes;     // [classes]
    int* before = total + classes;                  // [classes]: of the workgroups before this one
    int* carry = before + classes;                  // [wavefronts]
    for (int i = threadIdx.x; i < (kSortWaves + 2) * classes; i += kSortThreads) shared[i] = 0;
    __syncthreads();
    const int64_t first = ((int64_t)blockIdx.x * kSortWaves + wv) * a.per, last = min(a.n, first + a.per);
#pragma unroll 4
    for (int64_t i = first + lane; i < last; i += 64) atomicAdd(&next[wv * classes + sort_class(a, i)], 1);
    // (whole numbers: in whatever order they are added up)
    if (a.counts)
        for (int e = lane; e < classes; e += 64) {
            int all = 0, earlier = 0;
            for (int b0 = wv; b0 < (int)gridDim.x; b0 += 8 * kSortWaves) {
                int c[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int b = b0 + k * kSortWaves;
                    c[k] = b < (int)gridDim.x ? as_global(a.counts)[b * classes + e] : 0;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    all += c[k];
                    earlier += b0 + k * kSortWaves < (int)blockIdx.x ? c[k] : 0;
                }
            }
            if (all) atomicAdd(&total[e], all);
            if (earlier) atomicAdd(&before[e], earlier);
        }
    __syncthreads();
    // first row of each class: a thread each (kMaxExperts + 1 classes and no more than twice the threads)
    int sum = 0;
    for (int round = 0; round < classes; round += kSortThreads) {
        const int e = round + threadIdx.x;
        int of_wave[kSortWaves], mine = 0;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            of_wave[w] = e < classes ? next[w * classes + e] : 0;
            mine += of_wave[w];
        }
        if (a.counts) mine = e < classes ? total[e] : 0;
        int up = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(up, d);
            up += lane >= d ? o : 0;
        }
        if (lane == 63) carry[wv] = up;
        __syncthreads();
        int base = sum;
        for (int w = 0; w < kSortWaves; ++w) {
            base += w < wv ? carry[w] : 0;
            sum += carry[w];
        }
        const int start = base + up - mine;
        if (e < classes) {
            if (blockIdx.x == 0) as_global(a.offsets)[e] = start;       // (the last class' is the number of choices that count)
            int at = start + before[e];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                next[w * classes + e] = at;
                at += of_wave[w];
            }
        }
        __syncthreads();
    }
    int ahead = first + lane < last ? sort_class(a, first + lane) : 0;
    for (int64_t i0 = first; i0 < last; i0 += 64) {
        const int64_t i = i0 + lane;
        const bool in = i < last;
        const int e = ahead;
        ahead = i + 64 < last ? sort_class(a, i + 64) : 0;
        unsigned long long same = __ballot(in);
        for (int b = 0; b < a.bits; ++b) {
            const unsigned long long set = __ballot((e >> b) & 1);
            same &= (e >> b) & 1 ? set : ~set;
        }
        const int leader = __ffsll((long long)same) - 1, rank = __popcll(same & ((1ull << lane) - 1));
        int at = 0;
        if (in && rank == 0) at = atomicAdd(&next[wv * classes + e], (int)__popcll(same));
        at = __shfl(at, in ? leader : lane) + rank;
        if (in) {
            as_global(a.place)[i] = e < a.experts ? at : -1;
            as_global(a.order)[at] = e < a.experts ? (int)i : -1;
        }
    }
}

// ---- rows ----------------------------------------------------------------------------------------------------------------

struct RowsDev {
    int64_t tokens, n;      // n: tokens * slots
    int slots, cols;
    const int* place;
    const float* weight;    // nullable
    const void *in, *dy;
    int64_t ld_in, ld_dy;
    void* out;
    int64_t ld_out;
    float* dweight;         // nullable
};

// row of choice i; -1: none.  LANES: those of a wavefront that ask for the same
template <int LANES>
__device__ __forceinline__ int row_of(const RowsDev& a, int64_t i) {
    const int p = as_global(a.place)[i], row = (unsigned)p < (unsigned)a.n ? p : -1;
    return LANES == 64 ? __builtin_amdgcn_readfirstlane(row) : row;
}

// (A wavefront to a token, with two, four or eight of its rows at a time, reads dY once, which comes from the caches here, and is slower: gradients of 16384 tokens of eight
// rows of 2048 in bf16 200 us so, 5.7 TB/s, and 226 to 233 us; 8192 tokens of two rows of 4096 53, and 60 to 63.  Nor does a smaller grid gain anything: 212 to 217 us.)
// a wavefront to each choice: X[t] to its row (SCALE: times its weight, and the dot product with Ys' row)
// LANES: of a choice, 16 or 32 where a row has no more pieces; PIECES: of a lane at a time (16384 x 8 choices, rows of 64, 256 and 512 in bf16, gradients: 76, 80 and 88 us with
// (64, 4) for all, 11, 29 and 57 so).
template <class T, int LANES, int PIECES, bool SCALE, bool DOT, bool STREAM>
__global__ __launch_bounds__(kThreads) void expert_rows_kernel(RowsDev a) {
    constexpr int N = kPiece<T>, ROWS = kThreads / LANES;
    const int lane = threadIdx.x % LANES;
    for (int64_t i = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; i < a.n; i += (int64_t)gridDim.x * ROWS) {
        const int row = row_of<LANES>(a, i);
        if (row < 0) {
            if (DOT && lane == 0) as_global(a.dweight)[i] = 0.f;
            continue;
        }
        const int64_t t = (unsigned)i / (unsigned)a.slots;
        const float w = SCALE && a.weight ? as_global(a.weight)[i] : 1.f;
        float dot = 0.f;
        for (int c0 = 0; c0 < a.cols; c0 += PIECES * LANES * N) {
            uintx4 raw[PIECES], raw_y[PIECES];
            ActPlace p[PIECES];
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                p[k].row = t, p[k].col = c0 + N * (lane + LANES * k), p[k].in = p[k].col < a.cols;
                raw[k] = load_raw<false>(static_cast<const T*>(a.dy), a.ld_dy, p[k]);
                p[k].row = row;
                if constexpr (DOT) raw_y[k] = load_raw<STREAM>(static_cast<const T*>(a.in), a.ld_in, p[k]);
            }
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                float v[N];
                if (!SCALE && p[k].col + N <= a.cols) {         // (as it is)
                    st_act<STREAM>(reinterpret_cast<PSGD_GLOBAL uintx4*>(as_global(static_cast<T*>(a.out)) + p[k].row * a.ld_out + p[k].col), raw[k]);
                    continue;
                }
                if constexpr (DOT) {
                    float y[N];
                    clear_beyond<T>(raw[k], p[k], a.cols);
                    clear_beyond<T>(raw_y[k], p[k], a.cols);
                    widen<T>(raw_y[k], y);
                    widen<T>(raw[k], v);
#pragma unroll
                    for (int u = 0; u < N; ++u) dot = fmaf(v[u], y[u], dot);
                } else {
                    widen<T>(raw[k], v);
                }
                if constexpr (SCALE)
#pragma unroll
                    for (int u = 0; u < N; ++u) v[u] *= w;
                store_piece<STREAM>(static_cast<T*>(a.out), a.ld_out, p[k], a.cols, v);
            }
        }
        if constexpr (DOT) {
            dot = lanes_sum<LANES>(dot);
            if (lane == 0) as_global(a.dweight)[i] = dot;
        }
    }
}

// a wavefront to each token and 64 pieces of its columns, or 16 or 32 lanes to a token: the sum of its rows
template <class T, int LANES, bool STREAM>
__global__ __launch_bounds__(kThreads) void expert_combine_kernel(RowsDev a, int parts) {
    constexpr int N = kPiece<T>, AHEAD = 4, ROWS = kThreads / LANES;
    const int lane = threadIdx.x % LANES;
    const int64_t all = a.tokens * parts;
    for (int64_t j = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; j < all; j += (int64_t)gridDim.x * ROWS) {
        const int64_t t = j / parts;
        ActPlace p;
        p.col = N * ((int)(j - t * parts) * LANES + lane);
        float sum[N];
#pragma unroll
        for (int u = 0; u < N; ++u) sum[u] = 0.f;
        for (int s0 = 0; s0 < a.slots; s0 += AHEAD) {
            uintx4 raw[AHEAD];
            float w[AHEAD];
            bool there[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int64_t i = t * a.slots + s0 + k;
                const int row = s0 + k < a.slots ? row_of<LANES>(a, i) : -1;
                there[k] = row >= 0;
                w[k] = there[k] && a.weight ? as_global(a.weight)[i] : 1.f;
                p.row = row, p.in = there[k] && p.col < a.cols;
                raw[k] = load_raw<STREAM>(static_cast<const T*>(a.in), a.ld_in, p);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (there[k]) {
                    float v[N];
                    widen<T>(raw[k], v);
#pragma unroll
                    for (int u = 0; u < N; ++u) sum[u] = fmaf(v[u], w[k], sum[u]);
                }
        }
        p.row = t, p.in = p.col < a.cols;
        store_piece<STREAM>(static_cast<T*>(a.out), a.ld_out, p, a.cols, sum);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------

constexpr int64_t kRowStream = 96 << 20;        // bytes of a call's rows from which on they have the non-temporal hint (as act.hip's)
constexpr int64_t kRowBlocks = 1 << 20;

static int sort_shape(int64_t tokens, int64_t slots, int64_t experts) {
    if (tokens < 0 || slots < 1 || experts < 1 || experts > kMaxExperts || tokens > kMaxExtent || slots > kMaxExtent || tokens * slots > kMaxExtent) return PSGD_E_SHAPE;
    return PSGD_OK;
}
struct SortPlan { int blocks, per; };
static SortPlan sort_plan(int64_t n) {
    const int64_t most = n <= kSortOneBlock ? 1 : kSortBlocks;
    SortPlan p;
    p.per = (int)((n + most * kSortThreads - 1) / (most * kSortThreads) * 64);
    p.per = std::max(p.per, 64);
    p.blocks = (int)std::max<int64_t>(1, (n + (int64_t)p.per * kSortWaves - 1) / ((int64_t)p.per * kSortWaves));
    return p;
}
static int rows_shape(int64_t tokens, int64_t slots, int64_t cols) {
    if (tokens < 0 || slots < 1 || cols < 1 || tokens > kMaxExtent || slots > kMaxExtent || tokens * slots > kMaxExtent || cols > kMaxLd) return PSGD_E_SHAPE;
    return PSGD_OK;
}
static unsigned row_blocks(int64_t rows, int lanes) { return (unsigned)std::min<int64_t>((rows * lanes + kThreads - 1) / kThreads, kRowBlocks); }
static int row_pieces(int64_t cols, int dtype) { return (int)((cols + (dtype == PSGD_F32 ? 3 : 7)) / (dtype == PSGD_F32 ? 4 : 8)); }
static bool same_place(const RowArea& a, const RowArea& b) { return a.ptr == b.ptr && (a.stride == b.stride || a.rows == 1) && a.width == b.width; }

template <class T, bool SCALE, bool DOT>
static int launch_rows_as(const RowsDev& a, int pieces, hipStream_t st) {
    const bool stream_it = a.n * a.cols * (int64_t)sizeof(T) * (DOT ? 2 : 1) >= kRowStream;
    forget_errors();
#define PSGD_ROWS(LANES, PIECES, STREAM) \
    hipLaunchKernelGGL((expert_rows_kernel<T, LANES, PIECES, SCALE, DOT, STREAM>), dim3(row_blocks(a.n, LANES)), dim3(kThreads), 0, st, a)
    if (pieces <= 16) { if (stream_it) PSGD_ROWS(16, 1, true); else PSGD_ROWS(16, 1, false); }
    else if (pieces <= 32) { if (stream_it) PSGD_ROWS(32, 1, true); else PSGD_ROWS(32, 1, false); }
    else if (pieces <= 64) { if (stream_it) PSGD_ROWS(64, 1, true); else PSGD_ROWS(64, 1, false); }
    else { if (stream_it) PSGD_ROWS(64, 4, true); else PSGD_ROWS(64, 4, false); }
#undef PSGD_ROWS
    return hipGetLastError() == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}
template <bool SCALE, bool DOT>
static int launch_rows(const RowsDev& a, int dtype, hipStream_t st) {
    const int pieces = row_pieces(a.cols, dtype);
    return dtype == PSGD_F32 ? launch_rows_as<float, SCALE, DOT>(a, pieces, st) : launch_rows_as<bf16_t, SCALE, DOT>(a, pieces, st);
}

}  // namespace psgd

using namespace psgd;

extern "C" {

size_t psgd_expert_sort_workspace_bytes(int64_t tokens, int64_t slots, int64_t experts) {
    if (sort_shape(tokens, slots, experts)) return 0;
    return up256((size_t)sort_plan(tokens * slots).blocks * (experts + 1) * sizeof(int));
}

int psgd_expert_sort(void* workspace, void* stream, int64_t tokens, int64_t slots, int64_t experts, const int64_t* choice, int32_t* place, int32_t* order,
                     int32_t* offsets) {
    if (!workspace || !offsets || (tokens != 0 && (!choice || !place || !order))) return PSGD_E_INVALID_ARG;
    if (int rc = sort_shape(tokens, slots, experts)) return rc;
    if (misaligned(choice) || misaligned(place) || misaligned(order) || misaligned(offsets) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PSGD_E_ALIGN;
    const int64_t n = tokens * slots;
    const RowArea areas[] = {{place, 1, 0, n * 4}, {order, 1, 0, n * 4}, {offsets, 1, 0, (experts + 1) * 4}, {choice, 1, 0, n * 8}};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 4; ++j)
            if (overlap(areas[i], areas[j])) return PSGD_E_INVALID_ARG;
    const SortPlan p = sort_plan(n);
    SortDev a = {choice, n, p.per, (int)experts, 0, p.blocks > 1 ? static_cast<int*>(workspace) : nullptr, place, order, offsets};
    while ((experts >> a.bits) != 0) ++a.bits;      // (class `experts` is one of them)
    const int classes = (int)experts + 1, lds = ((kSortWaves + 2) * classes + kSortWaves) * 4;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    forget_errors();
    if (lds > 48 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void*>(expert_place_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
        return PSGD_E_HIP;
    if (a.counts) {
        hipLaunchKernelGGL(expert_count_kernel, dim3(p.blocks), dim3(kSortThreads), classes * 4, st, a);
        if (hipGetLastError() != hipSuccess) return PSGD_E_HIP;
    }
    hipLaunchKernelGGL(expert_place_kernel, dim3(p.blocks), dim3(kSortThreads), lds, st, a);
    return hipGetLastError() == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

int psgd_expert_rows(void* stream, int64_t tokens, int64_t slots, int64_t cols, int dtype, const void* x, int64_t ld_x, const int32_t* place, void* xs,
                     int64_t ld_xs) {
    if (bad_dtype(dtype) || (tokens != 0 && (!x || !place || !xs))) return PSGD_E_INVALID_ARG;
    if (int rc = rows_shape(tokens, slots, cols)) return rc;
    if (bad_ld(ld_x, cols) || bad_ld(ld_xs, cols) || misaligned(x) || misaligned(place) || misaligned(xs)) return PSGD_E_ALIGN;
    if (ld_x > kMaxLd || ld_xs > kMaxLd) return PSGD_E_SHAPE;
    if (tokens == 0) return PSGD_OK;
    const int64_t size = dtype == PSGD_F32 ? 4 : 2, n = tokens * slots;
    const RowArea out = {xs, n, ld_xs * size, cols * size};
    if (overlap(out, {x, tokens, ld_x * size, cols * size}) || overlap(out, {place, 1, 0, n * 4})) return PSGD_E_INVALID_ARG;
    RowsDev a = {};
    a.tokens = tokens, a.n = n, a.slots = (int)slots, a.cols = (int)cols, a.place = place;
    a.dy = x, a.ld_dy = ld_x, a.out = xs, a.ld_out = ld_xs;
    return launch_rows<false, false>(a, dtype, reinterpret_cast<hipStream_t>(stream));
}

int psgd_expert_combine(void* stream, int64_t tokens, int64_t slots, int64_t cols, int dtype, const void* ys, int64_t ld_ys, const int32_t* place,
                        const float* weight, void* y, int64_t ld_y) {
    if (bad_dtype(dtype) || (tokens != 0 && (!ys || !place || !y))) return PSGD_E_INVALID_ARG;
    if (int rc = rows_shape(tokens, slots, cols)) return rc;
    if (bad_ld(ld_ys, cols) || bad_ld(ld_y, cols) || misaligned(ys) || misaligned(place) || misaligned(weight) || misaligned(y)) return PSGD_E_ALIGN;
    if (ld_ys > kMaxLd || ld_y > kMaxLd) return PSGD_E_SHAPE;
    if (tokens == 0) return PSGD_OK;
    const int64_t size = dtype == PSGD_F32 ? 4 : 2, n = tokens * slots;
    const RowArea out = {y, tokens, ld_y * size, cols * size};
    if (overlap(out, {ys, n, ld_ys * size, cols * size}) || overlap(out, {place, 1, 0, n * 4}) || overlap(out, {weight, 1, 0, n * 4})) return PSGD_E_INVALID_ARG;
    RowsDev a = {};
    a.tokens = tokens, a.n = n, a.slots = (int)slots, a.cols = (int)cols, a.place = place, a.weight = weight;
    a.in = ys, a.ld_in = ld_ys, a.out = y, a.ld_out = ld_y;
    const int pieces = row_pieces(cols, dtype), lanes = pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64, parts = (pieces + lanes - 1) / lanes;
    const dim3 blocks(row_blocks(tokens * parts, lanes));
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const bool stream_it = n * cols * size >= kRowStream;
    forget_errors();
#define PSGD_ROWS(T, LANES, STREAM) hipLaunchKernelGGL((expert_combine_kernel<T, LANES, STREAM>), blocks, dim3(kThreads), 0, st, a, parts)
#define PSGD_ROWS_LANES(T, STREAM) do { if (lanes == 16) PSGD_ROWS(T, 16, STREAM); else if (lanes == 32) PSGD_ROWS(T, 32, STREAM); else PSGD_ROWS(T, 64, STREAM); } while (0)
    if (dtype == PSGD_F32) { if (stream_it) PSGD_ROWS_LANES(float, true); else PSGD_ROWS_LANES(float, false); }
    else                   { if (stream_it) PSGD_ROWS_LANES(bf16_t, true); else PSGD_ROWS_LANES(bf16_t, false); }
#undef PSGD_ROWS
#undef PSGD_ROWS_LANES
    return hipGetLastError() == hipSuccess ? PSGD_OK : PSGD_E_HIP;
}

int psgd_expert_combine_backward(void* stream, int64_t tokens, int64_t slots, int64_t cols, int dtype, const void* dy, int64_t ld_dy, const void* ys,
                                 int64_t ld_ys, const int32_t* place, const float* weight, void* dys, int64_t ld_dys, float* dweight) {
    if (bad_dtype(dtype) || (tokens != 0 && (!dy || !place || !dys || (dweight && !ys)))) return PSGD_E_INVALID_ARG;
    if (int rc = rows_shape(tokens, slots, cols)) return rc;
    if (bad_ld(ld_dy, cols) || (ys && bad_ld(ld_ys, cols)) || bad_ld(ld_dys, cols) || misaligned(dy) || misaligned(ys) || misaligned(place) || misaligned(weight) ||
        misaligned(dys) || misaligned(dweight)) return PSGD_E_ALIGN;
    if (ld_dy > kMaxLd || (ys && ld_ys > kMaxLd) || ld_dys > kMaxLd) return PSGD_E_SHAPE;
    if (tokens == 0) return PSGD_OK;
    const int64_t size = dtype == PSGD_F32 ? 4 : 2, n = tokens * slots;
    const RowArea out = {dys, n, ld_dys * size, cols * size}, dots = {dweight, 1, 0, n * 4};
    const RowArea in[] = {{dy, tokens, ld_dy * size, cols * size}, {ys, n, ld_ys * size, cols * size}, {place, 1, 0, n * 4}, {weight, 1, 0, n * 4}};
    for (const RowArea& i : in)
        if ((overlap(out, i) && !(&i == in + 1 && same_place(out, i))) || overlap(dots, i)) return PSGD_E_INVALID_ARG;
    if (overlap(out, dots)) return PSGD_E_INVALID_ARG;
    RowsDev a = {};
    a.tokens = tokens, a.n = n, a.slots = (int)slots, a.cols = (int)cols, a.place = place, a.weight = weight;
    a.dy = dy, a.ld_dy = ld_dy, a.in = ys, a.ld_in = ld_ys, a.out = dys, a.ld_out = ld_dys, a.dweight = dweight;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    return dweight ? launch_rows<true, true>(a, dtype, st) : launch_rows<true, false>(a, dtype, st);
}

}  // extern "C"
