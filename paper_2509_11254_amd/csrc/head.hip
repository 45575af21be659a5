// Softmax cross entropy at the output head, without logits in memory, and its gradients.
//
//   l_tv = x_t . w_v,  lse_t = log sum_v exp(l_tv),  loss_t = lse_t - l_t,y(t)
//   D_tv = c_t (exp(l_tv - lse_t) - [v = y(t)]),  dX = D W,  dW = D^T X,   c_t: the token's weight, or 1 / (tokens that count)
//   (D is kept relative to the largest c_t, which the products are multiplied by at their end)
//
// Tokens whose label lies outside [0, V) do not count: their rows are left out from the start (the others are copied together,
// in order), or, of few tokens, out of all that is made of their logits, so that what they hold, NaN or not, reaches no result.
//
// The vocabulary is walked in tiles of 256 (128 for few tokens; in fp32 128 or 64).  A workgroup has the logits of a tile of tokens and one tile in its accumulators, takes the
// tile's maximum and its sum of exponentials (the label's left out) per token, and writes these two numbers; for the gradients it writes the exponentials
// relative to the tile's maximum as well, for one piece of the tokens at a time.  One more pass over a piece joins the tiles'
// numbers to lse_t and turns the exponentials into D in place, and the two products with D follow.
//
// For results in bf16 D is rounded to bf16, like the result itself: errors against 64 bits of 1.8e-3 (8192 x 4096 x 64000) to 2.2e-3 (200 x 1024 x 10007) of the gradients' norm,
// where D in 32 bits and the result rounded has 1.7e-3.  A second plane of D would take the two products' time, most of the whole, once more.
//
// The three products bound it: of 8192 x 4096 x 64000 in bf16 (9.9 to 10.1 ms) the logits take 3.2 to 3.3 ms, 1.3 PFLOP/s, D W 3.1 and D^T X 3.2; the pass that makes D reads and writes 2.1 GB in
// 0.34 ms, 6.1 TB/s, and the tokens' copy takes 0.03.  Of one token the loss alone reads W at 5 TB/s.
#include "tile_dev.h"

namespace psgd {

typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));

// what is kept of exp(l - tile's maximum): nothing, fp16 of 2^15 times it (the range of fp16 starts 2^29 below the maximum;
// 11 bits, so that D is rounded once, to bf16), or fp32 (results in fp32)
enum HeadKeep { KEEP_NONE = 0, KEEP_F16 = 1, KEEP_F32 = 2 };
constexpr float kHalfScale = 32768.f;

struct HeadDev {
    const int64_t* labels;
    const float* weight;
    float* loss;
    int tokens, d, vocab;
    // in the workspace
    int* count;          // tokens that count
    float* scale;        // the largest c_t: D is kept relative to it and its products are multiplied by it
    int* rows;           // which they are
    int* label;          // and their labels
    uint64_t* counts;    // or, where X is taken as it is, a bit for every token
    float2* stats;       // [token of the piece][tile]: maximum, sum of exponentials without the label's
    float* at_label;     // logit of the label, by token of the piece
    void* e;             // exponentials, [token of the piece][ldv]
    bf16_t* D;           // planes of D, [token of the piece][ldv]; in place of e where that is fp16
    int64_t ldv, d_plane;
    int tiles, tile_width, keep;
    int direct;          // X is taken where it is: the tokens of the piece are all tokens
};

__device__ inline bool label_counts(int64_t label, int vocab) { return label >= 0 && label < vocab; }
// label of token l of the piece from `first` on; -1: it does not count
__device__ __forceinline__ int label_of(const HeadDev& h, int first, int l) {
    if (!h.direct) return h.label[first + l];
    const int64_t y = h.labels[first + l];
    return label_counts(y, h.vocab) ? (int)y : -1;
}

// ---- tokens that count ----------------------------------------------------------------------------------------------

constexpr int kGatherThreads = 256;

// Block b has tokens [b * per, ...): where its first token goes is the number of counted ones before it, which every block finds for
// itself (8 bytes per label, from L2).  x to its planes in `xc` (row length ldc, zeros beyond d); a token that does not count gets loss 0
// and a zero row of dX.
template <class T>
__global__ __launch_bounds__(kGatherThreads) void head_gather_kernel(HeadDev h, int per, const T* x, int64_t ldx, bf16_t* xc, int64_t ldc, int planes,
                                                                     T* dx, int64_t lddx) {
    __shared__ int sum[kGatherThreads / 64];
    __shared__ int place[kGatherThreads];
    const int first = blockIdx.x * per, last = min(h.tokens, first + per);
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    int mine = 0;
#pragma unroll 4        // (loads in flight: loss of 16384 x 512 x 256 66 -> 56 us)
    for (int i = threadIdx.x; i < first; i += kGatherThreads) mine += label_counts(h.labels[i], h.vocab) ? 1 : 0;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) mine += __shfl_xor(mine, s);
    if (lane == 0) sum[wv] = mine;
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int w = 0; w < kGatherThreads / 64; ++w) before += sum[w];
    for (int t0 = first; t0 < last; t0 += kGatherThreads) {
        const int t = t0 + threadIdx.x;
        const int64_t y = t < last ? h.labels[t] : -1;
        const bool in = label_counts(y, h.vocab);
        const unsigned long long mask = __ballot(in);
        __syncthreads();
        if (lane == 0) sum[wv] = __popcll(mask);
        __syncthreads();
        int at = before + __popcll(mask & ((1ull << lane) - 1));
        for (int w = 0; w < wv; ++w) at += sum[w];
        place[threadIdx.x] = in ? at : -1;
        if (in) { h.rows[at] = t; h.label[at] = (int)y; }
        else if (t < last) h.loss[t] = 0.f;
#pragma unroll
        for (int w = 0; w < kGatherThreads / 64; ++w) before += sum[w];
        __syncthreads();
        // a wave per row
        const int pieces = (h.d + 7) / 8;
        for (int r = wv; r < kGatherThreads && t0 + r < last; r += kGatherThreads / 64) {
            const int to = place[r];
            const PSGD_GLOBAL T* src = as_global(x) + (int64_t)(t0 + r) * ldx;
            if (to < 0) {
                if (dx) {
                    constexpr int N = 16 / sizeof(T);
                    PSGD_GLOBAL T* row = as_global(dx) + (int64_t)(t0 + r) * lddx;
                    for (int c = N * lane; c < h.d; c += N * 64) {
                        if (c + N <= h.d) *reinterpret_cast<PSGD_GLOBAL uintx4*>(row + c) = uintx4{0u, 0u, 0u, 0u};
                        else for (int u = c; u < h.d; ++u) row[u] = (T)0.f;
                    }
                }
                continue;
            }
            constexpr int AHEAD = 4, WORDS = sizeof(T) == 2 ? 1 : 2;       // loads of AHEAD pieces are in flight
            for (int p0 = lane; p0 < pieces; p0 += 64 * AHEAD) {
                uintx4 w[AHEAD][WORDS];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                    for (int k = 0; k < WORDS; ++k)
                        if (p0 + 64 * i < pieces) w[i][k] = reinterpret_cast<const PSGD_GLOBAL uintx4*>(src + 8 * (p0 + 64 * i))[k];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int p = p0 + 64 * i;
                    if (p >= pieces) break;
                    bf16x8 out[kMaxPlanes];
                    if constexpr (sizeof(T) == 2) {
                        const bf16x8 b = __builtin_bit_cast(bf16x8, w[i][0]);
#pragma unroll
                        for (int u = 0; u < 8; ++u) out[0][u] = 8 * p + u < h.d ? b[u] : (bf16_t)0.f;
                    } else {
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            bf16_t q[kMaxPlanes];
                            split_planes<kMaxPlanes>(8 * p + u < h.d ? __uint_as_float(w[i][u >> 2][u & 3]) : 0.f, q);
#pragma unroll
                            for (int k = 0; k < kMaxPlanes; ++k) out[k][u] = q[k];
                        }
                    }
#pragma unroll
                    for (int k = 0; k < (sizeof(T) == 2 ? 1 : kMaxPlanes); ++k)
                        *reinterpret_cast<PSGD_GLOBAL bf16x8*>(as_global(xc) + ((int64_t)k * h.tokens + to) * ldc + 8 * p) = out[k];
                }
            }
        }
    }
    if (last == h.tokens) {
        // (1 / count is not a bf16 number, and the same error in all of D would come out in the results; relative to the largest weight, D of
        // a token that its model gives no probability is -1)
        float most = 0.f;
        if (h.weight)
            for (int i = threadIdx.x; i < h.tokens; i += kGatherThreads) most = fmaxf(most, label_counts(h.labels[i], h.vocab) ? fabsf(h.weight[i]) : 0.f);
#pragma unroll
        for (int s = 32; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor(most, s));
        __syncthreads();
        float* all = reinterpret_cast<float*>(sum);
        if (lane == 0) all[wv] = most;
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int w = 0; w < kGatherThreads / 64; ++w) most = fmaxf(most, all[w]);
            *h.count = before;
            *h.scale = !h.weight ? 1.f / (float)max(before, 1) : most > 0.f && most < __builtin_inff() ? most : 1.f;
        }
    }
}

// ---- logits of a piece: statistics per tile, exponentials --------------------------------------------------------------

template <TileShape SHAPE, int KEEP>
__global__ __launch_bounds__(kTileThreads, tile_share(SHAPE)) void head_logits_kernel(TileArgs t, HeadDev h) {
    extern __shared__ __align__(16) unsigned char smem[];
    using T = Tile<true, true, SHAPE>;
    constexpr int BL = T::BL;
    const int nl = counted(t, t.L.extent);
    const TilePlace at = tile_place(blockIdx.x, tile_grid<SHAPE>(t, nl, 0));
    if (at.split < 0) return;
    const int p0 = at.p * T::BP, l0 = at.l * BL;
    T tile;
    tile.template run<true>(t, p0, l0, nl, t.K, 0, 1, (PSGD_TLDS unsigned char*)smem);
    constexpr float kLog2e = 1.4426950408889634f;
    // the wave's maximum per row, over its columns; a tile has at least one column
    float* red = reinterpret_cast<float*>(smem);        // [WP][BL]
    __syncthreads();
#pragma unroll
    for (int j = 0; j < T::FL; ++j) {
        float m = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < T::FP; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) m = fmaxf(m, tile.acc[i][j][v]);
        m = fmaxf(m, __shfl_xor(m, 32));
        if ((threadIdx.x & 63) < 32) red[tile.wp * BL + tile.row(j)] = m;
    }
    __syncthreads();
    float most[T::FL], sum[T::FL];
#pragma unroll
    for (int j = 0; j < T::FL; ++j) {
        const int row = tile.row(j), l = l0 + row;
        float m = red[row];
#pragma unroll
        for (int w = 1; w < T::WP; ++w) m = fmaxf(m, red[w * BL + row]);
        most[j] = m;
        const float base = m == -__builtin_inff() ? 0.f : m;
        // The label's element, if it is this lane's (of eight columns next to each other a lane has the first or the last four), is left out of
        // the sum.  Few tiles have it: the search for it stands apart, and only reads.
        const int y = l < nl ? label_of(h, t.first, l) - p0 - tile.col(0, 0) : -1;
        const bool found = y >= 0 && y < 32 * T::FP && (y & 4) == 0, any = __any(found);
        float at_label = 0.f, s = 0.f;
        if (any) {
#pragma unroll
            for (int i = 0; i < T::FP; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) at_label = y == 32 * i + 8 * (v >> 2) + (v & 3) ? tile.acc[i][j][v] : at_label;
            if (found) h.at_label[l] = at_label;
        }
#pragma unroll
        for (int i = 0; i < T::FP; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float e = __builtin_amdgcn_exp2f((tile.acc[i][j][v] - base) * kLog2e);
                s += e;
                tile.acc[i][j][v] = e;
            }
        if (any) {
            s = 0.f;
#pragma unroll
            for (int i = 0; i < T::FP; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) s += y == 32 * i + 8 * (v >> 2) + (v & 3) ? 0.f : tile.acc[i][j][v];
        }
        sum[j] = s + __shfl_xor(s, 32);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < T::FL; ++j)
        if ((threadIdx.x & 63) < 32) red[tile.wp * BL + tile.row(j)] = sum[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < T::FL; ++j) {
        const int row = tile.row(j), l = l0 + row;
        if (tile.wp == 0 && (threadIdx.x & 63) < 32 && l < nl) {
            float s = red[row];
#pragma unroll
            for (int w = 1; w < T::WP; ++w) s += red[w * BL + row];
            h.stats[(int64_t)l * h.tiles + at.p] = make_float2(most[j], s);
        }
    }
    if constexpr (KEEP == KEEP_F16) {
        tile.template for_rows<8>((PSGD_TLDS unsigned char*)smem, [&](int row, int col, const float (&v)[8]) {
            halfx8 o;
#pragma unroll
            for (int u = 0; u < 8; ++u) o[u] = (_Float16)(v[u] * kHalfScale);
            if (l0 + row < nl && p0 + col < h.ldv) *reinterpret_cast<PSGD_GLOBAL halfx8*>(as_global((_Float16*)h.e) + (l0 + row) * h.ldv + p0 + col) = o;
        });
    } else if constexpr (KEEP == KEEP_F32) {
        tile.template for_rows<4>((PSGD_TLDS unsigned char*)smem, [&](int row, int col, const float (&v)[4]) {
            if (l0 + row < nl && p0 + col < h.ldv)
                *reinterpret_cast<PSGD_GLOBAL floatx4*>(as_global((float*)h.e) + (l0 + row) * h.ldv + p0 + col) = floatx4{v[0], v[1], v[2], v[3]};
        });
    }
}

// ---- the row's sum, the loss, and D ------------------------------------------------------------------------------------

// Largest logit of row l and the sum of exp(logit - it) over all columns but the label's, by all threads of the block
struct RowSum { float most, others; };
__device__ __forceinline__ RowSum row_sum(const HeadDev& h, int l, float* shared) {
    const float2* st = h.stats + (int64_t)l * h.tiles;
    float m = -__builtin_inff(), s = 0.f;
    auto join = [&](float mo, float so) {
        const float n = fmaxf(m, mo);
        if (n != -__builtin_inff()) s = s * expf(m - n) + so * expf(mo - n);
        else s += so;
        m = n;
    };
    for (int i = threadIdx.x; i < h.tiles; i += kThreads) join(st[i].x, st[i].y);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const float mo = __shfl_xor(m, d), so = __shfl_xor(s, d);
        join(mo, so);
    }
    if ((threadIdx.x & 63) == 0) { shared[threadIdx.x >> 6] = m; shared[4 + (threadIdx.x >> 6)] = s; }
    __syncthreads();
    m = shared[0], s = shared[4];
#pragma unroll
    for (int w = 1; w < 4; ++w) join(shared[w], shared[4 + w]);
    return {m, s};
}

// Where no launch before has looked at the labels: the largest weight of a token that counts, or one over their number (see head_gather_kernel).
// write: their bits as well
__device__ __forceinline__ float direct_scale(const HeadDev& h, float* shared, bool write) {
    float x = 0.f;
    for (int i0 = 0; i0 < h.tokens; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        const bool in = i < h.tokens && label_counts(h.labels[i], h.vocab);
        if (in) x = h.weight ? fmaxf(x, fabsf(h.weight[i])) : x + 1.f;
        const uint64_t bits = __ballot(in);
        if (write && (threadIdx.x & 63) == 0 && i < h.tokens) h.counts[i >> 6] = bits;
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const float o = __shfl_xor(x, d);
        x = h.weight ? fmaxf(x, o) : x + o;
    }
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    x = shared[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) x = h.weight ? fmaxf(x, shared[w]) : x + shared[w];
    __syncthreads();
    if (!h.weight) return 1.f / fmaxf(x, 1.f);
    return x > 0.f && x < __builtin_inff() ? x : 1.f;
}

// block: one token's row, blockIdx.y its part of the vocabulary; without gradients one part and no D
template <int KEEP, int PL>
__global__ __launch_bounds__(kThreads) void head_rows_kernel(HeadDev h, int first, int most_rows, int span) {
    __shared__ float shared[8];
    const int l = blockIdx.x;
    if (l >= (h.direct ? most_rows : min(most_rows, *h.count - first))) return;
    const int token = h.direct ? first + l : h.rows[first + l], y = label_of(h, first, l);
    const int end = (int)min((int64_t)(blockIdx.y + 1) * span, h.ldv);
    float scale = 1.f;
    if (KEEP != KEEP_NONE && h.direct && (h.weight || (l == 0 && blockIdx.y == 0))) {
        const bool write = l == 0 && blockIdx.y == 0;
        scale = direct_scale(h, shared, write);
        if (write && threadIdx.x == 0) *h.scale = scale;
    }
    if (y < 0) {
        if (blockIdx.y == 0 && threadIdx.x == 0) h.loss[token] = 0.f;
        if constexpr (KEEP != KEEP_NONE)
            for (int v = blockIdx.y * span + 8 * threadIdx.x; v < end; v += 8 * kThreads)
#pragma unroll
                for (int k = 0; k < PL; ++k) *reinterpret_cast<PSGD_GLOBAL uintx4*>(as_global(h.D) + k * h.d_plane + l * h.ldv + v) = uintx4{0u, 0u, 0u, 0u};
        return;
    }
    // exponentials are read ahead (for the last time: the hint takes 8192 x 4096 x 64000 from 10.0 to 9.93 ms)
    uintx4 e[KEEP == KEEP_F32 ? 2 : 1];
    auto fetch = [&](int v) {
        if constexpr (KEEP == KEEP_F16) {
            e[0] = __builtin_nontemporal_load(reinterpret_cast<const PSGD_GLOBAL uintx4*>(as_global((_Float16*)h.e) + l * h.ldv + v));
        } else if constexpr (KEEP == KEEP_F32) {
            const PSGD_GLOBAL uintx4* p = reinterpret_cast<const PSGD_GLOBAL uintx4*>(as_global((float*)h.e) + l * h.ldv + v);
            e[0] = __builtin_nontemporal_load(p), e[1] = __builtin_nontemporal_load(p + 1);
        }
    };
    const int start = blockIdx.y * span + 8 * threadIdx.x;
    if (KEEP != KEEP_NONE && start < end) fetch(start);
    const RowSum r = row_sum(h, l, shared);
    const float at_label = h.at_label[l], e_label = expf(at_label - r.most), total = r.others + e_label;
    // log(1 + others / label's) keeps the loss of a token that is all but certain, which the difference of two logits does not
    if (blockIdx.y == 0 && threadIdx.x == 0)
        h.loss[token] = r.others < e_label ? log1pf(r.others / e_label) : r.most - at_label + logf(total);
    if constexpr (KEEP == KEEP_NONE) return;
    const float c = (h.weight ? h.weight[token] / (h.direct ? scale : *h.scale) : 1.f) / total;
    const float d_label = -r.others * c;        // (p - 1 as the sum of the other probabilities)
    for (int v = start; v < end; v += 8 * kThreads) {
        const float most = h.stats[(int64_t)l * h.tiles + v / h.tile_width].x;
        const float f = expf(most - r.most) * c * (KEEP == KEEP_F16 ? 1.f / kHalfScale : 1.f);
        float x[8];
        if constexpr (KEEP == KEEP_F16) {
            const halfx8 q = __builtin_bit_cast(halfx8, e[0]);
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = (float)q[u] * f;
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = __uint_as_float(e[KEEP == KEEP_F32 ? u >> 2 : 0][u & 3]) * f;
        }
        if (v + 8 * kThreads < end) fetch(v + 8 * kThreads);
        bf16x8 out[PL];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            bf16_t q[PL];
            split_planes<PL>(v + u == y ? d_label : x[u], q);
#pragma unroll
            for (int k = 0; k < PL; ++k) out[k][u] = q[k];
        }
#pragma unroll
        for (int k = 0; k < PL; ++k) *reinterpret_cast<PSGD_GLOBAL bf16x8*>(as_global(h.D) + k * h.d_plane + l * h.ldv + v) = out[k];
    }
}

// fp32 sums of all pieces to bf16
__global__ __launch_bounds__(kThreads) void head_round_kernel(const float* sum, int64_t rows, int cols, int64_t lds, bf16_t* out, int64_t ld, int accumulate) {
    const int quads = (cols + 3) / 4;
    const int64_t all = rows * quads;
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < all; e += (int64_t)gridDim.x * kThreads) {
        const int64_t r = e / quads;
        const int c = 4 * (int)(e - r * quads);
        const floatx4 s = *reinterpret_cast<const PSGD_GLOBAL floatx4*>(as_global(sum) + r * lds + c);
        PSGD_GLOBAL bf16_t* p = as_global(out) + r * ld + c;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (c + u < cols) p[u] = (bf16_t)(accumulate ? s[u] + (float)p[u] : s[u]);
    }
}

// ---- host --------------------------------------------------------------------------------------------------------------

// (Loss and gradients, tokens x d x vocab, in us: 1 x 512 x 4400 35.5 -> 26.5, 512 x 512 x 4400 56.5 -> 47, 500 x 1024 x 10008 87.7 -> 81.  The products take all tokens then:
// not where there may be many that do not count.)
constexpr int64_t kDirectTokens = 512;
constexpr size_t kPieceBytes = (size_t)1 << 30;     // what is kept of one piece of the tokens: exponentials and D, or statistics alone
// A launch has fewer than 2^32 threads: 256 to a token of a piece, and 256 to a tile of its logits, at least 64 x 64 (half of either, for what borders add).
constexpr int64_t kMaxPiece = (int64_t)1 << 23, kMaxPieceLogits = (int64_t)1 << 35;

struct HeadPlan {
    size_t bytes = 0;
    size_t count, scale, rows, label, counts, xc, wc, stats, at_label, e, D, part, dw_part, sum;
    int64_t ldc, ldv;
    int piece, pieces, tiles, x_planes, d_planes, keep;
    TilePlan logits, dx, dw;
    unsigned dw_pairs;
    int n_dw_pairs;
    bool copy_w, direct, pair;
};

static HeadPlan head_plan(const psgd_head_desc& s, bool gradients) {
    HeadPlan p = {};
    const bool f32 = s.dtype == PSGD_F32;
    p.ldc = up8(s.d);
    p.ldv = up8(s.vocab);
    p.x_planes = f32 ? 3 : 1;
    p.copy_w = !f32 && s.d % 8 != 0;        // (fp32 W is split into planes by the products)
    p.keep = !gradients ? KEEP_NONE : f32 || s.grad_dtype == PSGD_F32 ? KEEP_F32 : KEEP_F16;
    p.d_planes = p.keep == KEEP_F32 ? 3 : 1;
    // (Two planes of D for dW in fp32 from bf16 X: 2124 us in place of 2830 for 4096 x 2048 x 32000, 81 in place of 88 for 1391 x 384 x 4477, and an error of
    // dW of 1.5e-6 in place of 3e-7, where products in fp32 have 7e-7.)
    p.dw_pairs = !f32 && p.d_planes == 3 ? kPairsL3 : kPairs1, p.n_dw_pairs = !f32 ? p.d_planes : 1;
    // tokens per piece (statistics: 8 bytes for each tile of 128 words; tiles of 64 are not taken for so many tokens, but where all words are in one)
    const int64_t tokens = std::max<int64_t>(1, s.tokens);
    const size_t row = !gradients ? s.vocab / 128 * sizeof(float2) + 64 : (size_t)p.ldv * (p.keep == KEEP_F16 ? 2 : 4 + 2 * p.d_planes);
    const int64_t launch = std::min(kMaxPiece, std::max<int64_t>(1, kMaxPieceLogits / s.vocab));
    const int64_t most = std::min(std::min(tokens, launch), s.piece_tokens > 0 ? s.piece_tokens : std::max<int64_t>(256, (int64_t)(kPieceBytes / row) / 256 * 256));
    p.pieces = (int)((tokens + most - 1) / most);
    p.piece = (int)((tokens + p.pieces - 1) / p.pieces);
    if (p.pieces > 1 && s.piece_tokens <= 0) p.piece = (p.piece + 255) / 256 * 256;
    p.pieces = (int)((tokens + p.piece - 1) / p.piece);
    // Few tokens: X is taken where it is, and those that do not count are sorted out by their labels -- losses of one tile of rows, where they cost
    // nothing; gradients of up to kDirectTokens, whose launches are all there is to save.
    p.direct = !f32 && !p.copy_w && p.pieces == 1 && s.tokens > 0 && s.tokens <= (gradients ? kDirectTokens : tile_l(TILE_THIN));
    const int64_t step = f32 ? tile_k(TILE_SPLIT) : kTileK, d_chunks = (s.d + step - 1) / step;
    p.logits = f32 ? split_plan(s.vocab, p.piece, d_chunks, false) : tile_plan(s.vocab, p.piece, d_chunks, false, 0);
    p.tiles = (int)((s.vocab + tile_p(p.logits.shape) - 1) / tile_p(p.logits.shape));
    auto take = [&](size_t bytes) { const size_t at = p.bytes; p.bytes += up256(bytes); return at; };
    p.count = take(4);
    p.scale = take(4);
    p.rows = take((size_t)tokens * 4);
    p.label = take((size_t)tokens * 4);
    p.counts = take((size_t)(tokens + 63) / 64 * 8);
    p.xc = p.direct && !gradients ? 0 : take((size_t)tokens * p.ldc * 2 * p.x_planes);      // (direct: where dX takes X's place)
    p.wc = p.copy_w ? take((size_t)s.vocab * p.ldc * 2) : 0;
    p.stats = take((size_t)p.piece * p.tiles * sizeof(float2));
    p.at_label = take((size_t)p.piece * 4);
    if (gradients) {
        const size_t elems = (size_t)p.piece * p.ldv;
        p.e = take(elems * (p.keep == KEEP_F16 ? 2 : 4));
        p.D = p.keep == KEEP_F16 ? p.e : take(elems * 2 * p.d_planes);
        const int64_t dx_chunks = (s.vocab + step - 1) / step, dw_chunks = (p.piece + step - 1) / step * p.n_dw_pairs;
        p.dx = f32 ? split_plan(s.d, p.piece, dx_chunks, true) : tile_plan(s.d, p.piece, dx_chunks, true, 0);
        p.dw = f32 ? split_plan(s.d, s.vocab, dw_chunks, true) : tile_plan(s.d, s.vocab, dw_chunks, true, 0, p.direct);
        if (p.pieces == 1 && s.tokens > 0 && p.dw.shape == TILE_MANY) {
            const TilePlan many = tile_plan(s.d, p.piece, dx_chunks, true, 0, true);
            const int64_t wide = (s.d + 127) / 128;
            p.pair = pair_pays({many, s.d, p.piece, wide * ((p.piece + 127) / 128), dx_chunks}, {p.dw, s.d, s.vocab, wide * ((s.vocab + 127) / 128), dw_chunks}, p.dx);
            if (p.pair) p.dx = many;
        }
        p.part = take(tile_part_bytes(s.d, p.piece, p.dx));
        p.dw_part = p.pair ? take(tile_part_bytes(s.d, s.vocab, p.dw)) : p.part;
        if (!p.pair && tile_part_bytes(s.d, s.vocab, p.dw) > tile_part_bytes(s.d, p.piece, p.dx)) p.bytes = p.part + tile_part_bytes(s.d, s.vocab, p.dw);
        p.sum = p.pieces > 1 && s.grad_dtype == PSGD_BF16 ? take((size_t)s.vocab * p.ldc * 4) : 0;
    }
    return p;
}

static int head_shape(const psgd_head_desc* s) {
    if (!s || bad_dtype(s->dtype) || bad_dtype(s->grad_dtype) || s->piece_tokens < 0) return PSGD_E_INVALID_ARG;
    if (s->tokens < 0 || s->d < 1 || s->vocab < 1 || s->tokens > kMaxExtent || s->vocab > kMaxExtent || up8(s->d) > kMaxLd || up8(s->vocab) > kMaxLd) return PSGD_E_SHAPE;
    return PSGD_OK;
}

template <TileShape SHAPE, int KEEP>
static hipError_t launch_logits_as(const TileArgs& t, const HeadDev& h, hipStream_t st) {
    const int64_t blocks = h.tiles * (int64_t)((t.L.extent + tile_l(SHAPE) - 1) / tile_l(SHAPE));
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    auto kfn = head_logits_kernel<SHAPE, KEEP>;
    constexpr int lds = Tile<true, true, SHAPE>::LDS_BYTES;
    if (lds > 48 * 1024) {
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kfn), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kfn, dim3((unsigned)blocks), dim3(kTileThreads), lds, st, t, h);
    return hipGetLastError();
}
template <TileShape SHAPE>
static hipError_t launch_logits_shape(const TileArgs& t, const HeadDev& h, hipStream_t st) {
    if (h.keep == KEEP_NONE) return launch_logits_as<SHAPE, KEEP_NONE>(t, h, st);
    if (h.keep == KEEP_F16) return launch_logits_as<SHAPE, KEEP_F16>(t, h, st);
    return launch_logits_as<SHAPE, KEEP_F32>(t, h, st);
}
static hipError_t launch_logits(const TileArgs& t, const HeadDev& h, TileShape shape, hipStream_t st) {
    if (shape == TILE_256) return launch_logits_shape<TILE_256>(t, h, st);
    if (shape == TILE_128) return launch_logits_shape<TILE_128>(t, h, st);
    if (shape == TILE_MANY) return launch_logits_shape<TILE_MANY>(t, h, st);
    if (shape == TILE_SPLIT) return h.keep == KEEP_NONE ? launch_logits_as<TILE_SPLIT, KEEP_NONE>(t, h, st) : launch_logits_as<TILE_SPLIT, KEEP_F32>(t, h, st);
    if (shape == TILE_SPLIT_THIN) return h.keep == KEEP_NONE ? launch_logits_as<TILE_SPLIT_THIN, KEEP_NONE>(t, h, st) : launch_logits_as<TILE_SPLIT_THIN, KEEP_F32>(t, h, st);
    return launch_logits_shape<TILE_THIN>(t, h, st);
}

static hipError_t launch_rows(const HeadDev& h, int first, int rows, hipStream_t st) {
    if (h.keep == KEEP_NONE) {
        hipLaunchKernelGGL((head_rows_kernel<KEEP_NONE, 1>), dim3(rows), dim3(kThreads), 0, st, h, first, rows, 0);
        return hipGetLastError();
    }
    // parts of the vocabulary, so that a few rows fill the card as well
    int64_t parts = std::max<int64_t>(1, std::min<int64_t>((h.ldv + 8 * kThreads - 1) / (8 * kThreads), 2048 / std::max(1, rows)));
    const int span = (int)(((h.ldv + parts - 1) / parts + 7) / 8 * 8);
    parts = (h.ldv + span - 1) / span;
    const dim3 grid(rows, (unsigned)parts);
    if (h.keep == KEEP_F16) hipLaunchKernelGGL((head_rows_kernel<KEEP_F16, 1>), grid, dim3(kThreads), 0, st, h, first, rows, span);
    else hipLaunchKernelGGL((head_rows_kernel<KEEP_F32, 3>), grid, dim3(kThreads), 0, st, h, first, rows, span);
    return hipGetLastError();
}

// rows of `width` bytes, `stride` bytes apart
struct HeadArea { const void* ptr; int64_t rows, stride, width; };
// (columns of one buffer beside each other do not overlap; areas with different strides do where their ranges do)
static bool overlap(HeadArea a, HeadArea b) {
    if (a.rows == 0 || b.rows == 0 || a.width == 0 || b.width == 0 || !a.ptr || !b.ptr) return false;
    const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(b.ptr) - reinterpret_cast<uintptr_t>(a.ptr));
    if (apart >= (a.rows - 1) * a.stride + a.width || -apart >= (b.rows - 1) * b.stride + b.width) return false;
    if (a.rows == 1) a.stride = b.stride;
    if (b.rows == 1) b.stride = a.stride;
    if (a.stride != b.stride || a.width > a.stride || b.width > b.stride) return true;
    // b's first row begins in row `down` of a, at column `right`
    const int64_t down = apart >= 0 ? apart / a.stride : -((-apart + a.stride - 1) / a.stride), right = apart - down * a.stride;
    auto rows_meet = [&](int64_t d) { return d < a.rows && d + b.rows > 0; };
    return (right < a.width && rows_meet(down)) || (right + b.width > a.stride && rows_meet(down + 1));
}

static int head_run(const psgd_head_desc* s, bool gradients, void* workspace, void* stream, const void* x, const void* w, const int64_t* labels,
                    const float* weight, float* loss, void* dx, void* dw, int accumulate) {
    if (int rc = head_shape(s)) return rc;
    if (!workspace || !w || (gradients && !dw) || (s->tokens != 0 && (!x || !labels || !loss || (gradients && !dx)))) return PSGD_E_INVALID_ARG;
    const int64_t ldx = s->ldx ? s->ldx : s->d, ldw = s->ldw ? s->ldw : s->d, lddx = s->lddx ? s->lddx : s->d, lddw = s->lddw ? s->lddw : s->d;
    if (ldx > kMaxLd || ldw > kMaxLd || lddx > kMaxLd || lddw > kMaxLd) return PSGD_E_SHAPE;
    if (bad_ld(ldx, s->d) || bad_ld(ldw, s->d) || misaligned(x) || misaligned(w) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PSGD_E_ALIGN;
    if (gradients && (bad_ld(lddx, s->d) || bad_ld(lddw, s->d) || misaligned(dx) || misaligned(dw))) return PSGD_E_ALIGN;
    const int64_t size = s->dtype == PSGD_F32 ? 4 : 2, g_size = s->grad_dtype == PSGD_F32 ? 4 : 2;
    const bool in_place = gradients && x && x == dx && (ldx == lddx || s->tokens == 1);
    const HeadArea in[] = {{x, s->tokens, ldx * size, s->d * size}, {w, s->vocab, ldw * size, s->d * size}, {labels, 1, 0, s->tokens * 8},
                           {weight, 1, 0, s->tokens * 4}};
    const HeadArea out[] = {{dx, s->tokens, lddx * size, s->d * size}, {dw, s->vocab, lddw * g_size, s->d * g_size}, {loss, 1, 0, s->tokens * 4}};
    for (const HeadArea& o : out)
        for (const HeadArea& i : in)
            if (overlap(o, i) && !(in_place && &o == out && &i == in)) return PSGD_E_INVALID_ARG;
    if (overlap(out[0], out[1]) || overlap(out[0], out[2]) || overlap(out[1], out[2])) return PSGD_E_INVALID_ARG;
    const HeadPlan p = head_plan(*s, gradients);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    forget_errors();
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    const bool f32 = s->dtype == PSGD_F32;

    HeadDev h = {};
    h.labels = labels, h.weight = weight, h.loss = loss;
    h.tokens = (int)s->tokens, h.d = (int)s->d, h.vocab = (int)s->vocab;
    h.count = reinterpret_cast<int*>(ws + p.count);
    h.scale = reinterpret_cast<float*>(ws + p.scale);
    h.rows = reinterpret_cast<int*>(ws + p.rows);
    h.label = reinterpret_cast<int*>(ws + p.label);
    h.counts = reinterpret_cast<uint64_t*>(ws + p.counts);
    h.stats = reinterpret_cast<float2*>(ws + p.stats);
    h.at_label = reinterpret_cast<float*>(ws + p.at_label);
    h.e = ws + p.e;
    h.D = reinterpret_cast<bf16_t*>(ws + p.D);
    h.ldv = p.ldv, h.d_plane = (int64_t)p.piece * p.ldv;
    h.tiles = p.tiles, h.tile_width = tile_p(p.logits.shape), h.keep = p.keep;
    bf16_t* xc = reinterpret_cast<bf16_t*>(ws + p.xc);
    const bf16_t* wc = static_cast<const bf16_t*>(w);       // (fp32: cast, the products know)
    int64_t ldwc = ldw;

    h.direct = p.direct;
    // at most 1024 blocks, each of which reads the labels before its own, and a row per wave at least (2048 x 4096 x 512, loss: 48 us with four, 45 with one)
    const int per = std::max(4, (int)((s->tokens + 1023) / 1024));
    const dim3 blocks((unsigned)std::max<int64_t>(1, (s->tokens + per - 1) / per));
    if (h.direct) {}
    else if (f32) hipLaunchKernelGGL(head_gather_kernel<float>, blocks, dim3(kGatherThreads), 0, st, h, per, (const float*)x, ldx, xc, p.ldc, p.x_planes, (float*)dx, lddx);
    else hipLaunchKernelGGL(head_gather_kernel<bf16_t>, blocks, dim3(kGatherThreads), 0, st, h, per, (const bf16_t*)x, ldx, xc, p.ldc, p.x_planes, (bf16_t*)dx, lddx);
    if (hipGetLastError() != hipSuccess) return PSGD_E_HIP;
    if (p.copy_w) {
        bf16_t* to = reinterpret_cast<bf16_t*>(ws + p.wc);
        if (launch_planes(w, PSGD_BF16, s->vocab, s->d, ldw, to, 1, st) != hipSuccess) return PSGD_E_HIP;
        wc = to, ldwc = p.ldc;
    }
    if (p.direct && in_place) {        // dW takes X after dX, or beside it
        if (launch_planes(x, PSGD_BF16, s->tokens, s->d, ldx, xc, 1, st) != hipSuccess) return PSGD_E_HIP;
        x = xc;
    }
    const int64_t ld_direct = in_place ? p.ldc : ldx;
    for (int piece = 0; piece < p.pieces; ++piece) {
        const int first = piece * p.piece, rows = (int)std::min<int64_t>(p.piece, s->tokens - first);
        const TileOperand tokens = h.direct ? TileOperand{static_cast<const bf16_t*>(x) + (int64_t)first * ld_direct, ld_direct, 0, rows}
                                            : TileOperand{xc + (int64_t)first * p.ldc, p.ldc, s->tokens * p.ldc, rows};
        TileArgs t = {};
        t.count = h.direct ? nullptr : h.count, t.first = first, t.n_split = 1;
        if (rows > 0) {
            t.P = {wc, ldwc, 0, (int)s->vocab};
            t.L = tokens;
            t.K = (int)(f32 ? s->d : p.ldc);
            t.pairs = kPairs1, t.n_pairs = 1;
            if (launch_logits(t, h, p.logits.shape, st) != hipSuccess || launch_rows(h, first, rows, st) != hipSuccess) return PSGD_E_HIP;
        }
        if (!gradients) continue;
        TileArgs tx = t, tw = t;
        TileOut ox = {}, ow = {};
        ox.scale = ow.scale = h.scale;
        tx.P = {wc, ldwc, 0, (int)s->d};
        tx.L = {h.D, p.ldv, h.d_plane, rows};
        tx.K = (int)s->vocab;
        tx.n_split = p.dx.n_split;
        ox.part = reinterpret_cast<float*>(ws + p.part);
        ox.ptr = dx, ox.ld = lddx, ox.dtype = s->dtype;
        tw.P = tokens;
        tw.P.extent = (int)s->d;
        tw.L = {h.D, p.ldv, h.d_plane, (int)s->vocab};
        tw.K = rows, tw.count_is_k = 1;
        tw.pairs = p.dw_pairs, tw.n_pairs = p.n_dw_pairs, tw.n_split = p.dw.n_split;
        ow.part = reinterpret_cast<float*>(ws + p.dw_part);
        if (h.direct) ox.tokens = tw.steps = h.counts;
        else ox.rows = h.rows;
        if (p.sum) { ow.ptr = ws + p.sum; ow.ld = p.ldc; ow.dtype = PSGD_F32; ow.accumulate = piece > 0; }
        else { ow.ptr = dw; ow.ld = lddw; ow.dtype = s->grad_dtype; ow.accumulate = piece > 0 || accumulate; }
        ow.skip_empty = ow.accumulate;
        if (p.pair) {
            if (launch_pair(tx, ox, tw, ow, st) != hipSuccess) return PSGD_E_HIP;
        } else {
            if (rows > 0 && launch_product(true, p.dx.shape, tx, ox, st) != hipSuccess) return PSGD_E_HIP;
            if (launch_product(false, p.dw.shape, tw, ow, st) != hipSuccess) return PSGD_E_HIP;
        }
    }
    if (gradients && p.sum) {
        hipLaunchKernelGGL(head_round_kernel, dim3(2048), dim3(kThreads), 0, st, (const float*)(ws + p.sum), s->vocab, (int)s->d, p.ldc, (bf16_t*)dw, lddw, accumulate);
        if (hipGetLastError() != hipSuccess) return PSGD_E_HIP;
    }
    return PSGD_OK;
}

}  // namespace psgd

using namespace psgd;

extern "C" {

size_t psgd_head_workspace_bytes(const psgd_head_desc* desc, int gradients) {
    return head_shape(desc) ? 0 : head_plan(*desc, gradients != 0).bytes;
}

int psgd_head_loss(const psgd_head_desc* desc, void* workspace, void* stream, const void* x, const void* w, const int64_t* labels, float* loss) {
    return head_run(desc, false, workspace, stream, x, w, labels, nullptr, loss, nullptr, nullptr, 0);
}

int psgd_head_loss_grad(const psgd_head_desc* desc, void* workspace, void* stream, const void* x, const void* w, const int64_t* labels,
                        const float* weight, float* loss, void* dx, void* dw, int accumulate) {
    return head_run(desc, true, workspace, stream, x, w, labels, weight, loss, dx, dw, accumulate);
}

}  // extern "C"
