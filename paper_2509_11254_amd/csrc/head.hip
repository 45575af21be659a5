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

// A teacher's entries in the place of labels.  Per token of the piece a list of the words that its entries name, ascending, each once.  The logits kernel
// looks for them by 8 or 32 tokens (a group) and a range of words (a bucket: a tile's, or several tiles' where there are more than kBuckets): there they lie together, in no order.
struct HeadTop {
    const int64_t* index;
    const void* teacher;
    int dtype, top;
    int64_t ld;
    // in the workspace
    int *word, *place;   // [token of the piece][top]: the word, and its place among its group's
    float *q, *log_q;    // the teacher's probability of the word
    unsigned* flat;      // [group][its tokens * top]: word * 32 + token of the group
    float* logit;        // and its logit
    int* start;          // [group][buckets + 1]: the first place of each bucket
    int* words;          // [token of the piece]: how many
    int buckets, shift;  // word >> shift: its bucket
    int group;           // tokens of a group
};

struct HeadDev {
    const int64_t* labels;      // (of a teacher: 0 where there is an entry, -1 where there is none)
    HeadTop top;
    float inv_t;         // one over the temperature, which logits are multiplied by
    const float* weight;
    float* loss;
    int tokens, d, vocab;
    // in the workspace
    int* count;          // tokens that count
    float* scale;        // the largest c_t (in the second word): D is kept relative to it, and its products are multiplied by it over the temperature (the first)
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

__host__ __device__ constexpr int up4(int x) { return (x + 3) & ~3; }
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
            const float scale = !h.weight ? 1.f / (float)max(before, 1) : most > 0.f && most < __builtin_inff() ? most : 1.f;
            h.scale[0] = scale * h.inv_t, h.scale[1] = scale;
        }
    }
}

// ---- a teacher's entries -------------------------------------------------------------------------------------------------

constexpr int kMaxTop = 1024;

// what the wavefront's lanes have put into LDS, its other lanes find there
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ float teacher_logit(const HeadTop& k, int64_t i) {
    return k.dtype == PSGD_F32 ? as_global(static_cast<const float*>(k.teacher))[i] : (float)as_global(static_cast<const bf16_t*>(k.teacher))[i];
}
// whether an entry counts: a word of the vocabulary, of some probability
__device__ __forceinline__ bool entry_counts(const HeadTop& k, int64_t i, int vocab) {
    return label_counts(as_global(k.index)[i], vocab) && teacher_logit(k, i) != -__builtin_inff();
}

// which tokens have entries: a wavefront each
__global__ __launch_bounds__(kThreads) void head_top_count_kernel(HeadTop k, int tokens, int vocab, int64_t* labels) {
    const int lane = threadIdx.x & 63;
    for (int t = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); t < tokens; t += gridDim.x * (kThreads / 64)) {
        bool any = false;
        for (int i = lane; i < k.top; i += 64) any |= entry_counts(k, t * k.ld + i, vocab);
        any = __any(any);
        if (lane == 0) as_global(labels)[t] = any ? 0 : -1;
    }
}

// a and b of a sorting network
__device__ __forceinline__ void in_order(unsigned& a, unsigned& b, bool up) {
    const unsigned low = min(a, b), high = max(a, b);
    a = up ? low : high, b = up ? high : low;
}
// U keys of each lane, key lane + 64 u of them all, in order: Batcher's bitonic network, whose steps of 64 and more stay in a lane
template <int U>
__device__ __forceinline__ void sort_keys(unsigned (&key)[U], int lane) {
#pragma unroll
    for (int len = 2; len <= 64 * U; len <<= 1)
#pragma unroll
        for (int step = len >> 1; step > 0; step >>= 1) {
            if (step >= 64) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if ((u & (step / 64)) == 0) in_order(key[u], key[u | (step / 64)], ((64 * u) & len) == 0);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const unsigned other = (unsigned)__shfl_xor((int)key[u], step);
                    const bool up = ((lane + 64 * u) & len) == 0, first = (lane & step) == 0;
                    key[u] = up == first ? min(key[u], other) : max(key[u], other);
                }
            }
        }
}

// The lists of the piece's tokens, a group to a workgroup, whose wavefronts take a token after another, with up to U entries to a lane.  Entries are put in
// order (of word, then of place among the token's entries): up to 64 by the number of smaller ones, more by a sorting network (640 tokens, us of the launch, with 128,
// 256 and 1024 entries 9.5, 18.9 and 151 by numbers of smaller ones, 8.2, 13.2 and 44.9 so).  Those of one word become one with the sum of their probabilities.  Then the
// group's words are counted by bucket, and put there.
// write_labels: the tokens have not been looked at before (labels).
// Few tokens: groups of 8, so that more compute units have one (200 tokens of 100 entries: 16.4 us with groups of 32, 8.0 so).
constexpr int group_tokens(TileShape s) { return s == TILE_256 ? 32 : 8; }
constexpr int kBuckets = 4096;
template <int U, int GROUP> constexpr int kListWaves = U > 8 || GROUP < 16 ? 8 : 16;        // (12 bytes of LDS for each entry of a wavefront's token)
template <int U, int GROUP>
__global__ __launch_bounds__((64 * kListWaves<U, GROUP>)) void head_top_lists_kernel(HeadDev h, int first, int rows, int64_t* write_labels) {
    constexpr int SIZE = 64 * U, WAVES = kListWaves<U, GROUP>, THREADS = 64 * WAVES, EACH = GROUP / WAVES, AHEAD = U > 4 ? 1 : EACH;      // tokens whose loads are sent off first
    extern __shared__ __align__(16) unsigned char smem[];
    const HeadTop& k = h.top;
    const int threads = THREADS, waves = WAVES, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    int* count = reinterpret_cast<int*>(smem);                                              // [buckets]
    unsigned* key = reinterpret_cast<unsigned*>(smem) + up4(k.buckets) + 3 * SIZE * wv;    // [SIZE] of this wavefront: word, place among the entries
    float* value = reinterpret_cast<float*>(key);                                           // or its logits, as they came
    unsigned* sorted = key + SIZE;                                                          // the same in their order
    float* z = reinterpret_cast<float*>(key + 2 * SIZE);                                    // logits less the largest, over the temperature
    __shared__ int sums[16], listed[GROUP];
    const int group0 = blockIdx.x * GROUP, end = min(rows, h.direct ? rows : *h.count - first);
    if (group0 >= end) return;
    for (int b = threadIdx.x; b < k.buckets; b += threads) count[b] = 0;
    __syncthreads();
#pragma unroll 1
    for (int r0 = 0; r0 < EACH; r0 += AHEAD) {
        int64_t token[AHEAD], y[AHEAD][U];
        float v[AHEAD][U];
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) {
            const int l = group0 + wv + (r0 + r) * WAVES;
            token[r] = l >= end ? -1 : h.direct ? l : h.rows[first + l];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = lane + 64 * u;
                const bool in = token[r] >= 0 && i < k.top;
                y[r][u] = in ? as_global(k.index)[token[r] * k.ld + i] : -1;
                v[r][u] = in ? teacher_logit(k, token[r] * k.ld + i) : 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) {
            if (token[r] < 0) continue;
            const int l = group0 + wv + (r0 + r) * WAVES;
            const int64_t list = (int64_t)l * k.top;
            float most = -__builtin_inff();
            int n = 0;
            unsigned mine[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool in = label_counts(y[r][u], h.vocab) && v[r][u] != -__builtin_inff();
                mine[u] = in ? (unsigned)y[r][u] << 10 | (unsigned)(lane + 64 * u) : ~0u;
                most = in ? fmaxf(most, v[r][u]) : most;
                n += __popcll(__ballot(in));
                if constexpr (U == 1) key[lane] = mine[u];
                else value[lane + 64 * u] = v[r][u];
            }
            most = lanes_max<64>(most);
            wave_sync();
            // (what does not count is behind all that does)
            if constexpr (U == 1) {
                int rank = 0;
#pragma unroll 2
                for (int j = 0; j < k.top; j += 4) {
                    const uintx4 other = *reinterpret_cast<const uintx4*>(key + j);
#pragma unroll
                    for (int o = 0; o < 4; ++o) rank += other[o] < mine[0] ? 1 : 0;
                }
                if (rank < n) {
                    sorted[rank] = mine[0];
                    z[rank] = (v[r][0] - most) * h.inv_t;
                }
            } else {
                sort_keys(mine, lane);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (lane + 64 * u < n) {
                        sorted[lane + 64 * u] = mine[u];
                        z[lane + 64 * u] = (value[mine[u] & 1023] - most) * h.inv_t;
                    }
            }
            wave_sync();
            float total = 0.f;
            for (int i = lane; i < n; i += 64) total += expf(z[i]);
            total = lanes_sum<64>(total);
            const float log_total = logf(total);
            int to = 0;
            for (int i0 = 0; i0 < n; i0 += 64) {
                const int i = i0 + lane;
                const unsigned word = i < n ? sorted[i] >> 10 : 0u;
                const bool leads = i < n && (i == 0 || sorted[i - 1] >> 10 != word);
                const unsigned long long leaders = __ballot(leads);
                if (leads) {
                    float e = expf(z[i]), log_e = z[i];
                    int o = i + 1;
                    for (; o < n && sorted[o] >> 10 == word; ++o) e += expf(z[o]);
                    if (o > i + 1) log_e = logf(e);
                    const int64_t at = list + to + __popcll(leaders & ((1ull << lane) - 1));
                    as_global(k.word)[at] = (int)word;
                    as_global(k.q)[at] = e / total;
                    as_global(k.log_q)[at] = log_e - log_total;
                    atomicAdd(&count[word >> k.shift], 1);
                }
                to += __popcll(leaders);
            }
            if (lane == 0) {
                listed[l - group0] = to;
                as_global(k.words)[l] = to;
                if (write_labels) as_global(write_labels)[token[r]] = to > 0 ? 0 : -1;
            }
            wave_sync();
        }
    }
    __syncthreads();
    // first places of the buckets
    PSGD_GLOBAL int* start = as_global(k.start) + (int64_t)blockIdx.x * (k.buckets + 1);
    int before = 0;
    for (int b0 = 0; b0 < k.buckets; b0 += threads) {
        const int b = b0 + threadIdx.x, mine = b < k.buckets ? count[b] : 0;
        int up = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(up, d);
            up += lane >= d ? o : 0;
        }
        if (lane == 63) sums[wv] = up;
        __syncthreads();
        int at = before + up - mine;
        for (int w = 0; w < waves; ++w) {
            at += w < wv ? sums[w] : 0;
            before += sums[w];
        }
        if (b < k.buckets) { count[b] = at; start[b] = at; }
        __syncthreads();
    }
    if (threadIdx.x == 0) start[k.buckets] = before;
    const int64_t base = (int64_t)group0 * k.top;
    for (int l = group0 + wv; l < min(group0 + GROUP, end); l += waves) {
        const int n = listed[l - group0];
        for (int i = lane; i < n; i += 64) {
            const int64_t at = (int64_t)l * k.top + i;
            const int y = as_global(k.word)[at], place = atomicAdd(&count[y >> k.shift], 1);
            as_global(k.flat)[base + place] = (unsigned)y << 5 | (unsigned)(l - group0);
            as_global(k.place)[at] = place;
        }
    }
}

// ---- logits of a piece: statistics per tile, exponentials --------------------------------------------------------------

// The logits of the teacher's words in this tile: to their places, and out of the accumulators (minus infinity there).  32 rows at a time, through LDS, where any lane can
// look for any word, each wavefront in a place of its own.  (8192 x 4096 x 64000, 64 entries: 40 us of 3430 more than without a teacher; one word of a row after the
// other, sought among a lane's accumulators, took 365.  200 x 1024 x 10007, 100 entries, a quarter of them in one tile: 3 us of 20; 30 of 48.)
// Where they are is asked before the product.
template <class T, TileShape SHAPE> struct TileListed {
    static constexpr int GROUP = group_tokens(SHAPE), SUBS = 32 / GROUP;
    int from[T::FL][SUBS], to[T::FL][SUBS];
};
template <class T, TileShape SHAPE>
__device__ __forceinline__ void where_listed(TileListed<T, SHAPE>& w, const HeadTop& k, int p0, int l0, int nl) {
    constexpr int GROUP = group_tokens(SHAPE);
    const int wl = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) / T::WP;
#pragma unroll
    for (int j = 0; j < T::FL; ++j)
#pragma unroll
        for (int s = 0; s < 32 / GROUP; ++s) {
            const int row0 = l0 + (wl * T::FL + j) * 32 + s * GROUP;
            const PSGD_GLOBAL int* start = as_global(k.start) + (int64_t)(row0 / GROUP) * (k.buckets + 1) + (p0 >> k.shift);
            w.from[j][s] = row0 < nl ? start[0] : 0, w.to[j][s] = row0 < nl ? start[1] : 0;
        }
}
template <class T, TileShape SHAPE>
__device__ __forceinline__ void take_listed(T& tile, const HeadTop& k, const TileListed<T, SHAPE>& w, int p0, int l0, PSGD_TLDS unsigned char* lds) {
    constexpr int COLS = 32 * T::FP, LD = COLS + 4, GROUP = group_tokens(SHAPE), SUBS = 32 / GROUP, AHEAD = 4;
    // rounds of 64 whose loads are sent off first, where there are registers for them (a tile with a quarter of all words has four)
    constexpr int FIRST = tile_share(SHAPE) == 1 && SHAPE != TILE_256 ? 4 : 1;
    const int lane = tile.lane;
    auto base = [&](int j, int s) { return (int64_t)(l0 + (tile.wl * T::FL + j) * 32 + s * GROUP) * k.top; };
    unsigned first[T::FL][SUBS][FIRST];
#pragma unroll
    for (int j = 0; j < T::FL; ++j)
#pragma unroll
        for (int s = 0; s < SUBS; ++s)
#pragma unroll
            for (int r = 0; r < FIRST; ++r) {
                const int i = w.from[j][s] + 64 * r + lane;
                first[j][s][r] = i < w.to[j][s] ? as_global(k.flat)[base(j, s) + i] : 0u;
            }
    __syncthreads();        // (the chunks' reads are done)
    PSGD_TLDS float* mine = reinterpret_cast<PSGD_TLDS float*>(lds) + (tile.wl * T::WP + tile.wp) * 32 * LD;
#pragma unroll
    for (int j = 0; j < T::FL; ++j) {
        int n = 0;
#pragma unroll
        for (int s = 0; s < SUBS; ++s) n += w.to[j][s] - w.from[j][s];
        if (n == 0) continue;
        PSGD_TLDS float* own = mine + (lane & 31) * LD + 4 * (lane >> 5);
#pragma unroll
        for (int i = 0; i < T::FP; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<PSGD_TLDS floatx4*>(own + 32 * i + 8 * q) =
                    floatx4{tile.acc[i][j][4 * q], tile.acc[i][j][4 * q + 1], tile.acc[i][j][4 * q + 2], tile.acc[i][j][4 * q + 3]};
        wave_sync();
#pragma unroll
        for (int s = 0; s < SUBS; ++s) {
            const int64_t at = base(j, s);
            const int to = w.to[j][s];
            auto take = [&](int i, unsigned e) {
                const int col = (int)(e >> 5) - p0 - tile.wp * COLS;
                if (i < to && col >= 0 && col < COLS) {
                    PSGD_TLDS float* x = mine + (s * GROUP + (e & 31)) * LD + col;
                    as_global(k.logit)[at + i] = *x;
                    *x = -__builtin_inff();
                }
            };
#pragma unroll
            for (int r = 0; r < FIRST; ++r) take(w.from[j][s] + 64 * r + lane, first[j][s][r]);
            for (int i0 = w.from[j][s] + 64 * FIRST; i0 < to; i0 += 64 * AHEAD) {
                unsigned e[AHEAD];
#pragma unroll
                for (int r = 0; r < AHEAD; ++r) e[r] = i0 + 64 * r + lane < to ? as_global(k.flat)[at + i0 + 64 * r + lane] : 0u;
#pragma unroll
                for (int r = 0; r < AHEAD; ++r) take(i0 + 64 * r + lane, e[r]);
            }
        }
        wave_sync();
#pragma unroll
        for (int i = 0; i < T::FP; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const floatx4 x = *reinterpret_cast<const PSGD_TLDS floatx4*>(own + 32 * i + 8 * q);
#pragma unroll
                for (int u = 0; u < 4; ++u) tile.acc[i][j][4 * q + u] = x[u];
            }
        wave_sync();
    }
}

// TOP: a teacher's entries in the place of labels
template <TileShape SHAPE, int KEEP, bool TOP>
__global__ __launch_bounds__(kTileThreads, tile_share(SHAPE)) void head_logits_kernel(TileArgs t, HeadDev h) {
    extern __shared__ __align__(16) unsigned char smem[];
    using T = Tile<true, true, SHAPE>;
    constexpr int BL = T::BL;
    const int nl = counted(t, t.L.extent);
    const TilePlace at = tile_place(blockIdx.x, tile_grid<SHAPE>(t, nl, 0));
    if (at.split < 0) return;
    const int p0 = at.p * T::BP, l0 = at.l * BL;
    T tile;
    TileListed<T, SHAPE> listed;
    if constexpr (TOP) where_listed(listed, h.top, p0, l0, nl);
    // (Each tile begins with another chunk: all at the same, W's rows lie a power of two apart and ask for the same channels.  One token's loss, 4096 x 32000: 66 us, 59 so.)
    tile.template run<true>(t, p0, l0, nl, t.K, 0, 1, (PSGD_TLDS unsigned char*)smem, {}, TOP ? at.p % ((t.K + T::BK - 1) / T::BK) : 0);
    if constexpr (TOP) take_listed(tile, h.top, listed, p0, l0, (PSGD_TLDS unsigned char*)smem);
    const float log2e = TOP ? 1.4426950408889634f * h.inv_t : 1.4426950408889634f;
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
        const int y = !TOP && l < nl ? label_of(h, t.first, l) - p0 - tile.col(0, 0) : -1;
        const bool found = !TOP && y >= 0 && y < 32 * T::FP && (y & 4) == 0, any = !TOP && __any(found);
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
                const float e = __builtin_amdgcn_exp2f((tile.acc[i][j][v] - base) * log2e);
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

// exp(u) - 1 - u and exp(u) - 1 of small u by their series, without the digits that the differences lose
constexpr float kSmallU = 0.25f;        // (the next term: 2 u^6 / 40320 of the sum, 1.2e-8)
__device__ __forceinline__ float exp_rest(float u) {
    return u * u * fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, 1.f / 5040, 1.f / 720), 1.f / 120), 1.f / 24), 1.f / 6), 0.5f);
}

// The same against a teacher: with q its probabilities, p the head's and u = log p - log q,
//   loss = sum_v q log(q / p) = sum over the list of (p - q - q u = q (e^u - 1 - u)) + sum over the others of p,
// of whose terms none is negative;  D = c (p - q), p - q = q (e^u - 1).  The others' D comes of their exponentials, the list's is written over it.
// KEPT: rounds of 64 words of the list that a wavefront has in registers (1 for up to 64 entries: 333 x 515 x 10007, 8 entries, 8.9 us, with four 10.4; 4 for more:
// 8192 x 464 x 1280, losses, 256 entries 30.1 us, with four 25.4)
template <int KEEP, int PL, int KEPT>
__global__ __launch_bounds__(kThreads) void head_top_rows_kernel(HeadDev h, int first, int most_rows, int span) {
    __shared__ float shared[4];
    const HeadTop& k = h.top;
    const int l = blockIdx.x, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    if (l >= (h.direct ? most_rows : min(most_rows, *h.count - first))) return;
    const int token = h.direct ? first + l : h.rows[first + l], n = __builtin_amdgcn_readfirstlane(as_global(k.words)[l]);
    const int begin = blockIdx.y * span, end = (int)min((int64_t)(blockIdx.y + 1) * span, h.ldv);
    float scale = 1.f;
    if (KEEP != KEEP_NONE && h.direct && (h.weight || (l == 0 && blockIdx.y == 0))) {
        const bool write = l == 0 && blockIdx.y == 0;
        scale = direct_scale(h, shared, write);
        if (write && threadIdx.x == 0) h.scale[0] = scale * h.inv_t;
    }
    if (n == 0) {
        if (blockIdx.y == 0 && threadIdx.x == 0) h.loss[token] = 0.f;
        if constexpr (KEEP != KEEP_NONE)
            for (int v = begin + 8 * threadIdx.x; v < end; v += 8 * kThreads)
#pragma unroll
                for (int p = 0; p < PL; ++p) *reinterpret_cast<PSGD_GLOBAL uintx4*>(as_global(h.D) + p * h.d_plane + l * h.ldv + v) = uintx4{0u, 0u, 0u, 0u};
        return;
    }
    uintx4 e[KEEP == KEEP_F32 ? 2 : 1];
    auto fetch = [&](int v) {
        if constexpr (KEEP == KEEP_F16) {
            e[0] = __builtin_nontemporal_load(reinterpret_cast<const PSGD_GLOBAL uintx4*>(as_global((_Float16*)h.e) + l * h.ldv + v));
        } else if constexpr (KEEP == KEEP_F32) {
            const PSGD_GLOBAL uintx4* p = reinterpret_cast<const PSGD_GLOBAL uintx4*>(as_global((float*)h.e) + l * h.ldv + v);
            e[0] = __builtin_nontemporal_load(p), e[1] = __builtin_nontemporal_load(p + 1);
        }
    };
    const int start = begin + 8 * threadIdx.x;
    if (KEEP != KEEP_NONE && start < end) fetch(start);
    // (Each wavefront does all this for itself, for the list is short, and the statistics come from the caches: no wavefront waits for another's.)
    struct Word { float logit, q, log_q; int word; };
    const int64_t base = (int64_t)(l / k.group) * k.group * k.top;
    auto load_word = [&](int i) {
        Word w = {-__builtin_inff(), 0.f, 0.f, -1};
        const int64_t at = (int64_t)l * k.top + i;
        if (i < n) w = {as_global(k.logit)[base + as_global(k.place)[at]], as_global(k.q)[at], as_global(k.log_q)[at], as_global(k.word)[at]};
        return w;
    };
    Word kept[KEPT];
#pragma unroll
    for (int r = 0; r < KEPT; ++r) {
        kept[r] = {-__builtin_inff(), 0.f, 0.f, -1};
        if (64 * r < n) kept[r] = load_word(64 * r + lane);
    }
    auto for_words = [&](auto use) {
#pragma unroll
        for (int r = 0; r < KEPT; ++r)
            if (64 * r < n && kept[r].word >= 0) use(kept[r]);
        for (int i = 64 * KEPT + lane; i < n; i += 64) use(load_word(i));
    };
    // the largest logit, and the sums of exp(logit - it) of the list and of the others
    const float inv_t = h.inv_t;
    float most = -__builtin_inff(), mine = 0.f, others = 0.f;
    auto join = [&](float m, float s, float o) {
        const float both = fmaxf(most, m);
        if (both != -__builtin_inff()) {
            const float f = expf((most - both) * inv_t), g = expf((m - both) * inv_t);
            mine = mine * f + s * g, others = others * f + o * g;
        } else {
            mine += s, others += o;
        }
        most = both;
    };
    const float2* st = h.stats + (int64_t)l * h.tiles;
    for (int i = lane; i < h.tiles; i += 64) join(st[i].x, 0.f, st[i].y);
    for_words([&](const Word& w) { join(w.logit, 1.f, 0.f); });
    const float lane_most = most;
    most = lanes_max<64>(most);
    if (lane_most != most) {
        const float f = expf((lane_most - most) * inv_t);
        mine *= f, others *= f;
    }
    mine = lanes_sum<64>(mine), others = lanes_sum<64>(others);
    const float total = mine + others, log_total = logf(total), weight = h.weight ? h.weight[token] / (h.direct ? scale : h.scale[1]) : 1.f;
    struct Off { float p, u; bool small; };
    auto off = [&](const Word& w) {
        const float z = (w.logit - most) * inv_t, u = z - log_total - w.log_q;
        return Off{expf(z) / total, u, fabsf(u) <= kSmallU};
    };
    if (blockIdx.y == 0 && wv == 0) {
        float loss = 0.f;
        for_words([&](const Word& w) {
            const Off o = off(w);
            // (a probability that is 0 in 32 bits has a logarithm all the same, or none)
            loss += o.small ? w.q * exp_rest(o.u) : w.q == 0.f ? o.p : o.p - w.q - w.q * o.u;
        });
        loss = lanes_sum<64>(loss);
        if (lane == 0) h.loss[token] = loss + others / total;
    }
    if constexpr (KEEP == KEEP_NONE) return;
    // a word's D, of all its planes
    auto put = [&](const Word& w) {
        const Off o = off(w);
        bf16_t plane[PL];
        split_planes<PL>((o.small ? w.q * (o.u + exp_rest(o.u)) : o.p - w.q) * weight, plane);
#pragma unroll
        for (int p = 0; p < PL; ++p) as_global(h.D)[p * h.d_plane + l * h.ldv + w.word] = plane[p];
    };
    const float c = weight / total;
    for (int v0 = begin + 512 * wv; v0 < end; v0 += 8 * kThreads) {
        const int v = v0 + 8 * lane;
        if (v < end) {
            const float f = expf((st[v / h.tile_width].x - most) * inv_t) * c * (KEEP == KEEP_F16 ? 1.f / kHalfScale : 1.f);
            float x[8];
            if constexpr (KEEP == KEEP_F16) {
                const halfx8 y = __builtin_bit_cast(halfx8, e[0]);
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] = (float)y[u] * f;
            } else {
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] = __uint_as_float(e[KEEP == KEEP_F32 ? u >> 2 : 0][u & 3]) * f;
            }
            if (v + 8 * kThreads < end) fetch(v + 8 * kThreads);
            bf16x8 out[PL];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                bf16_t plane[PL];
                split_planes<PL>(x[u], plane);
#pragma unroll
                for (int p = 0; p < PL; ++p) out[p][u] = plane[p];
            }
#pragma unroll
            for (int p = 0; p < PL; ++p) *reinterpret_cast<PSGD_GLOBAL bf16x8*>(as_global(h.D) + p * h.d_plane + l * h.ldv + v) = out[p];
        }
        // the list's, as soon as their places are written (later, they would be parts of lines that have left the caches), by the same wavefront: its stores
        // come in their order
        wave_sync();
#pragma unroll
        for (int r = 0; r < KEPT; ++r)
            if (64 * r < n && kept[r].word >= v0 && kept[r].word < min(v0 + 512, end)) put(kept[r]);
    }
    wave_sync();
    for (int i = 64 * KEPT + lane; i < n; i += 64) {
        const Word w = load_word(i);
        if (w.word >= begin && w.word < end && ((w.word - begin) / 512) % (kThreads / 64) == wv) put(w);
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
    size_t entries, word, place, q, log_q, flat, logit, start, words;        // of a teacher
    int64_t ldc, ldv;
    int piece, pieces, tiles, x_planes, d_planes, keep;
    TilePlan logits, dx, dw;
    unsigned dw_pairs;
    int n_dw_pairs;
    bool copy_w, direct, pair;
    int shift, buckets, group;     // of a teacher's words
};

// top: entries of a teacher per token, 0 with labels
static HeadPlan head_plan(const psgd_head_desc& s, bool gradients, int64_t top) {
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
    const size_t row = (!gradients ? s.vocab / 128 * sizeof(float2) + 64 : (size_t)p.ldv * (p.keep == KEEP_F16 ? 2 : 4 + 2 * p.d_planes)) +
                       (top ? 24 * top + s.vocab / 256 + 8 : 0);
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
    p.scale = take(8);
    p.rows = take((size_t)tokens * 4);
    p.label = take((size_t)tokens * 4);
    p.counts = take((size_t)(tokens + 63) / 64 * 8);
    p.xc = p.direct && !gradients ? 0 : take((size_t)tokens * p.ldc * 2 * p.x_planes);      // (direct: where dX takes X's place)
    p.wc = p.copy_w ? take((size_t)s.vocab * p.ldc * 2) : 0;
    p.stats = take((size_t)p.piece * p.tiles * sizeof(float2));
    if (top) {
        p.entries = take((size_t)tokens * 8);
        p.group = group_tokens(p.logits.shape);
        const size_t groups = (p.piece + p.group - 1) / p.group, list = groups * p.group * top * 4;
        p.word = take(list), p.place = take(list), p.q = take(list), p.log_q = take(list), p.flat = take(list), p.logit = take(list);
        for (int width = tile_p(p.logits.shape); width > 1; width /= 2) ++p.shift;
        while (((s.vocab - 1) >> p.shift) >= kBuckets) ++p.shift;
        p.buckets = (int)((s.vocab - 1) >> p.shift) + 1;
        p.start = take(groups * (p.buckets + 1) * 4);
        p.words = take((size_t)p.piece * 4);
    } else {
        p.at_label = take((size_t)p.piece * 4);
    }
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

template <TileShape SHAPE, int KEEP, bool TOP>
static hipError_t launch_logits_as(const TileArgs& t, const HeadDev& h, hipStream_t st) {
    const int64_t blocks = h.tiles * (int64_t)((t.L.extent + tile_l(SHAPE) - 1) / tile_l(SHAPE));
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    auto kfn = head_logits_kernel<SHAPE, KEEP, TOP>;
    constexpr int lds = Tile<true, true, SHAPE>::LDS_BYTES;
    if (lds > 48 * 1024) {
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kfn), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kfn, dim3((unsigned)blocks), dim3(kTileThreads), lds, st, t, h);
    return hipGetLastError();
}
template <TileShape SHAPE, int KEEP>
static hipError_t launch_logits_for(const TileArgs& t, const HeadDev& h, hipStream_t st) {
    return h.top.top ? launch_logits_as<SHAPE, KEEP, true>(t, h, st) : launch_logits_as<SHAPE, KEEP, false>(t, h, st);
}
template <TileShape SHAPE>
static hipError_t launch_logits_shape(const TileArgs& t, const HeadDev& h, hipStream_t st) {
    if (h.keep == KEEP_NONE) return launch_logits_for<SHAPE, KEEP_NONE>(t, h, st);
    if constexpr (!tile_is_split(SHAPE))
        if (h.keep == KEEP_F16) return launch_logits_for<SHAPE, KEEP_F16>(t, h, st);
    return launch_logits_for<SHAPE, KEEP_F32>(t, h, st);
}
static hipError_t launch_logits(const TileArgs& t, const HeadDev& h, TileShape shape, hipStream_t st) {
    if (shape == TILE_256) return launch_logits_shape<TILE_256>(t, h, st);
    if (shape == TILE_128) return launch_logits_shape<TILE_128>(t, h, st);
    if (shape == TILE_MANY) return launch_logits_shape<TILE_MANY>(t, h, st);
    if (shape == TILE_SPLIT) return launch_logits_shape<TILE_SPLIT>(t, h, st);
    if (shape == TILE_SPLIT_THIN) return launch_logits_shape<TILE_SPLIT_THIN>(t, h, st);
    return launch_logits_shape<TILE_THIN>(t, h, st);
}

template <int KEEP, int PL>
static hipError_t launch_rows_as(const HeadDev& h, int first, int rows, int span, dim3 grid, hipStream_t st) {
    if (h.top.top > 64) hipLaunchKernelGGL((head_top_rows_kernel<KEEP, PL, 4>), grid, dim3(kThreads), 0, st, h, first, rows, span);
    else if (h.top.top) hipLaunchKernelGGL((head_top_rows_kernel<KEEP, PL, 1>), grid, dim3(kThreads), 0, st, h, first, rows, span);
    else hipLaunchKernelGGL((head_rows_kernel<KEEP, PL>), grid, dim3(kThreads), 0, st, h, first, rows, span);
    return hipGetLastError();
}
static hipError_t launch_rows(const HeadDev& h, int first, int rows, hipStream_t st) {
    if (h.keep == KEEP_NONE) return launch_rows_as<KEEP_NONE, 1>(h, first, rows, 0, dim3(rows), st);
    // parts of the vocabulary, so that a few rows fill the card as well
    int64_t parts = std::max<int64_t>(1, std::min<int64_t>((h.ldv + 8 * kThreads - 1) / (8 * kThreads), 2048 / std::max(1, rows)));
    const int span = (int)(((h.ldv + parts - 1) / parts + 7) / 8 * 8);
    parts = (h.ldv + span - 1) / span;
    const dim3 grid(rows, (unsigned)parts);
    return h.keep == KEEP_F16 ? launch_rows_as<KEEP_F16, 1>(h, first, rows, span, grid, st) : launch_rows_as<KEEP_F32, 3>(h, first, rows, span, grid, st);
}

// A teacher's entries, in the place of labels.
struct HeadTeacher {
    const int64_t* index;
    const void* logits;
    int dtype;
    int64_t ld, top;
    float temperature;
};
constexpr float kMinTemperature = 1e-30f;       // (what is multiplied by one over it stays in range)
static int teacher_shape(int64_t top) { return top < 1 || top > kMaxTop ? PSGD_E_SHAPE : PSGD_OK; }

template <int U, int GROUP>
static hipError_t launch_lists_as(const HeadDev& h, int first, int rows, int64_t* write_labels, hipStream_t st) {
    auto kfn = head_top_lists_kernel<U, GROUP>;
    constexpr int waves = kListWaves<U, GROUP>;
    const int lds = up4(h.top.buckets) * 4 + waves * U * 64 * 12;
    if (lds > 48 * 1024) {
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kfn), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kfn, dim3((rows + GROUP - 1) / GROUP), dim3(64 * waves), lds, st, h, first, rows, write_labels);
    return hipGetLastError();
}
template <int U>
static hipError_t launch_lists_for(const HeadDev& h, int first, int rows, int64_t* write_labels, hipStream_t st) {
    return h.top.group == 32 ? launch_lists_as<U, 32>(h, first, rows, write_labels, st) : launch_lists_as<U, 8>(h, first, rows, write_labels, st);
}
static hipError_t launch_lists(const HeadDev& h, int first, int rows, int64_t* write_labels, hipStream_t st) {
    const int top = h.top.top;
    return top <= 64 ? launch_lists_for<1>(h, first, rows, write_labels, st) : top <= 128 ? launch_lists_for<2>(h, first, rows, write_labels, st)
         : top <= 256 ? launch_lists_for<4>(h, first, rows, write_labels, st) : top <= 512 ? launch_lists_for<8>(h, first, rows, write_labels, st)
         : launch_lists_for<16>(h, first, rows, write_labels, st);
}

static int head_run(const psgd_head_desc* s, const HeadTeacher* teacher, bool gradients, void* workspace, void* stream, const void* x, const void* w, const int64_t* labels,
                    const float* weight, float* loss, void* dx, void* dw, int accumulate) {
    if (int rc = head_shape(s)) return rc;
    if (teacher) {
        if (bad_dtype(teacher->dtype) || !(teacher->temperature >= kMinTemperature && teacher->temperature <= 1.f / kMinTemperature)) return PSGD_E_INVALID_ARG;
        if (s->tokens != 0 && (!teacher->index || !teacher->logits)) return PSGD_E_INVALID_ARG;
        if (int rc = teacher_shape(teacher->top)) return rc;
        if (teacher->ld > kMaxLd) return PSGD_E_SHAPE;
        if (teacher->ld < teacher->top || misaligned(teacher->index) || misaligned(teacher->logits)) return PSGD_E_ALIGN;
    }
    if (!workspace || !w || (gradients && !dw) || (s->tokens != 0 && (!x || (!labels && !teacher) || !loss || (gradients && !dx)))) return PSGD_E_INVALID_ARG;
    const int64_t ldx = s->ldx ? s->ldx : s->d, ldw = s->ldw ? s->ldw : s->d, lddx = s->lddx ? s->lddx : s->d, lddw = s->lddw ? s->lddw : s->d;
    if (ldx > kMaxLd || ldw > kMaxLd || lddx > kMaxLd || lddw > kMaxLd) return PSGD_E_SHAPE;
    if (bad_ld(ldx, s->d) || bad_ld(ldw, s->d) || misaligned(x) || misaligned(w) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return PSGD_E_ALIGN;
    if (gradients && (bad_ld(lddx, s->d) || bad_ld(lddw, s->d) || misaligned(dx) || misaligned(dw))) return PSGD_E_ALIGN;
    const int64_t size = s->dtype == PSGD_F32 ? 4 : 2, g_size = s->grad_dtype == PSGD_F32 ? 4 : 2;
    const bool in_place = gradients && x && x == dx && (ldx == lddx || s->tokens == 1);
    const int64_t t_size = teacher && teacher->dtype == PSGD_BF16 ? 2 : 4, t_ld = teacher ? teacher->ld : 0, top = teacher ? teacher->top : 0;
    const RowArea in[] = {{teacher ? teacher->index : nullptr, s->tokens, t_ld * 8, top * 8}, {teacher ? teacher->logits : nullptr, s->tokens, t_ld * t_size, top * t_size},
                          {x, s->tokens, ldx * size, s->d * size}, {w, s->vocab, ldw * size, s->d * size}, {labels, 1, 0, s->tokens * 8},
                           {weight, 1, 0, s->tokens * 4}};
    const RowArea out[] = {{dx, s->tokens, lddx * size, s->d * size}, {dw, s->vocab, lddw * g_size, s->d * g_size}, {loss, 1, 0, s->tokens * 4}};
    for (const RowArea& o : out)
        for (const RowArea& i : in)
            if (overlap(o, i) && !(in_place && &o == out && &i == in + 2)) return PSGD_E_INVALID_ARG;
    if (overlap(out[0], out[1]) || overlap(out[0], out[2]) || overlap(out[1], out[2])) return PSGD_E_INVALID_ARG;
    const HeadPlan p = head_plan(*s, gradients, top);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    forget_errors();
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    const bool f32 = s->dtype == PSGD_F32;

    HeadDev h = {};
    int64_t* entries = reinterpret_cast<int64_t*>(ws + p.entries);
    h.labels = teacher ? entries : labels, h.weight = weight, h.loss = loss;
    h.inv_t = 1.f;
    if (teacher) {
        h.inv_t = 1.f / teacher->temperature;
        h.top = {teacher->index, teacher->logits, teacher->dtype, (int)top, teacher->ld};
        h.top.word = reinterpret_cast<int*>(ws + p.word), h.top.place = reinterpret_cast<int*>(ws + p.place);
        h.top.q = reinterpret_cast<float*>(ws + p.q), h.top.log_q = reinterpret_cast<float*>(ws + p.log_q);
        h.top.flat = reinterpret_cast<unsigned*>(ws + p.flat), h.top.logit = reinterpret_cast<float*>(ws + p.logit);
        h.top.start = reinterpret_cast<int*>(ws + p.start), h.top.words = reinterpret_cast<int*>(ws + p.words);
        h.top.buckets = p.buckets, h.top.shift = p.shift, h.top.group = p.group;
    }
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
    if (teacher && !h.direct && s->tokens > 0) {
        const int64_t groups = (s->tokens + kThreads / 64 - 1) / (kThreads / 64);
        hipLaunchKernelGGL(head_top_count_kernel, dim3((unsigned)std::min<int64_t>(groups, 1 << 16)), dim3(kThreads), 0, st, h.top, h.tokens, h.vocab, entries);
        if (hipGetLastError() != hipSuccess) return PSGD_E_HIP;
    }
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
            if (teacher && launch_lists(h, first, rows, h.direct ? entries : nullptr, st) != hipSuccess) return PSGD_E_HIP;
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
    return head_shape(desc) ? 0 : head_plan(*desc, gradients != 0, 0).bytes;
}

int psgd_head_loss(const psgd_head_desc* desc, void* workspace, void* stream, const void* x, const void* w, const int64_t* labels, float* loss) {
    return head_run(desc, nullptr, false, workspace, stream, x, w, labels, nullptr, loss, nullptr, nullptr, 0);
}

int psgd_head_loss_grad(const psgd_head_desc* desc, void* workspace, void* stream, const void* x, const void* w, const int64_t* labels,
                        const float* weight, float* loss, void* dx, void* dw, int accumulate) {
    return head_run(desc, nullptr, true, workspace, stream, x, w, labels, weight, loss, dx, dw, accumulate);
}

size_t psgd_head_distill_workspace_bytes(const psgd_head_desc* desc, int64_t top, int gradients) {
    return head_shape(desc) || teacher_shape(top) ? 0 : head_plan(*desc, gradients != 0, top).bytes;
}

int psgd_head_distill(const psgd_head_desc* desc, void* workspace, void* stream, const void* x, const void* w, int64_t top, const int64_t* index,
                      const void* teacher, int teacher_dtype, int64_t ld_top, float temperature, float* loss) {
    const HeadTeacher t = {index, teacher, teacher_dtype, ld_top, top, temperature};
    return head_run(desc, &t, false, workspace, stream, x, w, nullptr, nullptr, loss, nullptr, nullptr, 0);
}

int psgd_head_distill_grad(const psgd_head_desc* desc, void* workspace, void* stream, const void* x, const void* w, int64_t top, const int64_t* index,
                           const void* teacher, int teacher_dtype, int64_t ld_top, float temperature, const float* weight, float* loss, void* dx, void* dw,
                           int accumulate) {
    const HeadTeacher t = {index, teacher, teacher_dtype, ld_top, top, temperature};
    return head_run(desc, &t, true, workspace, stream, x, w, nullptr, weight, loss, dx, dw, accumulate);
}

}  // extern "C"
