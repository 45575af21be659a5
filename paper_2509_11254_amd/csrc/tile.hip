// Matrix products on tiles with a plain result (see tile_dev.h for the tile itself), the sum of split contractions, and bf16
// planes of fp32 operands.
#include "tile_dev.h"

namespace psgd {

// N consecutive elements of a row of C, of which the first n are inside
template <int N>
__device__ __forceinline__ void store_row(PSGD_GLOBAL float* p, const float (&v)[N], int n, bool add) {
#pragma unroll
    for (int h = 0; h < N; h += 4) {
        if (n >= h + 4) {
            floatx4 o = {v[h], v[h + 1], v[h + 2], v[h + 3]};
            PSGD_GLOBAL floatx4* q = reinterpret_cast<PSGD_GLOBAL floatx4*>(p + h);
            if (add) o += *q;
            *q = o;
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (h + u < n) p[h + u] = add ? p[h + u] + v[h + u] : v[h + u];
        }
    }
}
template <int N>
__device__ __forceinline__ void store_row(PSGD_GLOBAL bf16_t* p, const float (&v)[N], int n, bool add) {
    typedef __attribute__((__vector_size__(N * sizeof(__bf16)))) __bf16 piece;
    if (n >= N) {
        PSGD_GLOBAL piece* q = reinterpret_cast<PSGD_GLOBAL piece*>(p);
        piece o, b;
        if (add) b = *q;
#pragma unroll
        for (int u = 0; u < N; ++u) o[u] = (bf16_t)(add ? v[u] + (float)b[u] : v[u]);
        *q = o;
    } else {
#pragma unroll
        for (int u = 0; u < N; ++u)
            if (u < n) p[u] = (bf16_t)(add ? (float)p[u] + v[u] : v[u]);
    }
}

// what a product kernel writes
enum TileKind { TILE_PART = 0, TILE_F32 = 1, TILE_BF16 = 2 };

// contraction steps and rows of C that count, and the chunks that the shape takes them in
struct TileSize { int K, nl, chunks; };
template <TileShape SHAPE>
__device__ inline TileSize tile_size(const TileArgs& t) {
    TileSize s;
    s.K = t.count_is_k ? counted(t, t.K) : t.K;
    s.nl = t.count_is_k ? t.L.extent : counted(t, t.L.extent);
    s.chunks = (s.K + tile_k(SHAPE) - 1) / tile_k(SHAPE) * t.n_pairs;
    return s;
}

// workgroup `id` of a product
template <bool LKC, TileShape SHAPE, int KIND, bool CODES>
__device__ __forceinline__ void product_tile(int id, const TileArgs& t, const TileOut& o, const TileCodes& codes, PSGD_TLDS unsigned char* lds) {
    using T = Tile<false, LKC, SHAPE>;
    const TileSize size = tile_size<SHAPE>(t);
    const TileGrid grid = tile_grid<SHAPE>(t, size.nl, size.chunks);
    const TilePlace at = tile_place(id, grid);
    if (at.split < 0 || (size.K == 0 && o.skip_empty)) return;
    const int p0 = at.p * T::BP, l0 = at.l * T::BL, nl = size.nl;
    T tile;
    tile.template run<false, CODES>(t, p0, l0, nl, size.K, at.split, grid.n_split, lds, codes);
    const float scale = KIND != TILE_PART && o.scale ? *o.scale : 1.f;
    tile.template for_rows<KIND == TILE_BF16 ? 8 : 4>(lds, [&](int row, int col, auto& v) {
        const int l = l0 + row, c = p0 + col, n = t.P.extent - c;
        if (l >= nl || n <= 0) return;
        if constexpr (KIND == TILE_PART) {
            PSGD_GLOBAL float* p = as_global(o.part) + ((int64_t)at.split * nl + l) * o.part_ld + c;
            *reinterpret_cast<PSGD_GLOBAL floatx4*>(p) = floatx4{v[0], v[1], v[2], v[3]};
        } else {
            const bool in = token_counts(o.tokens, l);
#pragma unroll
            for (int u = 0; u < (KIND == TILE_BF16 ? 8 : 4); ++u) v[u] = in ? v[u] * scale : 0.f;
            const int64_t to = (o.rows ? o.rows[t.first + l] : l) * o.ld + c;
            if constexpr (KIND == TILE_F32) store_row(as_global((float*)o.ptr) + to, v, n, o.accumulate);
            else store_row(as_global((bf16_t*)o.ptr) + to, v, n, o.accumulate);
        }
    });
}

template <bool LKC, TileShape SHAPE, int KIND, bool CODES>
__global__ __launch_bounds__(kTileThreads, tile_share(SHAPE)) void product_kernel(TileArgs t, TileOut o, TileCodes codes) {
    extern __shared__ __align__(16) unsigned char smem[];
    product_tile<LKC, SHAPE, KIND, CODES>(blockIdx.x, t, o, codes, (PSGD_TLDS unsigned char*)smem);
}

// two products that do not depend on each other: together they fill the card better, and one launch is saved
template <int KIND_A, int KIND_B>
__global__ __launch_bounds__(kTileThreads, tile_share(TILE_MANY)) void pair_kernel(TileArgs ta, TileOut oa, TileArgs tb, TileOut ob) {
    extern __shared__ __align__(16) unsigned char smem[];
    if ((int)blockIdx.x < ta.blocks) product_tile<true, TILE_MANY, KIND_A, false>(blockIdx.x, ta, oa, {}, (PSGD_TLDS unsigned char*)smem);
    else product_tile<false, TILE_MANY, KIND_B, false>(blockIdx.x - ta.blocks, tb, ob, {}, (PSGD_TLDS unsigned char*)smem);
}

// sum over the splits, in their order, of four elements per thread
template <TileShape SHAPE>
__global__ __launch_bounds__(kThreads) void split_sum_kernel(TileArgs t, TileOut o) {
    const TileSize size = tile_size<SHAPE>(t);
    if (size.K == 0 && o.skip_empty) return;
    const int nl = size.nl, n_split = tile_grid<SHAPE>(t, nl, size.chunks).n_split;
    const float scale = o.scale ? *o.scale : 1.f;
    const int pieces = (t.P.extent + 3) / 4;
    const int64_t all = (int64_t)nl * pieces, layer = (int64_t)nl * o.part_ld;
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < all; e += (int64_t)gridDim.x * kThreads) {
        const int l = (int)(e / pieces), c = 4 * (int)(e - (int64_t)l * pieces);
        const PSGD_GLOBAL float* p = as_global(o.part) + l * o.part_ld + c;
        floatx4 s = {0.f, 0.f, 0.f, 0.f};
        int k = 0;
        for (; k + 8 <= n_split; k += 8) {        // eight loads in flight
            floatx4 x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = *reinterpret_cast<const PSGD_GLOBAL floatx4*>(p + (k + u) * layer);
#pragma unroll
            for (int u = 0; u < 8; ++u) s += x[u];
        }
        for (; k < n_split; ++k) s += *reinterpret_cast<const PSGD_GLOBAL floatx4*>(p + k * layer);
        const float c0 = token_counts(o.tokens, l) ? scale : 0.f;
        const float v[4] = {c0 != 0.f ? s[0] * c0 : 0.f, c0 != 0.f ? s[1] * c0 : 0.f, c0 != 0.f ? s[2] * c0 : 0.f, c0 != 0.f ? s[3] * c0 : 0.f};
        const int64_t row = o.rows ? o.rows[t.first + l] : l;
        if (o.dtype == PSGD_F32) store_row(as_global((float*)o.ptr) + row * o.ld + c, v, t.P.extent - c, o.accumulate);
        else store_row(as_global((bf16_t*)o.ptr) + row * o.ld + c, v, t.P.extent - c, o.accumulate);
    }
}

// eight columns of a row per thread
template <class T>
__global__ __launch_bounds__(kThreads) void planes_kernel(const T* src, int64_t rows, int cols, int64_t ld, bf16_t* dst, int planes) {
    const int pieces = (cols + 7) / 8;
    const int64_t all = rows * pieces, plane = rows * 8 * pieces;
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < all; e += (int64_t)gridDim.x * kThreads) {
        const int64_t r = e / pieces;
        const int c = 8 * (int)(e - r * pieces);
        const PSGD_GLOBAL T* p = as_global(src) + r * ld + c;
        bf16x8 out[kMaxPlanes];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            bf16_t q[kMaxPlanes];
            split_planes<kMaxPlanes>(c + u < cols ? (float)p[u] : 0.f, q);
#pragma unroll
            for (int k = 0; k < kMaxPlanes; ++k) out[k][u] = q[k];
        }
#pragma unroll
        for (int k = 0; k < kMaxPlanes; ++k)
            if (k < planes) *reinterpret_cast<PSGD_GLOBAL bf16x8*>(as_global(dst) + k * plane + 8 * e) = out[k];
    }
}

constexpr int kUnits = 256;     // compute units; a workgroup of a tile kernel fills one

static double split_us(int split, int64_t extent_p, int64_t extent_l) {
    return split > 1 ? 4 + 0.08 * split + split * (double)extent_p * (double)extent_l * 8e-6 / 8 : 0;
}

// Shape and splits by an estimate in microseconds.  A workgroup takes A before and after its chunks and C per chunk: 256 x 256 11 and 1.65 (the matrix
// cores' rate), 128 x 128 5 and 0.6, 128 x 64 4.5 and 0.45, one to a compute unit; TILE_MANY 5 and 1 with up to two to a compute unit, 0.52 for each
// of three and four (0.7 where it makes the operand of codes).  A split contraction costs a launch (4), its partial sums written and read at 8 TB/s (they stay in the caches), and 0.08 for
// each that a thread adds up.  Weight gradients tokens x out x in, each shape with its best number of splits, in us:
//                    256 x 256   128 x 128   128 x 64   TILE_MANY
//   1 x 4096 x 4096       20.9        29.8       39.5        15.7
//   64 x 11008 x 11008     113         170        244          56
//   300 x 11008 x 11008    161         242        340         112
//   800 x 4096 x 4096     42.8        62.3         82        43.3
//   2000 x 4096 x 4096    74.1       108.3      148.8        80.0
//   8192 x 2048 x 2048    87.4        99.6      131.6        96.6
//   1000 x 2048 x 2048    34.6        23.4       29.9        29.2
//   9001 x 256 x 1032     33.3        28.9       31.7        29.7
//   4096 x 512 x 512      29.8        21.4       19.7
TilePlan tile_plan(int64_t extent_p, int64_t extent_l, int64_t chunks, bool may_split, double restore, bool only_many) {
    struct Way { TileShape shape; bool from_codes; double before, chunk; };
    static const Way ways[] = {{TILE_256, false, 11, 1.65}, {TILE_128, false, 5, 0.6}, {TILE_THIN, false, 4.5, 0.45}, {TILE_MANY, false, 5, 0.52},
                               {TILE_MANY, true, 5, 0.70}};
    TilePlan best = {only_many ? TILE_MANY : TILE_256, 1, false, 1e300};
    for (const Way& way : ways) {
        if ((way.from_codes && !(restore > 0)) || (only_many && way.shape != TILE_MANY)) continue;
        const int64_t p = tile_p(way.shape), l = tile_l(way.shape), tiles = (extent_p + p - 1) / p * ((extent_l + l - 1) / l);
        const int64_t fill = tiles > 0 ? kUnits / tiles : 1;
        for (int64_t want : {(int64_t)1, fill / 4, fill / 2, fill, 2 * fill}) {
            if (want < 1 || (want > 1 && (!may_split || want > 64 || want > chunks))) continue;
            const int64_t share = (chunks + want - 1) / want, split = share > 0 ? (chunks + share - 1) / share : 1;
            const int64_t blocks = tiles * split;
            double us = way.from_codes ? 0 : restore;
            if (way.shape == TILE_MANY) {
                const int64_t last = (blocks % (4 * kUnits) + kUnits - 1) / kUnits;        // workgroups to a compute unit in the last round
                us += (double)(blocks / (4 * kUnits)) * (way.before + share * 4 * way.chunk);
                if (last > 0) us += way.before + share * std::max(way.from_codes ? 1.3 : 1.0, last * way.chunk);
            } else {
                us += (double)((blocks + kUnits - 1) / kUnits) * (way.before + share * way.chunk);
            }
            us += split_us((int)split, extent_p, extent_l);
            if (us < best.us) best = {way.shape, (int)split, way.from_codes, us};
        }
    }
    return best;
}

// As above for fp32 operands.  Measured, us per chunk of 32 steps: a compute unit with one workgroup 2.0 (128 x 128) and 0.7 (64 x 64, which loads three
// chunks ahead), full 1.4 and 0.55 for each of its three.  Loss, tokens x d x vocab: 1 x 4096 x 32000 on wide tiles 243 us, narrow 132;
// 256 x 4096 x 32000 382 and 520; 256 x 512 x 4400 39 and 26.  Two narrow ones to a compute unit with four chunks ahead: 512 x 512 x 4400 with gradients 100 us
// in place of 90, 200 x 1024 x 10008 141 in place of 131.
TilePlan split_plan(int64_t extent_p, int64_t extent_l, int64_t chunks, bool may_split) {
    constexpr int share_cu = tile_share(TILE_SPLIT);
    static_assert(share_cu == tile_share(TILE_SPLIT_THIN), "workgroups to a compute unit");
    TilePlan best = {TILE_SPLIT, 1, false, 1e300};
    for (TileShape shape : {TILE_SPLIT, TILE_SPLIT_THIN}) {
        const int64_t w = tile_p(shape), l = tile_l(shape), tiles = (extent_p + w - 1) / w * ((extent_l + l - 1) / l);
        const int64_t fill = tiles > 0 ? kUnits / tiles : 1;
        for (int64_t want : {(int64_t)1, fill / 2, fill, 2 * fill, share_cu * fill}) {
            want = std::min({want, chunks, (int64_t)64});
            if (want < 1 || (want > 1 && !may_split)) continue;
            const int64_t share = (chunks + want - 1) / want, split = share > 0 ? (chunks + share - 1) / share : 1, blocks = tiles * split;
            const double most = shape == TILE_SPLIT ? 1.4 : 0.55, least = shape == TILE_SPLIT ? 2.0 : 0.7;
            const int64_t last = (blocks % (share_cu * kUnits) + kUnits - 1) / kUnits;
            double us = (double)(blocks / (share_cu * kUnits)) * (6 + share * share_cu * most);
            if (last > 0) us += 6 + share * std::max(least, last * most);
            us += split_us((int)split, extent_p, extent_l);
            if (us < best.us) best = {shape, (int)split, false, us};
        }
    }
    return best;
}

// Both products' workgroups fill the compute units together and take as long as the longer contraction; a launch less (3 us).  (Gradients of the head, tokens x d x
// vocab, in us without the pair and with it: 16 x 512 x 4400 32.0, 26.7; 512 x 512 x 4400 54.6, 47.5; 128 x 1024 x 10008 46.0, 39.7; what is not paired by this rule,
// 200 x 1024 x 10008, was 57.2 and 59.)
bool pair_pays(const TilePair& a, const TilePair& b, const TilePlan& a_alone) {
    const int64_t blocks = a.tiles * a.plan.n_split + b.tiles * b.plan.n_split, rounds = (blocks + 4 * kUnits - 1) / (4 * kUnits);
    const int64_t share = std::max((a.chunks + a.plan.n_split - 1) / a.plan.n_split, (b.chunks + b.plan.n_split - 1) / b.plan.n_split);
    const double to_a_unit = (double)std::min<int64_t>(4, (blocks + kUnits - 1) / kUnits);
    const double pair = rounds * (5 + share * std::max(1.0, 0.52 * to_a_unit)) + split_us(a.plan.n_split, a.extent_p, a.extent_l) +
                        split_us(b.plan.n_split, b.extent_p, b.extent_l);
    return pair < a_alone.us + b.plan.us + 3;
}

size_t tile_part_bytes(int64_t extent_p, int64_t extent_l, const TilePlan& plan) {
    // (whole tiles: where fewer rows count there are more parts of as many tiles in all)
    const int64_t rows = (extent_l + tile_l(plan.shape) - 1) / tile_l(plan.shape) * tile_l(plan.shape);
    return plan.n_split > 1 ? up256((size_t)plan.n_split * rows * up8(extent_p) * sizeof(float)) : 0;
}

template <bool LKC, TileShape SHAPE, int KIND, bool CODES>
static hipError_t launch_kind(const TileArgs& t, const TileOut& o, const TileCodes& codes, hipStream_t st) {
    auto kfn = product_kernel<LKC, SHAPE, KIND, CODES>;
    constexpr int lds = Tile<false, LKC, SHAPE>::LDS_BYTES;
    if (lds > 48 * 1024) {
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kfn), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kfn, dim3(t.blocks), dim3(kTileThreads), lds, st, t, o, codes);
    return hipGetLastError();
}
// what a launch needs to know of a product
template <TileShape SHAPE>
static hipError_t complete(TileArgs& t, TileOut& o) {
    if (t.n_split == 1) o.part = nullptr;
    o.part_ld = up8(t.P.extent);
    const int64_t n_p = (t.P.extent + tile_p(SHAPE) - 1) / tile_p(SHAPE), n_l = (t.L.extent + tile_l(SHAPE) - 1) / tile_l(SHAPE);
    if (n_p * n_l * t.n_split > INT32_MAX / 2) return hipErrorInvalidValue;
    t.blocks = (int)(n_p * n_l * t.n_split);
    return hipSuccess;
}
template <TileShape SHAPE>
static hipError_t launch_sum(const TileArgs& t, const TileOut& o, hipStream_t st) {
    if (!o.part) return hipSuccess;
    const int64_t pieces = (int64_t)t.L.extent * ((t.P.extent + 3) / 4);
    hipLaunchKernelGGL(split_sum_kernel<SHAPE>, dim3((unsigned)std::min<int64_t>((pieces + kThreads - 1) / kThreads, 8 * kUnits)), dim3(kThreads), 0, st, t, o);
    return hipGetLastError();
}
template <bool LKC, TileShape SHAPE, bool CODES = false>
static hipError_t launch_shape(TileArgs t, TileOut o, hipStream_t st, const TileCodes& codes = {}) {
    hipError_t e = complete<SHAPE>(t, o);
    if (e != hipSuccess) return e;
    if (!o.part) return o.dtype == PSGD_F32 ? launch_kind<LKC, SHAPE, TILE_F32, CODES>(t, o, codes, st) : launch_kind<LKC, SHAPE, TILE_BF16, CODES>(t, o, codes, st);
    e = launch_kind<LKC, SHAPE, TILE_PART, CODES>(t, o, codes, st);
    return e != hipSuccess ? e : launch_sum<SHAPE>(t, o, st);
}

template <int KIND_A, int KIND_B>
static hipError_t launch_pair_as(const TileArgs& ta, const TileOut& oa, const TileArgs& tb, const TileOut& ob, hipStream_t st) {
    auto kfn = pair_kernel<KIND_A, KIND_B>;
    constexpr int lds = Tile<false, false, TILE_MANY>::LDS_BYTES;
    static_assert(lds == Tile<false, true, TILE_MANY>::LDS_BYTES, "one size for both");
    static_assert(lds <= 48 * 1024, "no attribute");
    hipLaunchKernelGGL(kfn, dim3(ta.blocks + tb.blocks), dim3(kTileThreads), lds, st, ta, oa, tb, ob);
    return hipGetLastError();
}
template <int KIND_A>
static hipError_t launch_pair_from(const TileArgs& ta, const TileOut& oa, const TileArgs& tb, const TileOut& ob, hipStream_t st) {
    if (ob.part) return launch_pair_as<KIND_A, TILE_PART>(ta, oa, tb, ob, st);
    return ob.dtype == PSGD_F32 ? launch_pair_as<KIND_A, TILE_F32>(ta, oa, tb, ob, st) : launch_pair_as<KIND_A, TILE_BF16>(ta, oa, tb, ob, st);
}
hipError_t launch_pair(const TileArgs& first, const TileOut& first_out, const TileArgs& second, const TileOut& second_out, hipStream_t st) {
    TileArgs ta = first, tb = second;
    TileOut oa = first_out, ob = second_out;
    hipError_t e = complete<TILE_MANY>(ta, oa);
    if (e == hipSuccess) e = complete<TILE_MANY>(tb, ob);
    if (e != hipSuccess) return e;
    e = oa.part ? launch_pair_from<TILE_PART>(ta, oa, tb, ob, st)
                : oa.dtype == PSGD_F32 ? launch_pair_from<TILE_F32>(ta, oa, tb, ob, st) : launch_pair_from<TILE_BF16>(ta, oa, tb, ob, st);
    if (e == hipSuccess) e = launch_sum<TILE_MANY>(ta, oa, st);
    return e != hipSuccess ? e : launch_sum<TILE_MANY>(tb, ob, st);
}

hipError_t launch_code_product(const TileCodes& codes, const TileArgs& t, const TileOut& o, hipStream_t st) {
    return launch_shape<false, TILE_MANY, true>(t, o, st, codes);
}

hipError_t launch_product(bool l_contiguous, TileShape shape, const TileArgs& t, const TileOut& o, hipStream_t st) {
    if (l_contiguous) {
        if (shape == TILE_256) return launch_shape<true, TILE_256>(t, o, st);
        if (shape == TILE_128) return launch_shape<true, TILE_128>(t, o, st);
        if (shape == TILE_MANY) return launch_shape<true, TILE_MANY>(t, o, st);
        if (shape == TILE_SPLIT) return launch_shape<true, TILE_SPLIT>(t, o, st);
        if (shape == TILE_SPLIT_THIN) return launch_shape<true, TILE_SPLIT_THIN>(t, o, st);
        return launch_shape<true, TILE_THIN>(t, o, st);
    }
    if (shape == TILE_256) return launch_shape<false, TILE_256>(t, o, st);
    if (shape == TILE_128) return launch_shape<false, TILE_128>(t, o, st);
    if (shape == TILE_MANY) return launch_shape<false, TILE_MANY>(t, o, st);
    if (shape == TILE_SPLIT) return launch_shape<false, TILE_SPLIT>(t, o, st);
    if (shape == TILE_SPLIT_THIN) return launch_shape<false, TILE_SPLIT_THIN>(t, o, st);
    return launch_shape<false, TILE_THIN>(t, o, st);
}

hipError_t launch_planes(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, bf16_t* dst, int planes, hipStream_t st) {
    if (rows == 0) return hipSuccess;
    const dim3 grid((unsigned)std::min<int64_t>((rows * ((cols + 7) / 8) + kThreads - 1) / kThreads, 32 * kUnits));
    if (dtype == PSGD_F32) hipLaunchKernelGGL(planes_kernel<float>, grid, dim3(kThreads), 0, st, (const float*)src, rows, (int)cols, ld, dst, planes);
    else hipLaunchKernelGGL(planes_kernel<bf16_t>, grid, dim3(kThreads), 0, st, (const bf16_t*)src, rows, (int)cols, ld, dst, planes);
    return hipGetLastError();
}

}  // namespace psgd
