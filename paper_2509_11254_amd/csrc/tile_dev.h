// The matrix product on bf16 operands that the training operators share: C[l][p] = sum_k L(l, k) P(p, k), one tile of BL x BP
// elements of C per workgroup, on v_mfma_f32_32x32x16_bf16 with fp32 accumulation.
//
// An operand is stored with the contraction along its rows ("K-contiguous": [extent][K], X and W in X W^T) or down its
// columns ("K-strided": [K][extent], both operands of a weight gradient dY^T X), always row-major.  Chunks of 32 or 64 contraction
// steps go to LDS by direct loads, 16 bytes per lane, without passing through registers; the buffer descriptor's range check
// turns what lies outside the operand into zeros.  K-contiguous chunks are [extent][steps], read 16 bytes (one fragment) per
// lane; K-strided chunks are [steps][extent], read by the transposing LDS load, which hands a lane four steps of its column.
//
// P runs along the accumulators' registers and L along the lanes, so that a lane holds four consecutive elements of a row of C,
// and half a wavefront's 32 lanes 32 rows.
#pragma once
#include "act_dev.h"
#include "train.h"

namespace psgd {

#define PSGD_TLDS __attribute__((address_space(3)))
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short shortx4;
typedef __attribute__((__vector_size__(8 * sizeof(short)))) short shortx8;

constexpr unsigned kOutside = 0x80000000u;      // byte offset beyond every descriptor's range

__device__ inline int counted(const TileArgs& a, int upper) {
    if (!a.count) return upper;
    return __builtin_amdgcn_readfirstlane(max(0, min(upper, *a.count - a.first)));
}

// Tiles and parts of the contraction of a product of nl rows that count: where that is fewer than the launch was planned for, its workgroups
// go to more parts.  chunks: of the whole contraction.
struct TileGrid { int n_p, n_l, n_split; };
template <TileShape SHAPE>
__device__ inline TileGrid tile_grid(const TileArgs& t, int nl, int chunks) {
    TileGrid g;
    g.n_p = (t.P.extent + tile_p(SHAPE) - 1) / tile_p(SHAPE);
    g.n_l = (nl + tile_l(SHAPE) - 1) / tile_l(SHAPE);
    g.n_split = t.n_split == 1 || nl == 0 ? 1 : max(1, min(chunks, t.blocks / (g.n_p * g.n_l)));
    return g;
}

// Which tile a workgroup takes (split < 0: none).  Consecutive workgroups go to consecutive XCDs; each XCD gets a run of consecutive tiles
// (its L2 then holds operands that its workgroups share), and a run goes through 8 tiles along L before the next along P.
struct TilePlace { int p, l, split; };
__device__ inline TilePlace tile_place(int id, const TileGrid& g) {
    const int n_p = g.n_p, n_l = g.n_l, n = n_p * n_l * g.n_split, q = n >> 3, r = n & 7, x = id & 7;
    if (id >= n) return {0, 0, -1};
    int t = (x < r ? x * (q + 1) : r * (q + 1) + (x - r) * q) + (id >> 3);
    TilePlace at;
    at.split = t / (n_p * n_l);
    t -= at.split * n_p * n_l;
    const int group = t / (8 * n_p), l0 = 8 * group, wide = min(8, n_l - l0);
    t -= group * 8 * n_p;
    at.p = t / wide;
    at.l = l0 + t - at.p * wide;
    return at;
}

__device__ __forceinline__ bool token_counts(TileTokens tokens, int i) { return !tokens || ((as_global(tokens)[i >> 6] >> (i & 63)) & 1); }

// a value that is the same in all lanes, in a scalar register
__device__ __forceinline__ unsigned scalar(unsigned x) { return (unsigned)__builtin_amdgcn_readfirstlane((int)x); }

// One operand's side of a tile: E elements of C wide, waves NW.
template <bool KC, int E, int BK, int NW>
struct TileSide {
    static constexpr int LOADS = E * BK * 2 / (NW * 1024);      // direct loads of 1 KB per wave and chunk
    static constexpr int BYTES = E * BK * 2;
    static_assert(LOADS >= 1 && LOADS * NW * 1024 == BYTES, "chunk");

    // K-contiguous: rows of 2 BK bytes, piece c of row r at place c ^ swizzle(r): sixteen rows' reads of one piece cover all 64
    // banks.  K-strided: rows of 2 E bytes, 64-byte piece c of row k at place c ^ turn(k): the four rows that a transposing read
    // takes lie in different banks.
    static constexpr int PIECES = BK / 8;       // of 16 bytes in a K-contiguous row
    __device__ static int turn(int k) { return E == 64 ? (k >> 1) & 1 : k & 3; }
    __device__ static int swizzle(int r) { return BK == 64 ? (r >> 1) & 7 : (r >> 2) & 3; }
    unsigned off[LOADS];
    int kpiece;          // K-contiguous: first step of this lane's pieces, K-strided: unused

    __device__ void init(const TileOperand& o, int start, int extent, int wv, int lane) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int block = i * NW + wv;
            if constexpr (KC) {
                const int row = block * (64 / PIECES) + lane / PIECES, piece = (lane % PIECES) ^ swizzle(row);
                kpiece = 8 * piece;      // the same for all i: the rows are multiples of 16 apart
                off[i] = start + row < extent ? (unsigned)(((int64_t)row * o.ld + 8 * piece) * 2) : kOutside;
            } else {
                constexpr int LANES = E / 8, ROWS = 64 / LANES;     // lanes per row, rows per load
                const int k = block * ROWS + lane / LANES, place = lane % LANES, col = 8 * (place ^ (turn(k) << 2));
                off[i] = start + col < extent ? (unsigned)(((int64_t)k * o.ld + col) * 2) : kOutside;
            }
        }
    }

    // chunk from step k0 on of K: where its loads take it from ...
    struct Source { uintx4 rsrc; int left; };
    __device__ __forceinline__ static Source source(const TileOperand& o, int plane, int start, int k0, int K, bool wanted) {
        const bf16_t* base = o.ptr + plane * o.plane + (KC ? (int64_t)start * o.ld + k0 : (int64_t)k0 * o.ld + start);
        const int64_t left = KC ? (int64_t)kOutside : (int64_t)(K - k0) * o.ld * 2 - 2 * start;
        const unsigned bytes = wanted ? (unsigned)min(left, (int64_t)kOutside) : 0u;
        const uint64_t at = reinterpret_cast<uint64_t>(base);
        return {uintx4{scalar((unsigned)at), scalar((unsigned)(at >> 32) & 0xffffu), scalar(bytes), 0x00020000u}, (int)scalar(K - k0)};
    }
    // ... and load I of them, to the chunk's place in LDS
    template <int I>
    __device__ __forceinline__ void load(const Source& s, PSGD_TLDS unsigned char* dst, int wv) const {
        const unsigned v = KC && kpiece >= s.left ? kOutside : off[I];
        // (Written out so that the compiler, which cannot tell the places in LDS apart, does not wait for all loads before each
        // transposing read.  No result: what is in flight holds no register.  run() does the waiting.  m0 is a register the compiler reserves, and sets
        // before each instruction of its own that takes it, of which these kernels have none.)
        const unsigned to = scalar((unsigned)(uintptr_t)(dst + (I * NW + wv) * 1024));
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(v), "s"(s.rsrc));
    }
    // K-strided: all loads of the chunk from step k0 on, without the steps that do not count
    __device__ __forceinline__ void load_counted(const Source& s, PSGD_TLDS unsigned char* dst, int wv, int lane, TileTokens tokens, int k0) {
        constexpr int LANES = E / 8, ROWS = 64 / LANES;
        static_assert(BK == 64, "one word of bits");
        const uint64_t counts = as_global(tokens)[k0 >> 6];
        unsigned kept[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int k = (i * NW + wv) * ROWS + lane / LANES;
            kept[i] = off[i];
            off[i] = (counts >> k) & 1 ? off[i] : kOutside;
        }
        load_all(s, dst, wv);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) off[i] = kept[i];
    }
    __device__ __forceinline__ void load_all(const Source& s, PSGD_TLDS unsigned char* dst, int wv) const {
        load<0>(s, dst, wv);
        if constexpr (LOADS > 1) load<1>(s, dst, wv);
        if constexpr (LOADS > 2) load<2>(s, dst, wv);
        if constexpr (LOADS > 3) load<3>(s, dst, wv);
        if constexpr (LOADS > 4) { load<4>(s, dst, wv); load<5>(s, dst, wv); load<6>(s, dst, wv); load<7>(s, dst, wv); }
        static_assert(LOADS <= 4 || LOADS == 8, "loads");
    }
};

// fragment of 32 elements from e0 on (a multiple of 32), steps 16 kk .. + 15 of the chunk: lane li + 32 lg gets steps 8 lg .. + 7 of element li
template <bool KC, int E, int BK>
struct TileFragment {
    unsigned base[4];   // K-contiguous: by kk.  K-strided: by fragment (up to 4 of a wave)
    __device__ void init(int e0, int lane) {
        const int li = lane & 31, lg = lane >> 5;
        if constexpr (KC) {
#pragma unroll
            for (int kk = 0; kk < BK / 16; ++kk)
                base[kk] = (unsigned)((e0 + li) * 2 * BK + (((2 * kk + lg) ^ TileSide<KC, E, BK, 4>::swizzle(li)) << 4));
        } else {
            const int row = 8 * lg + ((lane & 15) >> 2);
#pragma unroll
            for (int f = 0; f < 4; ++f)
                base[f] = (unsigned)(row * 2 * E + (((2 * (e0 + 32 * f)) ^ (TileSide<KC, E, BK, 4>::turn(row) << 6)) + 32 * ((lane >> 4) & 1) + 8 * (lane & 3)));
        }
    }
    template <int KK, int F>
    __device__ bf16x8 read(const PSGD_TLDS unsigned char* chunk) const {
        if constexpr (KC) {
            return *reinterpret_cast<const PSGD_TLDS bf16x8*>(chunk + base[KK] + F * 32 * 2 * BK);
        } else {
            const PSGD_TLDS unsigned char* at = chunk + base[F] + KK * 16 * 2 * E;
            const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PSGD_TLDS shortx4*)at);
            const shortx4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PSGD_TLDS shortx4*)(at + 4 * 2 * E));
            const shortx8 v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(bf16x8, v);
        }
    }
};

// Waves along P and L, chunks in LDS.  All have four waves, one per SIMD.
// workgroups to a compute unit
constexpr int tile_share(TileShape s) { return s == TILE_MANY ? 4 : tile_is_split(s) ? 3 : 1; }
template <TileShape SHAPE> struct TileWaves;
template <> struct TileWaves<TILE_256> { static constexpr int WP = 2, WL = 2, STAGES = 0; };
template <> struct TileWaves<TILE_128> { static constexpr int WP = 2, WL = 2, STAGES = 5; };
template <> struct TileWaves<TILE_MANY> { static constexpr int WP = 2, WL = 2, STAGES = 1; };
template <> struct TileWaves<TILE_SPLIT> { static constexpr int WP = 2, WL = 2, STAGES = 1; };
template <> struct TileWaves<TILE_SPLIT_THIN> { static constexpr int WP = 2, WL = 2, STAGES = 1; };
template <> struct TileWaves<TILE_THIN> { static constexpr int WP = 2, WL = 2, STAGES = 6; };

template <bool PKC, bool LKC, TileShape SHAPE>
struct Tile {
    using S = TileWaves<SHAPE>;
    static constexpr int BP = tile_p(SHAPE), BL = tile_l(SHAPE), WP = S::WP, WL = S::WL, NW = WP * WL, BK = tile_k(SHAPE), STAGES = S::STAGES;
    static constexpr bool FULL = SHAPE == TILE_256, SPLIT = tile_is_split(SHAPE);
    static constexpr int RING = SHAPE == TILE_SPLIT_THIN ? 3 : 1;      // chunks of L in LDS (SPLIT)
    static constexpr int FP = BP / WP / 32, FL = BL / WL / 32;      // fragments per wave
    using SideP = TileSide<PKC, BP, BK, NW>;
    using SideL = TileSide<LKC, BL, BK, NW>;
    static constexpr int STAGE_BYTES = SideP::BYTES + SideL::BYTES;
    static constexpr int ROWS_BYTES = NW * 32 * (32 * FP + 4) * 4;         // for_rows()
    static constexpr int CHUNK_BYTES = FULL ? 5 * SideP::BYTES : SPLIT ? kMaxPlanes * (SideP::BYTES + RING * SideL::BYTES) : STAGES * STAGE_BYTES;
    static constexpr int LDS_BYTES = CHUNK_BYTES > ROWS_BYTES ? CHUNK_BYTES : ROWS_BYTES;
    static constexpr int LOADS = SideP::LOADS + SideL::LOADS;
    static_assert(FP >= 1 && FL >= 1 && FP <= 4 && FL <= 4 && NW * 64 == kTileThreads && LDS_BYTES <= 160 * 1024, "waves");
    static_assert((STAGES - 1) * LOADS <= 63 && (STAGES < 2 || LOADS >= 3), "the wait counter's range, thirds");
    static_assert(tile_share(SHAPE) * LDS_BYTES <= 160 * 1024, "workgroups to a compute unit");

    floatx16 acc[FP][FL];
    int wp, wl, lane;

    template <int KK>
    __device__ __forceinline__ void read_ab(const PSGD_TLDS unsigned char* cp, const PSGD_TLDS unsigned char* cl, const TileFragment<PKC, BP, BK>& fp,
                                            const TileFragment<LKC, BL, BK>& fl, bf16x8 (&a)[FP], bf16x8 (&b)[FL]) {
        a[0] = fp.template read<KK, 0>(cp);
        if constexpr (FP > 1) a[1] = fp.template read<KK, 1>(cp);
        if constexpr (FP > 2) a[2] = fp.template read<KK, 2>(cp);
        if constexpr (FP > 3) a[3] = fp.template read<KK, 3>(cp);
        b[0] = fl.template read<KK, 0>(cl);
        if constexpr (FL > 1) b[1] = fl.template read<KK, 1>(cl);
        if constexpr (FL > 2) b[2] = fl.template read<KK, 2>(cl);
        if constexpr (FL > 3) b[3] = fl.template read<KK, 3>(cl);
    }
    __device__ __forceinline__ void multiply(const bf16x8 (&a)[FP], const bf16x8 (&b)[FL]) {
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int j = 0; j < FL; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
    }
    // 16 steps: multiply a, b; on the way read the fragments of steps 16 KK .. of (cp, cl) into an, bn and send off loads H, H + 1, .. + 3
    // of a side's chunk.  Loads and reads go between the products, two products apart.
    template <int KK, int H, class Side>
    __device__ __forceinline__ void round(const bf16x8 (&a)[FP], const bf16x8 (&b)[FL], bf16x8 (&an)[FP], bf16x8 (&bn)[FL],
                                          const PSGD_TLDS unsigned char* cp, const PSGD_TLDS unsigned char* cl, const TileFragment<PKC, BP, BK>& fp,
                                          const TileFragment<LKC, BL, BK>& fl, const Side& side, const typename Side::Source& src,
                                          PSGD_TLDS unsigned char* dst, int wv) {
        an[0] = fp.template read<KK, 0>(cp);
        bn[0] = fl.template read<KK, 0>(cl);
        two<0, 0>(a, b);
        an[1] = fp.template read<KK, 1>(cp);
        bn[1] = fl.template read<KK, 1>(cl);
        two<0, 2>(a, b);
        side.template load<H>(src, dst, wv);
        two<1, 0>(a, b);
        an[2] = fp.template read<KK, 2>(cp);
        bn[2] = fl.template read<KK, 2>(cl);
        two<1, 2>(a, b);
        side.template load<H + 1>(src, dst, wv);
        two<2, 0>(a, b);
        an[3] = fp.template read<KK, 3>(cp);
        bn[3] = fl.template read<KK, 3>(cl);
        two<2, 2>(a, b);
        side.template load<H + 2>(src, dst, wv);
        two<3, 0>(a, b);
        side.template load<H + 3>(src, dst, wv);
        two<3, 2>(a, b);
    }
    template <int I, int J>
    __device__ __forceinline__ void two(const bf16x8 (&a)[FP], const bf16x8 (&b)[FL]) {
        __builtin_amdgcn_sched_barrier(0);
        acc[I][J] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[I], b[J], acc[I][J], 0, 0, 0);
        acc[I][J + 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[I], b[J + 1], acc[I][J + 1], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    }

    // The large tile.  A wave has 128 x 128 elements: the least LDS traffic per product, and one wave per SIMD, which reads the
    // fragments of 16 steps while it multiplies those before.  Five places of 32 KB in LDS take the operands' chunks in turn, P's of a chunk, L's,
    // P's of the next.  The barrier is before a chunk's last 16 steps, when their fragments are in registers: every wave is then done
    // with both places of the chunk, and its loads of the next chunk have arrived.  After it L's part of the chunk after the next goes to
    // one of the places, and then P's of the chunk after that.  Past the end the loads bring zeros, so that no wait depends on where one is.
    // 8192 x 11008 x 4096 (both operands K-strided) takes 600 to 615 us in passes after each other, 1.20 to 1.23 PFLOP/s; eight waves of 64 x 128 in two stages reached 0.85.  Without its loads the loop does
    // 1.7 to 1.8 PFLOP/s, and with zeros for data 1.5: what bounds it is the power that its operands' bits take.
    __device__ __forceinline__ void run_full(const TileArgs& t, int p0, int l0, int K, int n0, int n, int per, int wv, const SideP& sp,
                                             const SideL& sl, const TileFragment<PKC, BP, BK>& fp, const TileFragment<LKC, BL, BK>& fl,
                                             PSGD_TLDS unsigned char* lds) {
        constexpr int PLACE = SideP::BYTES;
        static_assert(SideP::BYTES == SideL::BYTES && SideP::LOADS == 8 && SideL::LOADS == 8, "places");
        int left_p = n, left_l = n;
        int pair_p = n0 / per, kc_p = n0 - pair_p * per, pair_l = pair_p, kc_l = kc_p, at = 0;
        auto next_p = [&]() {
            const auto s = SideP::source(t.P, (t.pairs >> (4 * pair_p)) & 3, p0, kc_p * BK, K, left_p > 0);
            --left_p;
            const bool wrap = ++kc_p == per;
            kc_p = wrap ? 0 : kc_p;
            pair_p = min(pair_p + (wrap ? 1 : 0), 7);
            return s;
        };
        auto next_l = [&]() {
            const auto s = SideL::source(t.L, (t.pairs >> (4 * pair_l + 2)) & 3, l0, kc_l * BK, K, left_l > 0);
            --left_l;
            const bool wrap = ++kc_l == per;
            kc_l = wrap ? 0 : kc_l;
            pair_l = min(pair_l + (wrap ? 1 : 0), 7);
            return s;
        };
        auto place = [&](int i) { const int u = at + i; return lds + (u >= 5 ? u - 5 : u) * PLACE; };
        sp.load_all(next_p(), place(0), wv);
        sl.load_all(next_l(), place(1), wv);
        sp.load_all(next_p(), place(2), wv);
        typename SideL::Source source_l = next_l();
        sl.template load<0>(source_l, place(3), wv);
        sl.template load<1>(source_l, place(3), wv);
        sl.template load<2>(source_l, place(3), wv);
        sl.template load<3>(source_l, place(3), wv);
        asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        bf16x8 a0[FP], b0[FL], a1[FP], b1[FL];
        read_ab<0>(lds, lds + PLACE, fp, fl, a0, b0);
        for (int it = 0; it < n; ++it) {
            const PSGD_TLDS unsigned char* cp = place(0);
            const PSGD_TLDS unsigned char* cl = place(1);
            PSGD_TLDS unsigned char* dl = place(3);
            PSGD_TLDS unsigned char* dp = place(4);
            const typename SideP::Source source_p = next_p();
            round<1, 4>(a0, b0, a1, b1, cp, cl, fp, fl, sl, source_l, dl, wv);
            round<2, 0>(a1, b1, a0, b0, cp, cl, fp, fl, sp, source_p, dp, wv);
            round<3, 4>(a0, b0, a1, b1, cp, cl, fp, fl, sp, source_p, dp, wv);
            asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            PSGD_TLDS unsigned char* const now = place(0);      // where L's part of the chunk after the next goes: P's place of this one
            at = at + 2 >= 5 ? at - 3 : at + 2;
            source_l = next_l();
            round<0, 0>(a1, b1, a0, b0, place(0), place(1), fp, fl, sl, source_l, now, wv);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    }

    // acc = the tile at (p0, l0), part `split` of n_split of the contraction over K steps; nl: rows of C there are.  MINUS_INF: what lies beyond P's
    // extent comes out as -inf, where sums begin that only get zeros added.  turn: the chunk a ring begins with, where there is one pair of planes and one part
    template <bool MINUS_INF = false, bool CODES = false>
    __device__ void run(const TileArgs& t, int p0, int l0, int nl, int K, int split, int n_split, PSGD_TLDS unsigned char* lds,
                        const TileCodes& codes = {}, int turn = 0) {
        lane = threadIdx.x & 63;
        const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wp = wv % WP;
        wl = wv / WP;
        const int end = t.P.extent - p0 - col(0, 0);
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float start = MINUS_INF && 32 * i + 8 * (v >> 2) + (v & 3) >= end ? -__builtin_inff() : 0.f;
#pragma unroll
                for (int j = 0; j < FL; ++j) acc[i][j][v] = start;
            }
        SideP sp;
        SideL sl;
        if constexpr (!CODES && !(SPLIT && LKC)) sp.init(t.P, p0, t.P.extent, wv, lane);
        sl.init(t.L, l0, nl, wv, lane);
        TileFragment<PKC, BP, BK> fp;
        TileFragment<LKC, BL, BK> fl;
        fp.init(wp * FP * 32, lane);
        fl.init(wl * FL * 32, lane);

        const int per = (K + BK - 1) / BK, all = SPLIT ? per : per * t.n_pairs, share = (all + n_split - 1) / n_split;
        const int n0 = min(all, split * share), n = min(all, n0 + share) - n0;
        if (n <= 0) return;
        if constexpr (FULL) {
            run_full(t, p0, l0, K, n0, n, per, wv, sp, sl, fp, fl, lds);
        } else {
            if constexpr (SPLIT && LKC && RING > 1) run_split_ahead(t, p0, l0, K, n0, n, wv, sl, fp, fl, lds);
            else if constexpr (SPLIT) run_split(t, p0, l0, K, n0, n, wv, sp, sl, fp, fl, lds);
            else if constexpr (CODES) run_codes(t, codes, p0, l0, K, n0, n, per, wv, sl, fp, fl, lds);
            else if constexpr (STAGES == 1) run_single(t, p0, l0, K, n0, n, per, wv, sp, sl, fp, fl, lds);
            else run_ring(t, p0, l0, K, n0, n, per, wv, sp, sl, fp, fl, lds, turn);
        }
    }

    // 16 steps of the smaller tiles: as round(), with loads H .. H + COUNT - 1 of a chunk (P's first, then L's)
    template <int KK, int H, int COUNT>
    __device__ __forceinline__ void ring_round(const bf16x8 (&a)[FP], const bf16x8 (&b)[FL], bf16x8 (&an)[FP], bf16x8 (&bn)[FL],
                                               const PSGD_TLDS unsigned char* chunk, const TileFragment<PKC, BP, BK>& fp,
                                               const TileFragment<LKC, BL, BK>& fl, const SideP& sp, const SideL& sl, const typename SideP::Source& from_p,
                                               const typename SideL::Source& from_l, PSGD_TLDS unsigned char* to, int wv) {
        read_ab<KK>(chunk, chunk + SideP::BYTES, fp, fl, an, bn);
        ring_loads<H, COUNT>(sp, sl, from_p, from_l, to, wv);
        __builtin_amdgcn_sched_barrier(0);
        multiply(a, b);
        __builtin_amdgcn_sched_barrier(0);
    }
    template <int H, int COUNT>
    __device__ __forceinline__ static void ring_loads(const SideP& sp, const SideL& sl, const typename SideP::Source& from_p,
                                                      const typename SideL::Source& from_l, PSGD_TLDS unsigned char* to, int wv) {
        if constexpr (COUNT > 0) {
            if constexpr (H < SideP::LOADS) sp.template load<H>(from_p, to, wv);
            else if constexpr (H < LOADS) sl.template load<H - SideP::LOADS>(from_l, to + SideP::BYTES, wv);
            ring_loads<H + 1, COUNT - 1>(sp, sl, from_p, from_l, to, wv);
        }
    }

    // The smaller tiles: a ring of chunks, of which all but the one being read are loaded or on their way (with one workgroup per compute
    // unit the loads' latency is what counts).  Fragments, barrier and what lies past the end as in run_full.
    __device__ __forceinline__ void run_ring(const TileArgs& t, int p0, int l0, int K, int n0, int n, int per, int wv, const SideP& sp,
                                             const SideL& sl, const TileFragment<PKC, BP, BK>& fp, const TileFragment<LKC, BL, BK>& fl,
                                             PSGD_TLDS unsigned char* lds, int turn) {
        int left = n, pair = n0 / per, kc = n0 - pair * per + turn, into = 0, from = 0;     // of the next chunk to load
        typename SideP::Source from_p;
        typename SideL::Source from_l;
        auto next = [&]() {         // its place
            const unsigned which = t.pairs >> (4 * pair);
            from_p = SideP::source(t.P, which & 3, p0, kc * BK, K, left > 0);
            from_l = SideL::source(t.L, (which >> 2) & 3, l0, kc * BK, K, left > 0);
            PSGD_TLDS unsigned char* const to = lds + into * STAGE_BYTES;
            --left;
            const bool wrap = ++kc == per;
            kc = wrap ? 0 : kc;
            pair = min(pair + (wrap ? 1 : 0), 7);
            into = into + 1 == STAGES ? 0 : into + 1;
            return to;
        };
        constexpr int THIRD = (LOADS + 2) / 3;
        PSGD_TLDS unsigned char* to = nullptr;
        for (int i = 0; i < STAGES - 1; ++i) {
            to = next();
            ring_loads<0, LOADS>(sp, sl, from_p, from_l, to, wv);
        }
        to = next();
        ring_loads<0, THIRD>(sp, sl, from_p, from_l, to, wv);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 2) * LOADS + THIRD) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        bf16x8 a0[FP], b0[FL], a1[FP], b1[FL];
        read_ab<0>(lds, lds + SideP::BYTES, fp, fl, a0, b0);
        for (int it = 0; it < n; ++it) {
            const PSGD_TLDS unsigned char* chunk = lds + from * STAGE_BYTES;
            from = from + 1 == STAGES ? 0 : from + 1;
            ring_round<1, THIRD, THIRD>(a0, b0, a1, b1, chunk, fp, fl, sp, sl, from_p, from_l, to, wv);
            ring_round<2, 2 * THIRD, LOADS - 2 * THIRD>(a1, b1, a0, b0, chunk, fp, fl, sp, sl, from_p, from_l, to, wv);
            ring_round<3, 0, 0>(a0, b0, a1, b1, chunk, fp, fl, sp, sl, from_p, from_l, to, wv);
            // the next chunk has arrived, for every wave, and nobody reads this one's place any more: it is the next to be loaded
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STAGES - 2) * LOADS) : "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            to = next();
            ring_round<0, 0, THIRD>(a1, b1, a0, b0, lds + from * STAGE_BYTES, fp, fl, sp, sl, from_p, from_l, to, wv);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    }

    // One chunk in LDS: nothing of this workgroup goes on while it loads; the others of the compute unit do.
    __device__ __forceinline__ void run_single(const TileArgs& t, int p0, int l0, int K, int n0, int n, int per, int wv, SideP& sp,
                                               const SideL& sl, const TileFragment<PKC, BP, BK>& fp, const TileFragment<LKC, BL, BK>& fl,
                                               PSGD_TLDS unsigned char* lds) {
        int pair = n0 / per, kc = n0 - pair * per;
        for (int it = 0; it < n; ++it) {
            const unsigned which = t.pairs >> (4 * pair);
            const auto from_p = SideP::source(t.P, which & 3, p0, kc * BK, K, true);
            sl.load_all(SideL::source(t.L, (which >> 2) & 3, l0, kc * BK, K, true), lds + SideP::BYTES, wv);
            if constexpr (!PKC && !LKC) {
                if (t.steps) sp.load_counted(from_p, lds, wv, lane, t.steps, kc * BK);
                else sp.load_all(from_p, lds, wv);
            } else {
                sp.load_all(from_p, lds, wv);
            }
            if (++kc == per) { kc = 0; ++pair; }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            multiply_chunk(lds, fp, fl);
        }
    }

    // The same with P from an 8-bit checkpoint: a thread has 32 codes of a row, a group, at a time and writes their values to LDS where the direct loads would have
    // put them (16-byte pieces in an order that spreads four rows over the banks).  The next chunk's codes are loaded beside this one's part of L, with one wait
    // for both: a latency less per chunk, though none of it runs beside the products.
    __device__ __forceinline__ void run_codes(const TileArgs& t, const TileCodes& codes, int p0, int l0, int K, int n0, int n, int per, int wv, const SideL& sl,
                                              const TileFragment<PKC, BP, BK>& fp, const TileFragment<LKC, BL, BK>& fl, PSGD_TLDS unsigned char* lds) {
        static_assert(!PKC && BP == 128 && kTileThreads == 256, "32 codes per thread and chunk");
        const int row = threadIdx.x >> 2, col = p0 + 32 * (threadIdx.x & 3);
        PSGD_TLDS unsigned char* const to = lds + row * 2 * BP + (((threadIdx.x & 3) ^ SideP::turn(row)) << 6);
        uintx2 w[4];            // pieces of eight codes, in the order in which they are written
        float scale;
        auto fetch = [&](int k0) {
            const int k = k0 + row;
            const bool in = k < K && col < t.P.extent;
            const PSGD_GLOBAL signed char* const at = as_global(codes.codes) + (int64_t)k * codes.ldc + col;
            scale = 0.f;
            if (in) scale = __uint_as_float((unsigned)as_global(codes.scales)[k * (int64_t)codes.groups + (col >> 5)] << 23);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int piece = 8 * (j ^ (row & 3));
                w[j] = uintx2{0u, 0u};
                if (in && col + piece < t.P.extent) w[j] = *reinterpret_cast<const PSGD_GLOBAL uintx2*>(at + piece);
            }
        };
        int pair = n0 / per, kc = n0 - pair * per;
        fetch(kc * BK);
        for (int it = 0; it < n; ++it) {
            const unsigned which = t.pairs >> (4 * pair);
            sl.load_all(SideL::source(t.L, (which >> 2) & 3, l0, kc * BK, K, true), lds + SideP::BYTES, wv);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float v[8];
                values(ActCodes<2>{{w[j][0], w[j][1]}, scale}, v);
                bf16x8 piece;
#pragma unroll
                for (int u = 0; u < 8; ++u) piece[u] = (bf16_t)v[u];
                *reinterpret_cast<PSGD_TLDS bf16x8*>(to + 16 * (j ^ (row & 3))) = piece;
            }
            if (++kc == per) { kc = 0; ++pair; }
            if (it + 1 < n) fetch(kc * BK);
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            multiply_chunk(lds, fp, fl);
        }
    }
    // fp32 operands.  All three planes of a chunk of both sides are in LDS, and six products are made of each pair of chunks: a plane is loaded once, not
    // once per product, which is what bounds fp32 products that stream pairs of planes (1000 x 2048 x 20000, loss and gradients: 1621 us with pairs, 1264 us
    // so).  P's come from the fp32 matrix, four elements per load, split on the way (LKC): W is read as it is, where planes of it in memory cost six bytes
    // written and twelve read per element (64 x 4096 x 32000, loss alone: 636 us with them, 166 us without).  Or like L's from memory.
    static constexpr int RAW = BP * BK * 4 / (16 * kTileThreads);       // loads of a thread and chunk
    // piece i of this thread: its element and step in the chunk
    __device__ __forceinline__ static void raw_piece(int i, int wv, int lane, int& e, int& k) {
        const int block = i * NW + wv;
        if constexpr (PKC) e = block * 8 + (lane >> 3), k = 4 * (lane & 7);
        else k = block * (256 / BP) + lane / (BP / 4), e = 4 * (lane % (BP / 4));
    }
    // (Loads without a branch, out of range where there is nothing: the waits below count them.)
    __device__ __forceinline__ static void raw_fetch(const TileOperand& o, int p0, int k0, int K, int wv, int lane, floatx4 (&raw)[RAW]) {
        const float* base = reinterpret_cast<const float*>(o.ptr) + (PKC ? (int64_t)p0 * o.ld + k0 : (int64_t)k0 * o.ld + p0);
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(base), 0, (int)kOutside, 0x00020000);
#pragma unroll
        for (int i = 0; i < RAW; ++i) {
            int e, k;
            raw_piece(i, wv, lane, e, k);
            const unsigned at = (unsigned)((PKC ? e * o.ld + k : k * o.ld + e) * 4);
            raw[i] = __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(p0 + e < o.extent && k0 + k < K ? at : kOutside), 0, 0));
        }
    }
    __device__ __forceinline__ static void raw_store(const floatx4 (&raw)[RAW], int k0, int K, int wv, int lane, PSGD_TLDS unsigned char* lds) {
#pragma unroll
        for (int i = 0; i < RAW; ++i) {
            int e, k;
            raw_piece(i, wv, lane, e, k);
            bf16x4 plane[kMaxPlanes];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                bf16_t q[kMaxPlanes];
                split_planes<kMaxPlanes>(!PKC || k0 + k + u < K ? raw[i][u] : 0.f, q);      // (K may end inside a piece)
#pragma unroll
                for (int h = 0; h < kMaxPlanes; ++h) plane[h][u] = q[h];
            }
            const unsigned to = PKC ? (unsigned)(e * 2 * BK + (((k >> 3) ^ SideP::swizzle(e)) << 4) + 2 * (k & 4))
                                    : (unsigned)(k * 2 * BP + ((2 * e) ^ (SideP::turn(k) << 6)));
#pragma unroll
            for (int h = 0; h < kMaxPlanes; ++h) *reinterpret_cast<PSGD_TLDS bf16x4*>(lds + h * SideP::BYTES + to) = plane[h];
        }
    }
    __device__ __forceinline__ static void fence() { asm volatile("" ::: "memory"); }

    __device__ __forceinline__ void run_split(const TileArgs& t, int p0, int l0, int K, int n0, int n, int wv, const SideP& sp, const SideL& sl,
                                              const TileFragment<PKC, BP, BK>& fp, const TileFragment<LKC, BL, BK>& fl, PSGD_TLDS unsigned char* lds) {
        PSGD_TLDS unsigned char* const lds_l = lds + kMaxPlanes * SideP::BYTES;
        floatx4 raw[RAW];
        if constexpr (LKC) raw_fetch(t.P, p0, n0 * BK, K, wv, lane, raw);
        for (int kc = n0; kc < n0 + n; ++kc) {
#pragma unroll
            for (int q = 0; q < kMaxPlanes; ++q) {
                sl.load_all(SideL::source(t.L, q, l0, kc * BK, K, true), lds_l + q * SideL::BYTES, wv);
                if constexpr (!LKC) sp.load_all(SideP::source(t.P, q, p0, kc * BK, K, true), lds + q * SideP::BYTES, wv);
            }
            if constexpr (LKC) raw_store(raw, kc * BK, K, wv, lane, lds);
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            fence();
            if constexpr (LKC) raw_fetch(t.P, p0, (kc + 1) * BK, K, wv, lane, raw);
            split_step<0>(lds, lds_l, fp, fl);
            split_step<1>(lds, lds_l, fp, fl);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();       // every wave is done with the chunk
            fence();
        }
    }

    // the same with the loads of RING chunks ahead, for few workgroups
    __device__ __forceinline__ void run_split_ahead(const TileArgs& t, int p0, int l0, int K, int n0, int n, int wv, const SideL& sl,
                                                    const TileFragment<PKC, BP, BK>& fp, const TileFragment<LKC, BL, BK>& fl, PSGD_TLDS unsigned char* lds) {
        PSGD_TLDS unsigned char* const lds_l = lds + kMaxPlanes * SideP::BYTES;
        const int end = n0 + n;
        floatx4 raw[RING][RAW];
        auto load_l = [&](int kc) {
            fence();
#pragma unroll
            for (int q = 0; q < kMaxPlanes; ++q)
                sl.load_all(SideL::source(t.L, q, l0, kc * BK, K, kc < end), lds_l + ((kc - n0) % RING * kMaxPlanes + q) * SideL::BYTES, wv);
            fence();
        };
        raw_fetch(t.P, p0, n0 * BK, K, wv, lane, raw[0]);
#pragma unroll
        for (int i = 1; i < RING; ++i) {
            load_l(n0 + i - 1);
            raw_fetch(t.P, p0, (n0 + i) * BK, n0 + i < end ? K : 0, wv, lane, raw[i]);
        }
        for (int k4 = n0; k4 < end; k4 += RING)
#pragma unroll
            for (int i = 0; i < RING; ++i) {
                const int kc = k4 + i;
                if (kc >= end) break;
                raw_store(raw[i], kc * BK, K, wv, lane, lds);
                load_l(kc + RING - 1);
                raw_fetch(t.P, p0, (kc + RING) * BK, kc + RING < end ? K : 0, wv, lane, raw[i]);
                // all that was loaded after this chunk of L may be on its way
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(RING * RAW + (RING - 1) * kMaxPlanes * SideL::LOADS) : "memory");
                __builtin_amdgcn_s_barrier();
                fence();
                const PSGD_TLDS unsigned char* const from = lds_l + i * kMaxPlanes * SideL::BYTES;
                split_step<0>(lds, from, fp, fl);
                split_step<1>(lds, from, fp, fl);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();       // every wave is done with the chunk
                fence();
            }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // (LDS is the epilogue's next)
        __builtin_amdgcn_s_barrier();
        fence();
    }
    template <int KK>
    __device__ __forceinline__ void split_step(const PSGD_TLDS unsigned char* lds, const PSGD_TLDS unsigned char* lds_l, const TileFragment<PKC, BP, BK>& fp,
                                               const TileFragment<LKC, BL, BK>& fl) {
        bf16x8 a[kMaxPlanes][FP], b[kMaxPlanes][FL];
#pragma unroll
        for (int q = 0; q < kMaxPlanes; ++q) read_ab<KK>(lds + q * SideP::BYTES, lds_l + q * SideL::BYTES, fp, fl, a[q], b[q]);
        // smallest products first
#pragma unroll
        for (int sum = kMaxPlanes - 1; sum >= 0; --sum)
#pragma unroll
            for (int q = sum; q >= 0; --q) multiply(a[q], b[sum - q]);
    }

    // a chunk that is in LDS; the barrier says that every wave is done with it
    __device__ __forceinline__ void multiply_chunk(const PSGD_TLDS unsigned char* lds, const TileFragment<PKC, BP, BK>& fp, const TileFragment<LKC, BL, BK>& fl) {
        bf16x8 a0[FP], b0[FL], a1[FP], b1[FL];
        read_ab<0>(lds, lds + SideP::BYTES, fp, fl, a0, b0);
        read_ab<1>(lds, lds + SideP::BYTES, fp, fl, a1, b1);
        multiply(a0, b0);
        read_ab<2>(lds, lds + SideP::BYTES, fp, fl, a0, b0);
        multiply(a1, b1);
        read_ab<3>(lds, lds + SideP::BYTES, fp, fl, a1, b1);
        multiply(a0, b0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        multiply(a1, b1);
    }

    // row of C and first of the four columns of quad q (0..3) of fragment (i, j), relative to the tile; values acc[i][j][4 q ..]
    __device__ int row(int j) const { return (wl * FL + j) * 32 + (lane & 31); }
    __device__ int col(int i, int q) const { return (wp * FP + i) * 32 + 8 * q + 4 * (lane >> 5); }

    // Calls put(row, col, values[N]) for every N consecutive elements (N = 4 or 8) of the tile, rows of 32 FP elements of a wave after each
    // other, so that a wavefront's stores are whole lines.  From the accumulators, where a lane has four elements of a row and the lanes
    // next to it other rows, through LDS, 32 rows at a time, each wave in a place of its own.  (Stored from the accumulators, 16 or 32 bytes
    // of a line at a time, C takes 1.3 TB/s in fp32 and 0.9 in bf16.)
    template <int N, class F>
    __device__ __forceinline__ void for_rows(PSGD_TLDS unsigned char* lds, F put) {
        constexpr int COLS = 32 * FP, LD = COLS + 4;        // the 16 bytes spread 16 rows over all banks
        static_assert(NW * 32 * LD * 4 <= LDS_BYTES, "places");
        constexpr int PER = COLS / N, ROWS = 64 / PER;      // lanes per row, rows per store
        __syncthreads();
        PSGD_TLDS float* mine = reinterpret_cast<PSGD_TLDS float*>(lds) + (wl * WP + wp) * 32 * LD;
#pragma unroll
        for (int j = 0; j < FL; ++j) {
#pragma unroll
            for (int i = 0; i < FP; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<PSGD_TLDS floatx4*>(mine + (lane & 31) * LD + 32 * i + 8 * q + 4 * (lane >> 5)) =
                        floatx4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            __builtin_amdgcn_wave_barrier();
#pragma unroll 4
            for (int r = 0; r < 32; r += ROWS) {
                const int row = r + lane / PER, col = N * (lane % PER);
                float v[N];
#pragma unroll
                for (int u = 0; u < N; u += 4) {
                    const floatx4 x = *reinterpret_cast<const PSGD_TLDS floatx4*>(mine + row * LD + col + u);
#pragma unroll
                    for (int w = 0; w < 4; ++w) v[u + w] = x[w];
                }
                put((wl * FL + j) * 32 + row, wp * COLS + col, v);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
};

}  // namespace psgd
