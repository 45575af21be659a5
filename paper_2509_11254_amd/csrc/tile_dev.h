// The matrix product on bf16 operands that the training operators share: C[l][p] = sum_k L(l, k) P(p, k), one tile of BL x 256
// elements of C per workgroup, on v_mfma_f32_32x32x16_bf16 with fp32 accumulation.
//
// An operand is stored with the contraction along its rows ("K-contiguous": [extent][K], X and W in X W^T) or down its
// columns ("K-strided": [K][extent], both operands of a weight gradient dY^T X), always row-major.  Chunks of 64 contraction
// steps go to LDS by direct loads, 16 bytes per lane, without passing through registers; the buffer descriptor's range check
// turns what lies outside the operand into zeros.  K-contiguous chunks are [extent][64], read 16 bytes (one fragment) per
// lane; K-strided chunks are [64][extent], read by the transposing LDS load, which hands a lane four steps of its column.
//
// P runs along the accumulators' registers and L along the lanes, so that a lane holds four consecutive elements of a row of C,
// and half a wavefront's 32 lanes 32 rows.
#pragma once
#include "train.h"

namespace psgd {

#define PSGD_TLDS __attribute__((address_space(3)))
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short shortx4;
typedef __attribute__((__vector_size__(8 * sizeof(short)))) short shortx8;

constexpr int kTileP = 256;             // elements of a tile of C along P
constexpr int kTileK = 64;              // contraction steps per chunk
constexpr int kTileThreads = 512;
constexpr unsigned kOutside = 0x80000000u;      // byte offset beyond every descriptor's range

__device__ inline int counted(const TileArgs& a, int upper) {
    if (!a.count) return upper;
    return max(0, min(upper, *a.count - a.first));
}

// Which tile a workgroup takes.  Consecutive workgroups go to consecutive XCDs; each XCD gets a run of consecutive tiles (its L2 then
// holds operands that its workgroups share), and a run goes through 8 tiles along L before the next along P.
struct TilePlace { int p, l, split; };
__device__ inline TilePlace tile_place(int id, int n_p, int n_l, int n_split) {
    const int n = n_p * n_l * n_split, q = n >> 3, r = n & 7, x = id & 7;
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

// One operand's side of a tile: E elements of C wide, waves NW.
template <bool KC, int E, int NW>
struct TileSide {
    static constexpr int LOADS = E * kTileK * 2 / (NW * 1024);      // direct loads of 1 KB per wave and chunk
    static constexpr int BYTES = E * kTileK * 2;
    static_assert(LOADS >= 1 && LOADS * NW * 1024 == BYTES, "chunk");

    // K-contiguous: 8 rows of 128 bytes per load, piece c of row r at place c ^ ((r >> 1) & 7): 16 rows' reads of one piece
    // cover all 64 banks.  K-strided: rows of 2 E bytes, 64-byte piece c of row k at place c ^ (k & 3): the four rows that a
    // transposing read takes lie in different banks.
    unsigned off[LOADS];
    int kpiece;          // K-contiguous: first step of this lane's pieces, K-strided: unused

    __device__ void init(const TileOperand& o, int start, int extent, int wv, int lane) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int block = i * NW + wv;
            if constexpr (KC) {
                const int row = block * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
                kpiece = 8 * piece;      // the same for all i: blocks are 8 rows apart by NW
                off[i] = start + row < extent ? (unsigned)(((int64_t)row * o.ld + 8 * piece) * 2) : kOutside;
            } else {
                constexpr int LANES = E / 8, ROWS = 64 / LANES;     // lanes per row, rows per load
                const int k = block * ROWS + lane / LANES, place = lane % LANES, col = 8 * (place ^ ((k & 3) << 2));
                off[i] = start + col < extent ? (unsigned)(((int64_t)k * o.ld + col) * 2) : kOutside;
            }
        }
    }

    // chunk from step k0 on of K to LDS
    __device__ void load(const TileOperand& o, int plane, int start, int k0, int K, PSGD_TLDS unsigned char* dst, int wv) const {
        const bf16_t* base = o.ptr + plane * o.plane + (KC ? (int64_t)start * o.ld + k0 : (int64_t)k0 * o.ld + start);
        const int64_t left = KC ? (int64_t)kOutside : (int64_t)(K - k0) * o.ld * 2 - 2 * start;
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)(unsigned)min(left, (int64_t)kOutside), 0x00020000);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const unsigned v = KC && kpiece >= K - k0 ? kOutside : off[i];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (PSGD_TLDS void*)(dst + (i * NW + wv) * 1024), 16, (int)v, 0, 0, 0);
        }
    }
};

// fragment of 32 elements from e0 on (a multiple of 32), steps 16 kk .. + 15 of the chunk: lane li + 32 lg gets steps 8 lg .. + 7 of element li
template <bool KC, int E>
struct TileFragment {
    unsigned base[4];   // K-contiguous: by kk.  K-strided: by fragment (up to 4 of a wave)
    __device__ void init(int e0, int lane) {
        const int li = lane & 31, lg = lane >> 5;
        if constexpr (KC) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) base[kk] = (unsigned)((e0 + li) * 128 + (((2 * kk + lg) ^ ((li >> 1) & 7)) << 4));
        } else {
            const int row = 8 * lg + ((lane & 15) >> 2);
#pragma unroll
            for (int f = 0; f < 4; ++f)
                base[f] = (unsigned)(row * 2 * E + (((2 * (e0 + 32 * f)) ^ ((row & 3) << 6)) + 32 * ((lane >> 4) & 1) + 8 * (lane & 3)));
        }
    }
    template <int KK, int F>
    __device__ bf16x8 read(const PSGD_TLDS unsigned char* chunk) const {
        if constexpr (KC) {
            return *reinterpret_cast<const PSGD_TLDS bf16x8*>(chunk + base[KK] + F * 32 * 128);
        } else {
            const PSGD_TLDS unsigned char* at = chunk + base[F] + KK * 16 * 2 * E;
            const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PSGD_TLDS shortx4*)at);
            const shortx4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PSGD_TLDS shortx4*)(at + 4 * 2 * E));
            const shortx8 v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(bf16x8, v);
        }
    }
};

// shapes: waves along P and L, chunks in LDS
template <int BL> struct TileShape;
template <> struct TileShape<256> { static constexpr int WP = 2, WL = 4, STAGES = 2; };
template <> struct TileShape<128> { static constexpr int WP = 4, WL = 2, STAGES = 3; };
template <> struct TileShape<64> { static constexpr int WP = 4, WL = 2, STAGES = 3; };

template <bool PKC, bool LKC, int BL>
struct Tile {
    using S = TileShape<BL>;
    static constexpr int WP = S::WP, WL = S::WL, NW = WP * WL, STAGES = S::STAGES;
    static constexpr int FP = kTileP / WP / 32, FL = BL / WL / 32;      // fragments per wave
    using SideP = TileSide<PKC, kTileP, NW>;
    using SideL = TileSide<LKC, BL, NW>;
    static constexpr int STAGE_BYTES = SideP::BYTES + SideL::BYTES;
    static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
    static constexpr int LOADS = SideP::LOADS + SideL::LOADS;
    static constexpr int THREADS = NW * 64;
    static_assert(FP >= 1 && FL >= 1 && FP <= 4 && FL <= 4 && THREADS == kTileThreads, "waves");

    floatx16 acc[FP][FL];
    int wp, wl, lane;

    template <int KK>
    __device__ void step(const PSGD_TLDS unsigned char* chunk, const TileFragment<PKC, kTileP>& fp, const TileFragment<LKC, BL>& fl) {
        bf16x8 a[FP], b[FL];
        a[0] = fp.template read<KK, 0>(chunk);
        if constexpr (FP > 1) a[1] = fp.template read<KK, 1>(chunk);
        if constexpr (FP > 2) a[2] = fp.template read<KK, 2>(chunk);
        if constexpr (FP > 3) a[3] = fp.template read<KK, 3>(chunk);
        b[0] = fl.template read<KK, 0>(chunk + SideP::BYTES);
        if constexpr (FL > 1) b[1] = fl.template read<KK, 1>(chunk + SideP::BYTES);
        if constexpr (FL > 2) b[2] = fl.template read<KK, 2>(chunk + SideP::BYTES);
        if constexpr (FL > 3) b[3] = fl.template read<KK, 3>(chunk + SideP::BYTES);
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int j = 0; j < FL; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
    }

    // acc = the tile at (p0, l0), part `split` of the contraction over K steps; nl: rows of C there are
    __device__ void run(const TileArgs& t, int p0, int l0, int nl, int K, int split, PSGD_TLDS unsigned char* lds) {
        lane = threadIdx.x & 63;
        const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wp = wv % WP;
        wl = wv / WP;
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int j = 0; j < FL; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
        SideP sp;
        SideL sl;
        sp.init(t.P, p0, t.P.extent, wv, lane);
        sl.init(t.L, l0, nl, wv, lane);
        TileFragment<PKC, kTileP> fp;
        TileFragment<LKC, BL> fl;
        fp.init(wp * FP * 32, lane);
        fl.init(wl * FL * 32, lane);

        const int per = (K + kTileK - 1) / kTileK, all = per * t.n_pairs, share = (all + t.n_split - 1) / t.n_split;
        const int n0 = min(all, split * share), n = min(all, n0 + share) - n0;
        if (n <= 0) return;
        int pair = n0 / per, kc = n0 - pair * per;      // of the next chunk to load
        int into = 0;
        auto issue = [&]() {
            const unsigned which = t.pairs >> (4 * pair);
            PSGD_TLDS unsigned char* dst = lds + into * STAGE_BYTES;
            sp.load(t.P, which & 3, p0, kc * kTileK, K, dst, wv);
            sl.load(t.L, (which >> 2) & 3, l0, kc * kTileK, K, dst + SideP::BYTES, wv);
            asm volatile("" ::: "memory");
            if (++kc == per) { kc = 0; ++pair; }
            into = into + 1 == STAGES ? 0 : into + 1;
        };
        int issued = 0;
        for (; issued < STAGES - 1 && issued < n; ++issued) issue();
        int from = 0;
        for (int it = 0; it < n; ++it) {
            // this chunk has arrived, for every wave, and nobody reads the buffer of the one before any more
            if (STAGES == 3 && it + 1 < n) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LOADS) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (issued < n) { issue(); ++issued; }
            const PSGD_TLDS unsigned char* chunk = lds + from * STAGE_BYTES;
            step<0>(chunk, fp, fl);
            step<1>(chunk, fp, fl);
            step<2>(chunk, fp, fl);
            step<3>(chunk, fp, fl);
            from = from + 1 == STAGES ? 0 : from + 1;
        }
    }

    // row of C and first of the four columns of quad q (0..3) of fragment (i, j), relative to the tile; values acc[i][j][4 q ..]
    __device__ int row(int j) const { return (wl * FL + j) * 32 + (lane & 31); }
    __device__ int col(int i, int q) const { return (wp * FP + i) * 32 + 8 * q + 4 * (lane >> 5); }
};

}  // namespace psgd
