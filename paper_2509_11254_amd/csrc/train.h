// Host side of the training operators: the matrix products on tiles (tile.hip), 8-bit checkpoints (act.hip), the output
// head's loss (head.hip).
#pragma once
#include "psgd_dev.h"
#include "../../include/psgd.h"

namespace psgd {

constexpr int kTileK = 64;      // contraction steps per chunk
constexpr int kTileThreads = 256;

// Elements of a tile of C along P and L.  256 x 256, 128 x 128 (few tiles: one workgroup per compute unit, deep in loads) and 128 x 64 (few
// rows) have a compute unit's LDS for themselves; of TILE_MANY, 128 x 128 with one chunk in LDS, a compute unit takes four, which hide each
// other's loads and stores.  TILE_SPLIT, 128 x 128, and TILE_SPLIT_THIN, 64 x 64 (few tiles), multiply fp32 operands, whose three bf16 planes are in LDS side
// by side; a compute unit takes three of them.
enum TileShape { TILE_256 = 0, TILE_128 = 1, TILE_THIN = 2, TILE_MANY = 3, TILE_SPLIT = 4, TILE_SPLIT_THIN = 5 };
constexpr bool tile_is_split(TileShape s) { return s == TILE_SPLIT || s == TILE_SPLIT_THIN; }
constexpr int tile_p(TileShape s) { return s == TILE_256 ? 256 : s == TILE_SPLIT_THIN ? 64 : 128; }
constexpr int tile_l(TileShape s) { return s == TILE_256 ? 256 : s == TILE_THIN || s == TILE_SPLIT_THIN ? 64 : 128; }
constexpr int tile_k(TileShape s) { return tile_is_split(s) ? 32 : kTileK; }

// Whether tokens count, a bit each.  Nullable: all do
typedef const uint64_t* TileTokens;

struct TileOperand {
    const bf16_t* ptr;
    int64_t ld;         // elements, multiple of 8
    int64_t plane;      // elements between planes
    int extent;         // rows or columns of C that it covers
};

// (TILE_SPLIT shapes: three planes of each side and the six products of two whose places add up to at most two.  Where L is K-contiguous P is the fp32
// matrix itself, cast, and `ld` counts its elements.)
// What every kernel on tiles gets.  An operand may have several bf16 planes whose sum it is; `pairs` lists the products of planes to
// add up, smallest first, four bits each: P's plane in the lower two, L's in the upper two.
struct TileArgs {
    TileOperand P, L;
    int K;
    const int* count;   // nullable: device word, tokens that count; of them this call takes those from `first` on, at most K or L.extent ...
    int first;
    int count_is_k;     // ... as contraction steps (1) or as rows of C (0)
    TileTokens steps;   // contraction steps that do not count bring zeros from P (TILE_MANY, both K-strided)
    unsigned pairs;
    int n_pairs;
    int n_split;        // parts of the contraction, each a workgroup of its own; more where fewer rows count (tile_grid)
    int blocks;         // workgroups of the launch (set by it)
};
constexpr unsigned kPairs1 = 0x0, kPairsL3 = 0x048;

// An 8-bit checkpoint in the place of P, K-strided: codes [K][ldc], scales [K][groups]
struct TileCodes {
    const signed char* codes;
    int64_t ldc;
    const unsigned char* scales;
    int groups;
};

// Where a product goes: C row l to row `rows[first + l]` (or l), columns as they are
struct TileOut {
    void* ptr;
    int64_t ld;
    int dtype;          // PSGD_F32 or PSGD_BF16
    int accumulate;     // add to what is there
    int skip_empty;     // write nothing where no token counts (a later piece of an accumulated product)
    const int* rows;    // nullable
    TileTokens tokens;  // rows of C that do not count come out as zeros
    const float* scale; // nullable: device word that C is multiplied by
    float* part;        // n_split > 1: partial sums [split][rows of C that count][part_ld]
    int64_t part_ld;
};

// shape and number of parts of the contraction of a product: extents of C, chunks of the contraction (of all pairs of planes)
struct TilePlan { TileShape shape; int n_split; bool from_codes; double us; };     // us: the estimate it was chosen by
// restore: microseconds that P's values take to get from an 8-bit checkpoint to memory first (0: P is no checkpoint); from_codes: do without
// only_many: TILE_MANY or nothing
TilePlan tile_plan(int64_t extent_p, int64_t extent_l, int64_t chunks, bool may_split, double restore, bool only_many = false);
// the same for fp32 operands; chunks: of one plane
TilePlan split_plan(int64_t extent_p, int64_t extent_l, int64_t chunks, bool may_split);
size_t tile_part_bytes(int64_t extent_p, int64_t extent_l, const TilePlan& plan);
// C = L P^T over the operands' orientations: P K-strided, L K-contiguous or K-strided
hipError_t launch_product(bool l_contiguous, TileShape shape, const TileArgs& t, const TileOut& o, hipStream_t st);
// two products of TILE_MANY in one launch: the first's L K-contiguous, the second's K-strided; whether that is faster than a and b each in its own
// launch, or a_alone and b
struct TilePair { TilePlan plan; int64_t extent_p, extent_l, tiles, chunks; };
bool pair_pays(const TilePair& a, const TilePair& b, const TilePlan& a_alone);
hipError_t launch_pair(const TileArgs& ta, const TileOut& oa, const TileArgs& tb, const TileOut& ob, hipStream_t st);
// the same from a checkpoint: L K-strided, TILE_MANY
hipError_t launch_code_product(const TileCodes& codes, const TileArgs& t, const TileOut& o, hipStream_t st);
// rows x cols (ld) of fp32 or bf16 to `planes` bf16 planes [rows][round_up(cols, 8)], zeros beyond cols
hipError_t launch_planes(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, bf16_t* dst, int planes, hipStream_t st);

// Whether a launch succeeded is asked of hipGetLastError(), which keeps what any earlier call of the program left: each entry point begins without it.
inline void forget_errors() { (void)hipGetLastError(); }
inline int64_t up8(int64_t x) { return (x + 7) & ~(int64_t)7; }
inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool bad_dtype(int t) { return t != PSGD_F32 && t != PSGD_BF16; }
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline bool bad_ld(int64_t ld, int64_t cols) { return ld < cols || (ld & 7) != 0; }
constexpr int64_t kMaxLd = 1 << 22;     // 255 rows * ld * 2 bytes stay within a buffer descriptor's range
constexpr int64_t kMaxExtent = 1 << 30;

}  // namespace psgd
