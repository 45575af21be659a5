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
    static_assert(N == 8, "pieces");
    if (n >= 8) {
        PSGD_GLOBAL bf16x8* q = reinterpret_cast<PSGD_GLOBAL bf16x8*>(p);
        bf16x8 o, b;
        if (add) b = *q;
#pragma unroll
        for (int u = 0; u < 8; ++u) o[u] = (bf16_t)(add ? v[u] + (float)b[u] : v[u]);
        *q = o;
    } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (u < n) p[u] = (bf16_t)(add ? (float)p[u] + v[u] : v[u]);
    }
}

// what a product kernel writes
enum TileKind { TILE_PART = 0, TILE_F32 = 1, TILE_BF16 = 2 };

template <bool PKC, bool LKC, int BL, int KIND>
__global__ __launch_bounds__(tile_threads<BL>(), BL == 256 ? 1 : 2) void product_kernel(TileArgs t, TileOut o, int n_p, int n_l) {
    extern __shared__ __align__(16) unsigned char smem[];
    using T = Tile<PKC, LKC, BL>;
    const TilePlace at = tile_place(blockIdx.x, n_p, n_l, t.n_split);
    const int p0 = at.p * kTileP, l0 = at.l * BL;
    const int K = t.count_is_k ? counted(t, t.K) : t.K, nl = t.count_is_k ? t.L.extent : counted(t, t.L.extent);
    if (l0 >= nl || (K == 0 && o.skip_empty)) return;
    T tile;
    tile.run(t, p0, l0, nl, K, at.split, (PSGD_TLDS unsigned char*)smem);
    tile.template for_rows<KIND == TILE_BF16 ? 8 : 4>((PSGD_TLDS unsigned char*)smem, [&](int row, int col, const auto& v) {
        const int l = l0 + row, c = p0 + col, n = t.P.extent - c;
        if (l >= nl || n <= 0) return;
        if constexpr (KIND == TILE_PART) {
            PSGD_GLOBAL float* p = as_global(o.part) + ((int64_t)at.split * t.L.extent + l) * o.part_ld + c;
            *reinterpret_cast<PSGD_GLOBAL floatx4*>(p) = floatx4{v[0], v[1], v[2], v[3]};
        } else {
            const int64_t to = (o.rows ? o.rows[t.first + l] : l) * o.ld + c;
            if constexpr (KIND == TILE_F32) store_row(as_global((float*)o.ptr) + to, v, n, o.accumulate);
            else store_row(as_global((bf16_t*)o.ptr) + to, v, n, o.accumulate);
        }
    });
}

// sum over the splits, in their order, of eight elements per thread
__global__ __launch_bounds__(kThreads) void split_sum_kernel(TileArgs t, TileOut o) {
    const int K = t.count_is_k ? counted(t, t.K) : t.K, nl = t.count_is_k ? t.L.extent : counted(t, t.L.extent);
    if (K == 0 && o.skip_empty) return;
    const int pieces = (t.P.extent + 7) / 8;
    const int64_t all = (int64_t)nl * pieces, layer = (int64_t)t.L.extent * o.part_ld;
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < all; e += (int64_t)gridDim.x * kThreads) {
        const int l = (int)(e / pieces), c = 8 * (int)(e - (int64_t)l * pieces);
        const PSGD_GLOBAL float* p = as_global(o.part) + l * o.part_ld + c;
        floatx4 s = {0.f, 0.f, 0.f, 0.f}, r = s;
        for (int k = 0; k < t.n_split; ++k) {
            s += *reinterpret_cast<const PSGD_GLOBAL floatx4*>(p + k * layer);
            r += *reinterpret_cast<const PSGD_GLOBAL floatx4*>(p + k * layer + 4);
        }
        const float v[8] = {s[0], s[1], s[2], s[3], r[0], r[1], r[2], r[3]};
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

constexpr int kUnits = 256;     // compute units; one workgroup of a 256-row tile fills one

int tile_rows(int64_t extent_l) { return extent_l <= 64 ? 64 : extent_l <= 128 ? 128 : 256; }

int tile_splits(int64_t n_p, int64_t n_l, int64_t chunks, int64_t elems) {
    (void)elems;
    const int64_t tiles = n_p * n_l;
    if (tiles >= kUnits || tiles == 0) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>({kUnits / tiles, chunks / 4, 64}));
}

size_t tile_part_bytes(int extent_p, int extent_l, int n_split) {
    return n_split > 1 ? up256((size_t)n_split * extent_l * ((extent_p + 7) / 8 * 8) * sizeof(float)) : 0;
}

template <bool PKC, bool LKC, int BL, int KIND>
static hipError_t launch_kind(const TileArgs& t, const TileOut& o, int n_p, int n_l, hipStream_t st) {
    auto kfn = product_kernel<PKC, LKC, BL, KIND>;
    constexpr int lds = Tile<PKC, LKC, BL>::LDS_BYTES;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kfn), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kfn, dim3(n_p * n_l * t.n_split), dim3(tile_threads<BL>()), lds, st, t, o, n_p, n_l);
    return hipGetLastError();
}
template <bool PKC, bool LKC, int BL>
static hipError_t launch_tiles(const TileArgs& t, const TileOut& o, int n_p, int n_l, hipStream_t st) {
    if (o.part) return launch_kind<PKC, LKC, BL, TILE_PART>(t, o, n_p, n_l, st);
    if (o.dtype == PSGD_F32) return launch_kind<PKC, LKC, BL, TILE_F32>(t, o, n_p, n_l, st);
    return launch_kind<PKC, LKC, BL, TILE_BF16>(t, o, n_p, n_l, st);
}

hipError_t launch_product(bool p_contiguous, bool l_contiguous, int bl, const TileArgs& t, const TileOut& out, hipStream_t st) {
    TileOut o = out;
    if (t.n_split == 1) o.part = nullptr;
    o.part_ld = (t.P.extent + 7) / 8 * 8;
    const int n_p = (t.P.extent + kTileP - 1) / kTileP, n_l = (t.L.extent + bl - 1) / bl;
    if (n_p * (int64_t)n_l * t.n_split > INT32_MAX) return hipErrorInvalidValue;
    hipError_t e = hipErrorInvalidValue;
    if (!p_contiguous && l_contiguous) {
        if (bl == 256) e = launch_tiles<false, true, 256>(t, o, n_p, n_l, st);
        else if (bl == 128) e = launch_tiles<false, true, 128>(t, o, n_p, n_l, st);
        else if (bl == 64) e = launch_tiles<false, true, 64>(t, o, n_p, n_l, st);
    } else if (!p_contiguous && !l_contiguous && bl == 256) {
        e = launch_tiles<false, false, 256>(t, o, n_p, n_l, st);
    }
    if (e != hipSuccess || t.n_split == 1) return e;
    const int64_t pieces = (int64_t)t.L.extent * ((t.P.extent + 7) / 8);
    hipLaunchKernelGGL(split_sum_kernel, dim3((unsigned)std::min<int64_t>((pieces + kThreads - 1) / kThreads, 8 * kUnits)), dim3(kThreads), 0, st, t, o);
    return hipGetLastError();
}

hipError_t launch_planes(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, bf16_t* dst, int planes, hipStream_t st) {
    if (rows == 0) return hipSuccess;
    const dim3 grid((unsigned)std::min<int64_t>((rows * ((cols + 7) / 8) + kThreads - 1) / kThreads, 32 * kUnits));
    if (dtype == PSGD_F32) hipLaunchKernelGGL(planes_kernel<float>, grid, dim3(kThreads), 0, st, (const float*)src, rows, (int)cols, ld, dst, planes);
    else hipLaunchKernelGGL(planes_kernel<bf16_t>, grid, dim3(kThreads), 0, st, (const bf16_t*)src, rows, (int)cols, ld, dst, planes);
    return hipGetLastError();
}

}  // namespace psgd
