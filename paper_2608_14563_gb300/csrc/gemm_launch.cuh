// gemm_launch.cuh -- host side of the tcgen05 GEMMs, shared by their translation units:
// tensor maps, problem shapes, launches of the single-CTA and the pair kernel, the split of
// the last partial wave along K and the sums of its parts.
//
// Tensor maps are encoded per call (a few microseconds of host work) through
// the driver entry point of cuTensorMapEncodeTiled, so the library does not
// link libcuda directly.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <mutex>

#include "internal.h"
#include "tc_gemm.cuh"
#include "tc_gemm_pair.cuh"

namespace fpo {

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                   const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                   const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                             &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

// 2-D tensor [outer, inner] of bf16 (esz 2) or fp32 (esz 4) with row stride
// `ld` elements, box {box_inner, box_outer}, 128-byte swizzle, zero fill
// outside the tensor on loads (and clipping on stores).  L2 promotion of 128 bytes:
// one box row; 256-byte promotion fetched 15-55% more from DRAM in the step's GEMMs
// for the same time.
inline bool make_map(CUtensorMap* m, const void* base, uint64_t inner, uint64_t outer, uint64_t ld,
              uint32_t box_inner, uint32_t box_outer, int esz = 2) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {inner, outer};
    cuuint64_t strides[1] = {ld * static_cast<uint64_t>(esz)};
    cuuint32_t box[2] = {box_inner, box_outer};
    cuuint32_t es[2] = {1, 1};
    const CUtensorMapDataType dt =
        esz == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    return fn(m, dt, 2, const_cast<void*>(base), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Output maps of the epilogues: 32 rows x 128 bytes per store.
inline bool map_out_f32(CUtensorMap* m, void* base, int rows, int cols) {
    return make_map(m, base, cols, rows, cols, 32, 32, 4);
}
inline bool map_out_bf16(CUtensorMap* m, void* base, int rows, int cols) {
    return make_map(m, base, cols, rows, cols, 64, 32, 2);
}

// K-major operand [rows, K]: box {64 (K), rows_per_tile}
inline bool map_kmajor(CUtensorMap* m, const void* base, int rows, int K, int box_rows) {
    return make_map(m, base, K, rows, K, kBK, box_rows);
}
// MN-major operand [K, mn]: box {64 (MN), 64 (K)}
inline bool map_mnmajor(CUtensorMap* m, const void* base, int K, int mn) {
    return make_map(m, base, mn, K, mn, 64, kBK);
}

inline GemmShape make_shape(int M, int N, int K, int BN, int groups, int band, int BM = kBM) {
    GemmShape sh;
    sh.M = M;
    sh.N = N;
    sh.K = K;
    sh.m_blocks = (M + BM - 1) / BM;
    sh.n_blocks = (N + BN - 1) / BN;
    sh.k_blocks = (K + kBK - 1) / kBK;
    sh.groups = groups;
    sh.band = band;
    sh.tiles = static_cast<long long>(groups) * sh.m_blocks * sh.n_blocks;
    sh.tail_tiles = 0;
    sh.tail_split = 0;
    sh.sk_scratch = nullptr;
    sh.m_dev = nullptr;
    return sh;
}

template <int BN, bool A_MN, bool B_MN, int STAGES, int MAXG, class Epi>
cudaError_t run_gemm(const GemmMaps<MAXG>& maps, const typename Epi::Params& ep,
                     const GemmShape& sh, unsigned* status, cudaStream_t st) {
    if (sh.tiles <= 0 || sh.k_blocks <= 0) return cudaSuccess;
    using L = GemmSmem<BN, STAGES>;
    constexpr auto kern = tc_gemm_kernel<BN, A_MN, B_MN, STAGES, MAXG, Epi>;
    const cudaError_t attr_err = set_smem_limit<kern>(L::kBytes);
    if (attr_err != cudaSuccess) return attr_err;
    DevInfo di;
    if (!current_device_info(&di)) return cudaErrorUnknown;
    const long long grid = sh.tiles < di.sm_count ? sh.tiles : di.sm_count;
    return launch_chained(kern, dim3(static_cast<unsigned>(grid)), gemm_threads<Epi>(), L::kBytes, st,
                          maps, ep, sh, status, wait_limit_ns());
}

// Clusters (of `cta` CTAs, the kernel's cluster size) that can be resident at once for a
// pair-kernel instantiation.
template <class Kern>
int pair_clusters(Kern kern, int threads, int smem_bytes, int sm_count, int cta) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(sm_count / cta * cta), 1, 1);
    cfg.blockDim = dim3(static_cast<unsigned>(threads), 1, 1);
    cfg.dynamicSmemBytes = static_cast<size_t>(smem_bytes);
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = sm_count / cta;
    }
    return n;
}

// pair_clusters for the current device, computed once per device (after the kernel's
// shared-memory limit is raised there).
template <auto Kern>
int resident_clusters(int threads, int smem_bytes, int sm_count, int cta) {
    static std::atomic<int> cache[kMaxDevices];
    const int dev = current_device();
    if (dev < 0) return sm_count / cta;
    int n = cache[dev].load(std::memory_order_relaxed);
    if (n > 0) return n;
    n = pair_clusters(Kern, threads, smem_bytes, sm_count, cta);
    cache[dev].store(n, std::memory_order_relaxed);
    return n;
}

// Split-K tail of one launch: tail_tiles tiles, each in tail_split k ranges (0: whole).
struct SkPlan {
    long long tail_tiles = 0;
    int tail_split = 0;
};

// Units of split tail tiles a scratch area must hold: up to three waves of pair clusters.
constexpr int kTailWaves = 3;

// The split of the last partial wave of `tiles` tiles over `clusters` clusters: R tail
// tiles in S k ranges, S chosen so that the R S units fill whole waves as nearly as
// possible (at most kTailWaves waves, at least 8 k-blocks per range); none if no split
// beats the plain partial wave.
inline SkPlan tail_plan(long long tiles, long long clusters, int k_blocks) {
    SkPlan p;
    const long long R = tiles % clusters;
    if (tiles < clusters || R == 0) return p;
    double best = static_cast<double>(R) / clusters;  // busy fraction of the plain last wave
    for (int S = 2; S <= 64; ++S) {
        if (R * S > kTailWaves * clusters || k_blocks / S < 8) break;
        const long long waves = (R * S + clusters - 1) / clusters;
        const double eff = static_cast<double>(R * S) / (waves * clusters);
        if (eff > best + 1e-9) {
            best = eff;
            p.tail_tiles = R;
            p.tail_split = S;
        }
    }
    return p;
}

// With sk_scratch non-null, the tiles are split by `split` k ranges each when that is above
// 1, else those of the last partial wave by tail_plan, or as *tail says (SegCursor); the caller
// then runs sk_fixup over them (plan->tail_tiles > 0).  sk_scratch holds 256 x BN fp32 per unit.
template <int BN, bool A_MN, bool B_MN, int STAGES, int MAXG, class Epi>
cudaError_t run_gemm_pair(const GemmMaps<MAXG>& maps, const typename Epi::Params& ep,
                          const GemmShape& sh_in, unsigned* status, cudaStream_t st,
                          float* sk_scratch = nullptr, SkPlan* plan = nullptr, int split = 0,
                          const SkPlan* tail = nullptr) {
    if (plan) *plan = SkPlan{};
    if (sh_in.tiles <= 0 || sh_in.k_blocks <= 0) return cudaSuccess;
    using L = GemmPairSmem<BN, STAGES, pair_ksub<BN, A_MN, B_MN>()>;
    static_assert(L::kBytes + 2 * kSmemReserve <= kSmemPerSm,
                  "the stages leave the shared memory that a block of the host-input copy takes");
    constexpr auto kern = tc_gemm_pair_kernel<BN, A_MN, B_MN, STAGES, MAXG, Epi>;
    const cudaError_t attr_err = set_smem_limit<kern>(L::kBytes);
    if (attr_err != cudaSuccess) return attr_err;
    DevInfo di;
    if (!current_device_info(&di)) return cudaErrorUnknown;
    const int max_clusters = resident_clusters<kern>(gemm_threads<Epi>(), L::kBytes, di.sm_count, 2);
    const long long units = split > 1 ? sh_in.tiles * split : sh_in.tiles;
    const long long clusters = units < max_clusters ? units : max_clusters;
    GemmShape sh = sh_in;
    if (sk_scratch) {
        SkPlan p;
        if (split > 1) {
            p.tail_tiles = sh.tiles;
            p.tail_split = split;
        } else {
            p = tail ? *tail : tail_plan(sh.tiles, clusters, sh.k_blocks);
        }
        if (p.tail_tiles > 0) {
            sh.tail_tiles = p.tail_tiles;
            sh.tail_split = p.tail_split;
            sh.sk_scratch = sk_scratch;
            if (plan) *plan = p;
        }
    }
    return launch_chained(kern, dim3(static_cast<unsigned>(2 * clusters)), gemm_threads<Epi>(),
                          L::kBytes, st, maps, ep, sh, status, wait_limit_ns());
}

// Fixups of the split-K tail: sum the tail_split k-range partials of every split tail
// tile in range order, then apply the epilogue the whole tiles got.
// Grid (tail tiles, 256 rows / rows per block): one thread per 4 columns of a row.
constexpr int kFixupThreads = 256;

// The summed partials of this thread's 4 columns; false outside the matrix.
template <int BN>
__device__ __forceinline__ bool sk_tail_sum(const GemmShape& sh, const float* scratch,
                                            int& row, int& n, float (&s4)[4]) {
    constexpr int kThreadsPerRow = BN / 4;
    constexpr int kRowsPerBlock = kFixupThreads / kThreadsPerRow;
    const long long R = sh.tail_tiles;
    const long long r_tile = blockIdx.x;
    const int r = blockIdx.y * kRowsPerBlock + threadIdx.x / kThreadsPerRow;
    const int col = (threadIdx.x % kThreadsPerRow) * 4;
    int g, mp, nb;
    tile_coords(sh.tiles - R + r_tile, sh, g, mp, nb);
    row = mp * kPairBM + r;
    n = nb * BN + col;
    if (row >= sh.M || n >= sh.N) return false;  // N % 8 == 0: whole groups of 4
    s4[0] = s4[1] = s4[2] = s4[3] = 0.f;
    const float* p = scratch + (static_cast<size_t>(r_tile) * kPairBM + r) * BN + col;
    const size_t step = static_cast<size_t>(R) * kPairBM * BN;  // one range to the next
#pragma unroll 4
    for (int q = 0; q < sh.tail_split; ++q) {
        const float4 u = *reinterpret_cast<const float4*>(p + q * step);
        s4[0] += u.x;
        s4[1] += u.y;
        s4[2] += u.z;
        s4[3] += u.w;
    }
    return true;
}

template <int BN>
dim3 sk_fixup_grid(const SkPlan& plan) {
    constexpr int kRowsPerBlock = kFixupThreads / (BN / 4);
    return dim3(static_cast<unsigned>(plan.tail_tiles), kPairBM / kRowsPerBlock);
}

inline GemmShape sk_fixup_shape(const SkPlan& plan, const GemmShape& sh_in) {
    GemmShape sh = sh_in;
    sh.tail_tiles = plan.tail_tiles;
    sh.tail_split = plan.tail_split;
    return sh;
}

constexpr int kPairStages = 3;   // 256 x 256 pair tiles: 64 KB stages of two k-blocks

// 0 = single-CTA tiles, 1 and 2 = CTA-pair tiles (gemm_variant, gemm_bf16.cu).
inline bool use_pair() { return gemm_variant() >= 1; }

// Rasterisation band in tile rows, unless overridden: 16 tile rows, i.e. 2048
// output rows of single-CTA tiles and 4096 of pair tiles.  With pair tiles the
// 4096-row band gave the lowest DRAM traffic of the three GEMMs of the OLMo-2-7B
// shape (band heights 2 to 32 measured).
constexpr int kBandTiles = 16;
inline int band_for(bool) {
    const int o = band_override();
    return o > 0 ? o : kBandTiles;
}

// Whether a GEMM of `tiles` 256 x 256 pair tiles runs on tiles of 128 columns instead: when
// twice as many tiles still have a cluster each.  What bounds so small a GEMM is the
// epilogue's traffic through one SM (32 bytes a clock to L2), which twice as many SMs share.
// T 200, d 256, d_ff 384, V 1024, 2 layers: update 13.1 -> 9.5 us, projection 15.1 -> 12.1.
inline bool half_tiles(long long tiles) {
    DevInfo di;
    return current_device_info(&di) && 2 * tiles <= di.sm_count / 2;
}

constexpr int kHalfBN = 128;     // 48 KB stages of two k-blocks
constexpr int kHalfStages = 4;

// A GEMM with an 8-warp epilogue (MN-major B) on the kernel and tiles its size calls for.
template <bool A_MN, int MAXG, template <int> class Epi>
cudaError_t run_quad(const GemmMaps<MAXG>& maps, const typename Epi<2>::Params& ep, int M, int N,
                     int K, int groups, unsigned* status, cudaStream_t st) {
    constexpr int kBN = 256, kStages = 4;
    if (!use_pair())
        return run_gemm<kBN, A_MN, true, kStages, MAXG, Epi<2>>(
            maps, ep, make_shape(M, N, K, kBN, groups, band_for(false)), status, st);
    const GemmShape sh = make_shape(M, N, K, kBN, groups, band_for(true), kPairBM);
    if (!half_tiles(sh.tiles))
        return run_gemm_pair<kBN, A_MN, true, kPairStages, MAXG, Epi<2>>(maps, ep, sh, status, st);
    GemmShape hs = sh;
    hs.n_blocks = 2 * sh.n_blocks;  // also a last half outside the matrix: its slots are written
    hs.tiles = 2 * sh.tiles;
    return run_gemm_pair<kHalfBN, A_MN, true, kHalfStages, MAXG, Epi<1>>(maps, ep, hs, status, st);
}

}  // namespace fpo
