// ns_gemm.cuh -- the GEMMs of the Newton-Schulz iteration (newton_schulz.cu): batches of fp16
// matrices on CTA pairs, with fp32 accuracy (kSplit) or fp16 operands' (not kSplit).
//
//   A  = X X^T            (or X^T X: the smaller side)       EpiSym
//   B  = b A + c A A                                         EpiSym
//   X' = a X + B X        (or a X + X B)                     EpiApply
//
// The roles, barriers, bounded waits and teardown are those of tc_gemm_pair_kernel: a cluster
// of two CTAs, a TMA producer in each, one MMA issuer in the leader, 8 epilogue warps in each,
// 256 x BN tiles.  A pipeline stage is two A boxes of 128 rows x 64 k (16 KB each) and two B
// boxes of BN / 2 rows:
//   fp16   the boxes of two consecutive k-blocks; a full barrier for each k-block
//   kSplit high and low parts of one k-block (each operand the sum of two fp16 matrices, 22
//          bits); one full barrier
//
// A and A A are symmetric: their GEMMs visit the tiles on and under the diagonal only, and the
// epilogue writes each tile a second time, turned over.
//
// kSplit: the tensor core truncates its fp32 sums.  Positive sums of 11008 products came out
// 4.1e-5 too small, random ones 1.2e-5 off in norm; the iteration multiplies such errors by
// ten and more.  So an accumulator holds one 64-deep k-block only: the 8 MMAs with one low
// operand first, while the sums (and what is truncated of them) are 2^-11 of the final size,
// then the 4 high x high MMAs; the epilogue warps add it to sums in their registers, rounding
// to nearest, while the next k-block fills the other accumulator.  BN is 128 there: 64 sums per
// thread of 8 warps (with 128, and 168 registers, the loop spilled and took 2.7 us a k-block,
// three times its MMAs).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "error_math.cuh"
#include "tc_gemm_pair.cuh"

namespace fpo {

// tma_load_2d_pair (ptx.cuh) for a batch of matrices: matrix z.
__device__ __forceinline__ void tma_load_3d_pair(const CUtensorMap* map, uint32_t smem_dst,
                                                 uint32_t bar_cluster_addr, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar_cluster_addr), "r"(x), "r"(y), "r"(z)
        : "memory");
}

// tmem_ld_32x32b_x32 (ptx.cuh) for 16 columns.
__device__ __forceinline__ void tmem_ld_32x32b_x16(uint32_t taddr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
          "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// idesc_bf16_f32 (ptx.cuh) with fp16 A and B (format fields 0).
__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N, bool a_mn, bool b_mn) {
    return idesc_bf16_f32(M, N, a_mn, b_mn) & ~((1u << 7) | (1u << 10));
}

constexpr int kNsWarps = 8;                   // epilogue warps
constexpr int kNsThreads = 64 + 32 * kNsWarps;

template <int BN>
struct NsSmem {
    static constexpr int kStages = BN == 256 ? 3 : 4;
    static constexpr int kABox = 128 * kBK * 2;        // bytes of one operand box
    static constexpr int kBBox = (BN / 2) * kBK * 2;
    static constexpr int kStageBytes = 2 * (kABox + kBBox);
    static constexpr int kOutOffset = kStages * kStageBytes;
    static constexpr int kBarOffset = kOutOffset + kNsWarps * kOutBufBytes;
    static constexpr int kNumBars = 3 * kStages + 5;
    static constexpr int kMiscOffset = kBarOffset + kNumBars * 8;
    static constexpr int kBytes = kMiscOffset + 16 + 1024;
};

struct NsShape {
    GemmShape g;   // M, N, K, blocks; tiles of all matrices
    bool tri;      // only tiles that reach under or onto the diagonal (M = N)
};

struct NsMaps {
    CUtensorMap a[2], b[2];  // high and low parts (low: kSplit only)
};

// Tile t: matrix g, block row mb of 256, block column nb of BN.  tri: block row mb has the
// columns up to its own last one, (mb + 1) 256 / BN blocks (those past the matrix, in the last
// block row, are empty).
template <int BN>
__device__ __forceinline__ void ns_tile(long long t, const NsShape& sh, int& g, int& mb, int& nb) {
    if (!sh.tri) {
        tile_coords(t, sh.g, g, mb, nb);
        return;
    }
    constexpr int kRatio = kPairBM / BN;
    const int n = sh.g.m_blocks;
    const int per = kRatio * (n * (n + 1) / 2);
    g = static_cast<int>(t / per);
    const int r = static_cast<int>(t - static_cast<long long>(g) * per);
    const int q = r / kRatio;  // of the 256 x 256 blocks
    mb = static_cast<int>((sqrtf(8.f * q + 1.f) - 1.f) * 0.5f);
    while (mb * (mb + 1) / 2 > q) --mb;
    while ((mb + 1) * (mb + 2) / 2 <= q) ++mb;
    nb = r - kRatio * (mb * (mb + 1) / 2);
}

// One CTA's box (ROWS rows x 64 k, or turned) of matrix z, counted on the leader's barrier.
template <bool MN, int ROWS>
__device__ __forceinline__ void ns_load(const CUtensorMap* map, uint32_t dst, uint32_t bar, int row0,
                                        int k0, int z) {
    if constexpr (!MN) {
        tma_load_3d_pair(map, dst, bar, k0, row0, z);
    } else {
#pragma unroll
        for (int i = 0; i < ROWS / 64; ++i)
            tma_load_3d_pair(map, dst + i * (64 * kBK * 2), bar, row0 + 64 * i, k0, z);
    }
}

__device__ __forceinline__ uint32_t pack_f16x2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_f16x2(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// ---------------------------------------------------------------------------
// Symmetric results S [M, M] of one matrix: s = lin_coef L + acc_coef acc, rounded to fp16 (with
// kSplit: high and low parts), to (row, col) and (col, row).  L (null: no such term) is read in
// the row layout of the accumulator; both are [M, ld], ld a multiple of 8, the columns from M to
// ld zero.
template <bool kSplit>
struct EpiSymBase {
    struct Params {
        const __half* lin[2];  // high, low parts of L, or null
        __half* out[2];
        long long stride;      // of one matrix in a batch
        int M, ld;
        float lin_coef, acc_coef;
    };
};

template <int BN, bool kSplit>
struct EpiSym : EpiSymBase<kSplit> {
    using Params = typename EpiSymBase<kSplit>::Params;
    static constexpr int kParts = kSplit ? 2 : 1;
    static constexpr int kChunks = BN / 2 / 32;

    const Params& p;
    long long base;
    int row, col0;
    bool mirror;
    uint4 l[kParts][4];  // the next chunk's 32 elements of L

    __device__ __forceinline__ void fetch(int c) {
        if (!p.lin[0]) return;
#pragma unroll
        for (int h = 0; h < kParts; ++h) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int col = col0 + 32 * c + 8 * q;
                l[h][q] = row < p.M && col < p.ld
                              ? *reinterpret_cast<const uint4*>(
                                    p.lin[h] + base + static_cast<long long>(row) * p.ld + col)
                              : make_uint4(0u, 0u, 0u, 0u);
            }
        }
    }

    __device__ __forceinline__ EpiSym(const Params& p_, int g, int row0, int col0_, int lane,
                                      bool mirror_)
        : p(p_), base(g * p_.stride), row(row0 + lane), col0(col0_), mirror(mirror_) {
        fetch(0);
    }

    __device__ __forceinline__ void chunk(float (&v)[32], uint32_t, int, int c) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] *= p.acc_coef;
        if (p.lin[0]) {
#pragma unroll
            for (int h = 0; h < kParts; ++h) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t w[4] = {l[h][q].x, l[h][q].y, l[h][q].z, l[h][q].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 f = unpack_f16x2(w[k]);
                        v[8 * q + 2 * k] = fmaf(p.lin_coef, f.x, v[8 * q + 2 * k]);
                        v[8 * q + 2 * k + 1] = fmaf(p.lin_coef, f.y, v[8 * q + 2 * k + 1]);
                    }
                }
            }
            if (c + 1 < kChunks) fetch(c + 1);
        }
        if (row >= p.M) return;
        const int cc = col0 + 32 * c;
#pragma unroll
        for (int h = 0; h < kParts; ++h) {
            __half* o = p.out[h] + base;
            uint32_t w[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) w[k] = pack_f16x2(v[2 * k], v[2 * k + 1]);
            uint4* dst = reinterpret_cast<uint4*>(o + static_cast<long long>(row) * p.ld + cc);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (cc + 8 * q < p.ld)
                    dst[q] = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
            if (mirror) {  // a column of the tile: 32 lanes, 64 bytes of one row
                unsigned short* m = reinterpret_cast<unsigned short*>(o) + row;
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (cc + j < p.M)
                        m[static_cast<long long>(cc + j) * p.ld] =
                            static_cast<unsigned short>(w[j / 2] >> (16 * (j % 2)));
            }
            if constexpr (kSplit) {
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float2 f = unpack_f16x2(w[k]);
                    v[2 * k] -= f.x;
                    v[2 * k + 1] -= f.y;
                }
            }
        }
    }
};

// ---------------------------------------------------------------------------
// X' = lin_coef X + acc_coef acc over [M, N] (row stride ld, a multiple of 8, what lies
// between N and ld zero).  What becomes of it:
//   kNext    the next X: its high part, and its low part (not kSplit: for the linear term
//            only) or (kSplit) low part and the fp32 value
//   kResult  O [M, N] (row stride N) in the call's type
//   kWeight  W <- keep W - rate X', and W_out in the call's type
// The linear term takes X in more bits than the operands have: of a direction in which X is
// small B X is next to nothing, so a X carries it, 3.4 times larger after every step, and with
// it any rounding of X (fp16: up to 10% of the result for a matrix of low rank).  fp16 reads
// the low part where it was kept (lin_lo), kSplit the fp32 value.
enum NsOut { kNext = 0, kResult = 1, kWeight = 2 };

template <bool kSplit, int kOut>
struct EpiApplyBase {
    using Out = std::conditional_t<kSplit, float, __nv_bfloat16>;
    struct Params {
        const __half* hi;     // X (fp16)
        __half* lo;           // X's low part: read if lin_lo, written (kNext) if next_lo
        float* x32;           // kSplit: X in fp32, updated in place (kNext)
        __half* next_hi;      // kNext
        __half* next_lo;
        long long stride;     // of one matrix in a batch
        int M, N, ld;
        float lin_coef, acc_coef;
        bool lin_lo;
        float keep, rate;              // kWeight
        Out* out[kMaxGroups];          // kResult: O; kWeight: W_out or null
        float* W[kMaxGroups];          // kWeight
    };
};

template <int BN, bool kSplit, int kOut>
struct EpiApply : EpiApplyBase<kSplit, kOut> {
    using Out = typename EpiApplyBase<kSplit, kOut>::Out;
    using Params = typename EpiApplyBase<kSplit, kOut>::Params;
    static constexpr int kChunks = BN / 2 / 32;
    static constexpr int kAcc = 8;     // accesses of a chunk: 4 rows, 8 lanes of 4 columns to a row

    const Params& p;
    long long base;
    float* W;    // of this matrix (kWeight)
    Out* out;    // of this matrix
    int r0, c0;
    uint2 hi[kSplit ? 1 : kAcc], lo[kSplit ? 1 : kAcc];
    float4 x[kSplit ? kAcc : 1], w[kOut == kWeight ? kAcc : 1];

    __device__ __forceinline__ bool in(int i, int c) const {
        return r0 + 4 * i < p.M && c0 + 32 * c < (kOut == kNext ? p.ld : p.N);
    }
    // 4 elements of a row of N floats from column col, those inside it (N > col)
    __device__ __forceinline__ float4 ld4(const float* q, int col) const {
        if ((p.N & 3) == 0) return *reinterpret_cast<const float4*>(q);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        v.x = q[0];
        if (col + 1 < p.N) v.y = q[1];
        if (col + 2 < p.N) v.z = q[2];
        if (col + 3 < p.N) v.w = q[3];
        return v;
    }
    __device__ __forceinline__ void st4(float* q, const float4& v, int col) const {
        if ((p.N & 3) == 0) {
            *reinterpret_cast<float4*>(q) = v;
            return;
        }
        q[0] = v.x;
        if (col + 1 < p.N) q[1] = v.y;
        if (col + 2 < p.N) q[2] = v.z;
        if (col + 3 < p.N) q[3] = v.w;
    }
    // (N is a multiple of 8 for bf16)
    __device__ __forceinline__ void st4(__nv_bfloat16* q, const float4& v, int) const {
        *reinterpret_cast<uint2*>(q) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    }

    __device__ __forceinline__ void fetch(int c) {
#pragma unroll
        for (int i = 0; i < kAcc; ++i) {
            const bool ok = in(i, c);
            const long long o =
                ok ? base + static_cast<long long>(r0 + 4 * i) * p.ld + c0 + 32 * c : base;
            if constexpr (kSplit) {
                x[i] = *reinterpret_cast<const float4*>(p.x32 + o);
            } else {
                hi[i] = *reinterpret_cast<const uint2*>(p.hi + o);
                if (p.lin_lo) lo[i] = *reinterpret_cast<const uint2*>(p.lo + o);
            }
            if constexpr (kOut == kWeight) {
                const int col = ok ? c0 + 32 * c : 0;
                w[i] = ld4(W + (ok ? static_cast<long long>(r0 + 4 * i) * p.N + col : 0), col);
            }
        }
    }

    __device__ __forceinline__ EpiApply(const Params& p_, int g, int row0, int col0, int lane, bool)
        : p(p_), base(g * p_.stride), W(kOut == kWeight ? p_.W[g] : nullptr),
          out(kOut == kNext ? nullptr : p_.out[g]), r0(row0 + lane / 8), c0(col0 + 4 * (lane % 8)) {
        fetch(0);
    }

    __device__ __forceinline__ void chunk(float (&v)[32], uint32_t buf, int lane, int c) {
        uint32_t u[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) u[j] = __float_as_uint(v[j]);
        out_stage_row(buf, lane, u);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kAcc; ++i) {
            const uint32_t r = static_cast<uint32_t>(4 * i + lane / 8);
            float4 a = ld_shared_f4(buf + r * 128u + (((lane % 8) ^ (r & 7u)) << 4));
            float4 xl;
            if constexpr (kSplit) {
                xl = x[i];
            } else {
                const float2 h0 = unpack_f16x2(hi[i].x), h1 = unpack_f16x2(hi[i].y);
                xl = make_float4(h0.x, h0.y, h1.x, h1.y);
                if (p.lin_lo) {
                    const float2 l0 = unpack_f16x2(lo[i].x), l1 = unpack_f16x2(lo[i].y);
                    xl.x += l0.x;
                    xl.y += l0.y;
                    xl.z += l1.x;
                    xl.w += l1.y;
                }
            }
            a.x = fmaf(p.lin_coef, xl.x, a.x * p.acc_coef);
            a.y = fmaf(p.lin_coef, xl.y, a.y * p.acc_coef);
            a.z = fmaf(p.lin_coef, xl.z, a.z * p.acc_coef);
            a.w = fmaf(p.lin_coef, xl.w, a.w * p.acc_coef);
            if (!in(i, c)) continue;
            const int row = r0 + 4 * i, col = c0 + 32 * c;
            if constexpr (kOut == kNext) {
                const long long o = base + static_cast<long long>(row) * p.ld + col;
                const uint2 h = make_uint2(pack_f16x2(a.x, a.y), pack_f16x2(a.z, a.w));
                *reinterpret_cast<uint2*>(p.next_hi + o) = h;
                if (p.next_lo) {
                    const float2 h0 = unpack_f16x2(h.x), h1 = unpack_f16x2(h.y);
                    *reinterpret_cast<uint2*>(p.next_lo + o) =
                        make_uint2(pack_f16x2(a.x - h0.x, a.y - h0.y),
                                   pack_f16x2(a.z - h1.x, a.w - h1.y));
                }
                if constexpr (kSplit) *reinterpret_cast<float4*>(p.x32 + o) = a;
            } else {
                const long long o = static_cast<long long>(row) * p.N + col;
                if constexpr (kOut == kWeight) {
                    a.x = fmaf(-p.rate, a.x, p.keep * w[i].x);
                    a.y = fmaf(-p.rate, a.y, p.keep * w[i].y);
                    a.z = fmaf(-p.rate, a.z, p.keep * w[i].z);
                    a.w = fmaf(-p.rate, a.w, p.keep * w[i].w);
                    st4(W + o, a, col);
                    if (out) st4(out + o, a, col);
                } else {
                    st4(out + o, a, col);
                }
            }
        }
        if (c + 1 < kChunks) fetch(c + 1);
        __syncwarp();
    }
};

// ---------------------------------------------------------------------------
template <int BN, bool A_MN, bool B_MN, bool kSplit, class Epi>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kNsThreads, 1)
    ns_gemm_kernel(const __grid_constant__ NsMaps maps,
                   const __grid_constant__ typename Epi::Params ep, const NsShape sh,
                   unsigned int* status, unsigned long long wait_limit_ns) {
    using L = NsSmem<BN>;
    constexpr int kStages = L::kStages;
    constexpr int kSub = kSplit ? 1 : 2;   // k-blocks (and full barriers) per stage
    constexpr uint32_t kIdesc = idesc_f16_f32(kPairBM, BN, A_MN, B_MN);
    constexpr uint16_t kBoth = 0x3;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t pad = (1024u - (raw & 1023u)) & 1023u;
    uint8_t* smem = smem_raw + pad;
    const uint32_t sbase = raw + pad;

    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    const long long cluster = blockIdx.x / 2;
    const long long n_clusters = gridDim.x / 2;
    const int stages_k = (sh.g.k_blocks + kSub - 1) / kSub;  // stages per tile

    const uint32_t bar0 = sbase + L::kBarOffset;
    constexpr int kFull = kStages * kSub;
    auto full_bar = [&](int s, int j) { return bar0 + 8u * (s * kSub + j); };
    auto empty_bar = [&](int s) { return bar0 + 8u * (kFull + s); };
    auto tfull_bar = [&](int a) { return bar0 + 8u * (kFull + kStages + a); };
    auto tempty_bar = [&](int a) { return bar0 + 8u * (kFull + kStages + 2 + a); };
    const uint32_t drain_bar = bar0 + 8u * (kFull + kStages + 4);
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem + L::kMiscOffset + kMiscTmem);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::kMiscOffset + kMiscAbort);
    uint32_t* issued_word = reinterpret_cast<uint32_t*>(smem + L::kMiscOffset + kMiscIssued);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            for (int j = 0; j < kSub; ++j) mbar_init(full_bar(s, j), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull_bar(a), 1);
            mbar_init(tempty_bar(a), 2 * kNsWarps);
        }
        mbar_init(drain_bar, 1);
        *abort_flag = 0;
        *issued_word = 0;
        fence_mbar_init();
        tma_prefetch_desc(&maps.a[0]);
        tma_prefetch_desc(&maps.b[0]);
    }
    if (warp == 1) {
        tmem_alloc_pair<2 * BN>(smem_u32(tmem_holder));
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;
    grid_dependency_wait();

    const WaitGuard guard{abort_flag, status, wait_limit_ns};

    if (warp == 0) {
        // ------------------------------------------------------- TMA producer (both CTAs)
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, issued = 0;
            bool ok = true;
            for (long long t = cluster; ok && t < sh.g.tiles; t += n_clusters) {
                int g, mb, nb;
                ns_tile<BN>(t, sh, g, mb, nb);
                const int a_row = mb * kPairBM + 128 * static_cast<int>(rank);
                const int b_row = nb * BN + (BN / 2) * static_cast<int>(rank);
                for (int kb = 0; kb < stages_k; ++kb) {
                    if (!mbar_wait_cl(empty_bar(stage), phase ^ 1u, guard)) { ok = false; break; }
                    const uint32_t sa = sbase + stage * L::kStageBytes, sb = sa + 2 * L::kABox;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int bar_j = kSplit ? 0 : j, part = kSplit ? j : 0;
                        const uint32_t fb = mapa_shared(full_bar(stage, bar_j), 0);
                        if (leader && (!kSplit || j == 0))
                            mbar_arrive_expect_tx(full_bar(stage, bar_j),
                                                  2 * (L::kStageBytes / kSub));
                        const int k0 = (kSplit ? kb : 2 * kb + j) * kBK;
                        ns_load<A_MN, 128>(&maps.a[part], sa + j * L::kABox, fb, a_row, k0, g);
                        ns_load<B_MN, BN / 2>(&maps.b[part], sb + j * L::kBBox, fb, b_row, k0, g);
                    }
                    ++issued;
                    if (++stage == kStages) { stage = 0; phase ^= 1u; }
                }
            }
            *issued_word = issued;
            grid_dependency_trigger();
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------- pair MMA (leader only)
        if (leader && lane == 0) {
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool ok = true, issued_any = false;
            for (long long t = cluster; ok && t < sh.g.tiles; t += n_clusters) {
                for (int kb = 0; kb < stages_k; ++kb) {
                    if (kSplit || kb == 0) {
                        if (!mbar_wait_cl(tempty_bar(acc), acc_phase ^ 1u, guard)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                    }
                    const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(acc * BN);
                    const uint32_t sa = sbase + stage * L::kStageBytes, sb = sa + 2 * L::kABox;
                    if constexpr (kSplit) {
                        if (!mbar_wait_cl_poll(full_bar(stage, 0), phase, guard)) { ok = false; break; }
                        tc_fence_after();
                        // high x low, low x high, then high x high
#pragma unroll
                        for (int m = 0; m < 3; ++m) {
#pragma unroll
                            for (int kk = 0; kk < kBK / kUmmaK; ++kk)
                                tc_mma_bf16_pair(
                                    d_tmem, operand_desc<A_MN>(sa + (m == 1 ? L::kABox : 0), kk),
                                    operand_desc<B_MN>(sb + (m == 0 ? L::kBBox : 0), kk), kIdesc,
                                    (m != 0 || kk != 0) ? 1u : 0u);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            if (!mbar_wait_cl_poll(full_bar(stage, j), phase, guard)) { ok = false; break; }
                            tc_fence_after();
#pragma unroll
                            for (int kk = 0; kk < kBK / kUmmaK; ++kk)
                                tc_mma_bf16_pair(d_tmem, operand_desc<A_MN>(sa + j * L::kABox, kk),
                                                 operand_desc<B_MN>(sb + j * L::kBBox, kk), kIdesc,
                                                 (kb != 0 || j != 0 || kk != 0) ? 1u : 0u);
                            issued_any = true;
                        }
                        if (!ok) break;
                    }
                    issued_any = true;
                    tc_commit_pair_multicast(empty_bar(stage), kBoth);
                    if (++stage == kStages) { stage = 0; phase ^= 1u; }
                    if (kSplit || kb == stages_k - 1) {
                        tc_commit_pair_multicast(tfull_bar(acc), kBoth);
                        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
                    }
                }
            }
            if (issued_any) {
                tc_commit_pair_multicast(drain_bar, 0x1);
                mbar_wait_cl_drain(drain_bar, 0, kDrainLimitNs);
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------- epilogue (both CTAs)
        const int q = warp & 3;               // TMEM lanes [32 q, 32 q + 32)
        const int half = (warp - 2) / 4;
        constexpr int kWarpCols = BN / 2;     // columns [kWarpCols half, kWarpCols (half + 1))
        const uint32_t buf = sbase + L::kOutOffset + static_cast<uint32_t>(warp - 2) * kOutBufBytes;
        int acc = 0;
        uint32_t acc_phase = 0;
        auto ready = [&] {
            if (!mbar_wait_cl(tfull_bar(acc), acc_phase, guard)) return false;
            tc_fence_after();
            return true;
        };
        auto release = [&] {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (leader)
                    mbar_arrive(tempty_bar(acc));
                else
                    mbar_arrive_cluster(mapa_shared(tempty_bar(acc), 0));
            }
            if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
        };
        auto t_row = [&] {
            return tmem_base + (static_cast<uint32_t>(q * 32) << 16) +
                   static_cast<uint32_t>(acc * BN + half * kWarpCols);
        };
        constexpr int kChunks = kWarpCols / 32;
        bool ok = true;
        for (long long t = cluster; ok && t < sh.g.tiles; t += n_clusters) {
            int g, mb, nb;
            ns_tile<BN>(t, sh, g, mb, nb);
            const int row0 = mb * kPairBM + 128 * static_cast<int>(rank) + 32 * q;
            const int col0 = nb * BN + half * kWarpCols;
            const bool mirror = sh.tri && nb * BN / kPairBM != mb;
            if constexpr (kSplit) {
                float s[kChunks][32];
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int j = 0; j < 32; ++j) s[c][j] = 0.f;
                for (int kb = 0; ok && kb < stages_k; ++kb) {
                    ok = ready();
                    if (!ok) break;
#pragma unroll
                    for (int c = 0; c < 2 * kChunks; ++c) {
                        float v[16];
                        tmem_ld_32x32b_x16(t_row() + 16 * c, v);
#pragma unroll
                        for (int j = 0; j < 16; ++j) s[c / 2][16 * (c % 2) + j] += v[j];
                    }
                    release();
                }
                if (!ok) break;
                Epi epi(ep, g, row0, col0, lane, mirror);
#pragma unroll
                for (int c = 0; c < kChunks; ++c) epi.chunk(s[c], buf, lane, c);
                __syncwarp();
            } else {
                Epi epi(ep, g, row0, col0, lane, mirror);
                ok = ready();
                if (!ok) break;
                const uint32_t tr = t_row();
#pragma unroll 1
                for (int c = 0; c < kChunks; ++c) {
                    float v[32];
                    tmem_ld_32x32b_x32(tr + 32 * c, v);
                    if (c == kChunks - 1) release();
                    epi.chunk(v, buf, lane, c);
                    __syncwarp();
                }
            }
        }
        __syncwarp();
    }

    // Teardown, as in tc_gemm_pair_kernel.
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    if (leader && threadIdx.x == 0)
        pair_drain_copies<kStages, kSub>(bar0, *issued_word,
                                           ld_shared_cluster_u32(mapa_shared(smem_u32(issued_word), 1)),
                                           L::kStageBytes / kSub);
    __syncthreads();
    cluster_sync();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair<2 * BN>(tmem_base);
    }
}

}  // namespace fpo
