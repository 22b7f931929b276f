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
// to nearest, while the next k-blocks fill other accumulators: 64 sums per thread with BN 128,
// 0.85 us a k-block (0.4 of MMAs at the tensor rate, 0.6 of operands from shared memory), and 128
// with BN 256, 1.03 us (0.8 of MMAs), where the warps share registers out anew (with 168 each
// the loop spilled and took 2.7 us).  The gradient of the Muon step (EpiMomentum) is drained the
// same way, every kRun stages.
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

// idesc_bf16_f32 (ptx.cuh) with fp16 A and B (format fields 0).
__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N, bool a_mn, bool b_mn) {
    return idesc_bf16_f32(M, N, a_mn, b_mn) & ~((1u << 7) | (1u << 10));
}

constexpr int kNsWarps = 8;                   // epilogue warps
constexpr int kNsThreads = 64 + 32 * kNsWarps;

// Stages whose sums one accumulator holds before the epilogue warps add it to their registers
// ("drained"); 0: all of a tile's.
template <bool kSplit, class Epi>
constexpr int ns_run() {
    return kSplit ? 1 : Epi::kRun;
}

// Accumulators in TMEM.  kSplit: four, as the MMAs of a k-block take no longer than the way to
// the epilogue warps and back (eight fp32 256 x 4096, five steps: 421 us with two, 388 with four).
constexpr int kNsMaxAccs = 4;
template <bool kSplit, int BN = 128>
constexpr int ns_accs() {
    return kSplit && BN == 128 ? kNsMaxAccs : 2;
}

// Warps before the epilogue's.  kSplit with 256 columns, and EpiMomentum, which holds the momentum
// beside the sums: a warpgroup of its own for the producer and the MMA issuer, whose registers the
// epilogue's two warpgroups take over (128 sums a thread): 384 threads are launched with 168 each
// (launch_ns looks), and go on with 40, 232 and 232.
constexpr int kNsFewRegs = 40, kNsManyRegs = 232;
template <int BN, bool kSplit, class Epi>
constexpr int ns_first_warp() {
    return (kSplit ? BN == 256 : Epi::kRun > 0) ? 4 : 2;
}
template <int BN, bool kSplit, class Epi>
constexpr int ns_threads() {
    return 32 * (ns_first_warp<BN, kSplit, Epi>() + kNsWarps);
}
template <int R>
__device__ __forceinline__ void ns_more_registers() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R));
}
template <int R>
__device__ __forceinline__ void ns_fewer_registers() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R));
}

template <int BN>
struct NsSmem {
    static constexpr int kStages = BN == 256 ? 3 : 4;
    static constexpr int kABox = 128 * kBK * 2;        // bytes of one operand box
    static constexpr int kBBox = (BN / 2) * kBK * 2;
    static constexpr int kStageBytes = 2 * (kABox + kBBox);
    static constexpr int kOutOffset = kStages * kStageBytes;
    static constexpr int kBarOffset = kOutOffset + kNsWarps * kOutBufBytes;
    static constexpr int kNumBars = 3 * kStages + 2 * kNsMaxAccs + 1;
    static constexpr int kMiscOffset = kBarOffset + kNumBars * 8;
    static constexpr int kBytes = kMiscOffset + 16 + 1024;
};

struct NsShape {
    GemmShape g;   // M, N, K, blocks; tiles of all matrices
    bool tri;      // only tiles that reach under or onto the diagonal (M = N)
    // EpiSym with kSplit (kRanges): a tile's k-blocks in `splits` ranges of their own units (unit u:
    // range u % splits of tile u / splits).  With splits > 1 every warp of a unit leaves its sums in
    // slots[unit][CTA][warp], and the last of a tile to arrive at counts[tile][CTA][warp] (zero
    // before and after) adds them in the ranges' order and goes on to the epilogue: none waits.
    int splits;
    float* slots;
    unsigned* counts;
};

struct NsMaps {
    CUtensorMap a[2], b[2];  // of a batch: high and low parts (low: kSplit only)
    __device__ __forceinline__ const CUtensorMap* A(int part, int) const { return &a[part]; }
    __device__ __forceinline__ const CUtensorMap* B(int part, int) const { return &b[part]; }
    static __device__ __forceinline__ int z(int g) { return g; }
};

struct NsGradMaps {          // a matrix of its own for every g
    CUtensorMap a[kMaxGroups], b[kMaxGroups];
    __device__ __forceinline__ const CUtensorMap* A(int, int g) const { return &a[g]; }
    __device__ __forceinline__ const CUtensorMap* B(int, int g) const { return &b[g]; }
    static __device__ __forceinline__ int z(int) { return 0; }
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

// An accumulator is free again: arrival on the barrier `bar` of the pair's leader.  What goes before
// it are TMEM loads, which tcgen05.wait::ld and the tcgen05 fence order, and nothing in memory is
// handed over: no release at cluster scope, which waits for the warp's stores and took most
// of a k-block's turn in the kSplit kernels (fp32 2048 x 8192, five steps, 2046 us and 1640).
__device__ __forceinline__ void arrive_leader(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cta.shared::cluster.b64 _, [%0];" ::"r"(
                     mapa_shared(bar, 0))
                 : "memory");
}

// ---------------------------------------------------------------------------
// Epilogues.  A warp has 32 rows x BN / 2 columns of a tile and takes them 32 columns at a time:
// the accumulator's chunk (one row per lane) goes through the warp's staging buffer, and each
// lane takes 4 columns of 8 rows back (access i: row 4 i + lane / 8), so that a global access of
// the warp covers 64 or 128 bytes of 4 rows.  (One row per lane touches 32 rows with every
// access: five steps on two 256 x 384 matrices took 116 us then, 100 us now.)  What a chunk
// reads is loaded two chunks ahead into one of two slots of registers (kSplit, whose sums fill
// them: one ahead).
template <bool kSplit>
constexpr int ns_slots() {
    return kSplit ? 1 : 2;
}

// The staged chunk: access i of this lane, and where it lies.
__device__ __forceinline__ uint32_t ns_piece(uint32_t buf, int lane, int i) {
    const uint32_t r = static_cast<uint32_t>(4 * i + lane / 8);
    return buf + r * 128u + (((lane % 8) ^ (r & 7u)) << 4);
}
__device__ __forceinline__ void ns_stage(uint32_t buf, int lane, const float (&v)[32]) {
    uint32_t u[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) u[j] = __float_as_uint(v[j]);
    out_stage_row(buf, lane, u);
    __syncwarp();
}

// Symmetric results S [M, M] of one matrix: s = lin_coef L + acc_coef acc, rounded to fp16 (with
// kSplit: high and low parts), to (row, col) and, off the diagonal blocks, to (col, row).  L
// null: no such term.  L and S are [M, ld], ld a multiple of 64; of the columns from M on, which
// nothing reads, a row gets what the last access over M writes.
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
    using Maps = NsMaps;
    static constexpr bool kBf16 = false;
    static constexpr int kRun = 0;
    static constexpr bool kRanges = kSplit;
    using Params = typename EpiSymBase<kSplit>::Params;
    static constexpr int kParts = kSplit ? 2 : 1;
    static constexpr int kChunks = BN / 2 / 32;

    // (by value: a reference to a kernel's parameters, kept in an object, turns into an address
    // that global loads do not accept)
    const __half* lin[kParts];  // of this matrix, or null
    __half* out[kParts];
    int M, ld;
    float lin_coef, acc_coef;
    int row0, col0, r0, c0;
    bool mirror;
    static constexpr int kAcc = 8, kSlots = ns_slots<kSplit>();
    uint2 l[kSlots][kParts][kAcc];

    __device__ __forceinline__ bool in(int i, int c) const {
        return r0 + 4 * i < M && c0 + 32 * c < M;
    }
    template <int SLOT>
    __device__ __forceinline__ void fetch(int c) {
        if (!lin[0]) return;
#pragma unroll
        for (int h = 0; h < kParts; ++h) {
#pragma unroll
            for (int i = 0; i < kAcc; ++i) {
                l[SLOT][h][i] = make_uint2(0u, 0u);
                if (in(i, c))
                    l[SLOT][h][i] = *reinterpret_cast<const uint2*>(
                        lin[h] + static_cast<long long>(r0 + 4 * i) * ld + c0 + 32 * c);
            }
        }
    }

    __device__ __forceinline__ EpiSym(const Params& p, int g, int row0_, int col0_, int lane,
                                      bool mirror_)
        : M(p.M), ld(p.ld), lin_coef(p.lin_coef), acc_coef(p.acc_coef), row0(row0_), col0(col0_),
          r0(row0_ + lane / 8), c0(col0_ + 4 * (lane % 8)), mirror(mirror_) {
        const long long base = g * p.stride;
#pragma unroll
        for (int h = 0; h < kParts; ++h) {
            lin[h] = p.lin[h] ? p.lin[h] + base : nullptr;
            out[h] = p.out[h] + base;
        }
        fetch<0>(0);
        if constexpr (kSlots == 2) fetch<1>(1);
    }

    __device__ __forceinline__ void finish(int) {}

    template <int SLOT>
    __device__ __forceinline__ void chunk(const float (&v)[32], uint32_t buf, int lane, int c) {
        ns_stage(buf, lane, v);
#pragma unroll
        for (int i = 0; i < kAcc; ++i) {
            const uint32_t at = ns_piece(buf, lane, i);
            float4 a = ld_shared_f4(at);
            a = make_float4(a.x * acc_coef, a.y * acc_coef, a.z * acc_coef, a.w * acc_coef);
            if (lin[0]) {
#pragma unroll
                for (int h = 0; h < kParts; ++h) {
                    const float2 f0 = unpack_f16x2(l[SLOT][h][i].x), f1 = unpack_f16x2(l[SLOT][h][i].y);
                    a.x = fmaf(lin_coef, f0.x, a.x);
                    a.y = fmaf(lin_coef, f0.y, a.y);
                    a.z = fmaf(lin_coef, f1.x, a.z);
                    a.w = fmaf(lin_coef, f1.y, a.w);
                }
            }
            if (mirror)
                st_shared_v4(at, __float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(a.z),
                             __float_as_uint(a.w));
#pragma unroll
            for (int h = 0; h < kParts; ++h) {
                const uint2 w = make_uint2(pack_f16x2(a.x, a.y), pack_f16x2(a.z, a.w));
                if (in(i, c))
                    *reinterpret_cast<uint2*>(out[h] + static_cast<long long>(r0 + 4 * i) * ld + c0 +
                                              32 * c) = w;
                if constexpr (kSplit) {
                    const float2 f0 = unpack_f16x2(w.x), f1 = unpack_f16x2(w.y);
                    a = make_float4(a.x - f0.x, a.y - f0.y, a.z - f1.x, a.w - f1.y);
                }
            }
        }
        if (mirror) {  // the block is turned over: a lane's row becomes 32 elements of a column
            __syncwarp();
            const int row = row0 + lane, col = col0 + 32 * c;
            if (row < M) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float4 f = ld_shared_f4(buf + lane * 128u + ((k ^ (lane & 7)) << 4));
                    const float e[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (col + 4 * k + j >= M) continue;
                        const long long o = static_cast<long long>(col + 4 * k + j) * ld + row;
                        const __half hi = __float2half_rn(e[j]);
                        out[0][o] = hi;
                        if constexpr (kSplit) out[1][o] = __float2half_rn(e[j] - __half2float(hi));
                    }
                }
            }
        }
        if constexpr (kSlots == 2) {
            if (c + 2 < kChunks) fetch<SLOT>(c + 2);
        } else {
            if (c + 1 < kChunks) fetch<SLOT>(c + 1);
        }
        __syncwarp();
    }
};

// ---------------------------------------------------------------------------
// X' = lin_coef X + acc_coef acc over [M, N] (row stride ld, a multiple of 64; the columns from N
// on as in EpiSym).  What becomes of it:
//   kNext     the next X: its high part, and its low part (not kSplit: for the linear term
//             only) or (kSplit) low part and the fp32 value
//   kResult   O [M, N] (row stride N) in bf16
//   kResult32 O in fp32
// The linear term takes X in more bits than the operands have: of a direction in which X is
// small B X is next to nothing, so a X carries it, 3.4 times larger after every step, and with
// it any rounding of X (fp16: up to 10% of the result for a matrix of low rank).  fp16 reads
// the low part where it was kept (lin_lo), kSplit the fp32 value.
enum NsOut { kNext = 0, kResult = 1, kResult32 = 2 };

struct NsApplyStep {      // what changes from step to step
    const __half* hi;     // X (fp16)
    const __half* lo;     // X's low part, read if lin_lo
    __half* next_hi;      // kNext
    __half* next_lo;      // kNext, or null (may be lo)
    float lin_coef, acc_coef;
    bool lin_lo;
};

template <bool kSplit, int kOut>
struct EpiApplyBase {
    using Out = std::conditional_t<kOut == kResult, __nv_bfloat16, float>;
    struct Params {
        NsApplyStep s;
        float* x32;           // kSplit: X in fp32, updated in place (kNext)
        long long stride;     // of one matrix in a batch
        int M, N, ld;
        Out* out[kMaxGroups];          // kResult, kResult32: O
    };
};

template <int BN, bool kSplit, int kOut>
struct EpiApply : EpiApplyBase<kSplit, kOut> {
    using Maps = NsMaps;
    static constexpr bool kBf16 = false;
    static constexpr int kRun = 0;
    static constexpr bool kRanges = false;
    using Out = typename EpiApplyBase<kSplit, kOut>::Out;
    using Params = typename EpiApplyBase<kSplit, kOut>::Params;
    static constexpr int kChunks = BN / 2 / 32;
    static constexpr int kAcc = 8, kSlots = ns_slots<kSplit>();

    // (by value, as in EpiSym)
    const __half *hi_p, *lo_p;   // of this matrix, from its first element
    __half *next_hi, *next_lo;   // kNext (next_lo: or null)
    float* x32;                  // kSplit
    Out* out;                    // kResult, kResult32
    int M, N, ld;
    float lin_coef, acc_coef;
    int r0, c0;
    uint2 hi[kSlots][kSplit ? 1 : kAcc], lo[kSlots][kSplit ? 1 : kAcc];
    float4 x[kSplit ? kAcc : 1];

    __device__ __forceinline__ bool in(int i, int c) const {
        return r0 + 4 * i < M && c0 + 32 * c < N;
    }
    // 4 elements of a row of N from column col, those inside it (N > col)
    __device__ __forceinline__ void st4(float* q, const float4& v, int col) const {
        if ((N & 3) == 0) {
            *reinterpret_cast<float4*>(q) = v;
            return;
        }
        q[0] = v.x;
        if (col + 1 < N) q[1] = v.y;
        if (col + 2 < N) q[2] = v.z;
        if (col + 3 < N) q[3] = v.w;
    }
    // (N is a multiple of 8 for bf16)
    __device__ __forceinline__ void st4(__nv_bfloat16* q, const float4& v, int) const {
        *reinterpret_cast<uint2*>(q) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    }

    template <int SLOT>
    __device__ __forceinline__ void fetch(int c) {
#pragma unroll
        for (int i = 0; i < kAcc; ++i) {
            const bool ok = in(i, c);
            const long long o = static_cast<long long>(r0 + 4 * i) * ld + c0 + 32 * c;
            if constexpr (kSplit) {
                x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (ok) x[i] = *reinterpret_cast<const float4*>(x32 + o);
            } else {
                hi[SLOT][i] = lo[SLOT][i] = make_uint2(0u, 0u);
                if (ok) hi[SLOT][i] = *reinterpret_cast<const uint2*>(hi_p + o);
                if (ok && lo_p) lo[SLOT][i] = *reinterpret_cast<const uint2*>(lo_p + o);
            }
        }
    }

    __device__ __forceinline__ EpiApply(const Params& p, int g, int row0, int col0, int lane, bool)
        : EpiApply(p, p.s, g, row0, col0, lane) {}
    __device__ __forceinline__ EpiApply(const Params& p, const NsApplyStep& s, int g, int row0,
                                        int col0, int lane)
        : M(p.M), N(p.N), ld(p.ld), lin_coef(s.lin_coef), acc_coef(s.acc_coef),
          r0(row0 + lane / 8), c0(col0 + 4 * (lane % 8)) {
        const long long base = g * p.stride;
        hi_p = s.hi + base;
        lo_p = s.lin_lo ? s.lo + base : nullptr;
        if constexpr (kOut == kNext) {
            next_hi = s.next_hi + base;
            next_lo = s.next_lo ? s.next_lo + base : nullptr;
        } else {
            out = p.out[g];
        }
        if constexpr (kSplit) x32 = p.x32 + base;
        fetch<0>(0);
        if constexpr (kSlots == 2) fetch<1>(1);
    }

    __device__ __forceinline__ void finish(int) {}

    template <int SLOT>
    __device__ __forceinline__ void chunk(const float (&v)[32], uint32_t buf, int lane, int c) {
        ns_stage(buf, lane, v);
#pragma unroll
        for (int i = 0; i < kAcc; ++i) {
            float4 a = ld_shared_f4(ns_piece(buf, lane, i));
            float4 xl;
            if constexpr (kSplit) {
                xl = x[i];
            } else {
                const float2 h0 = unpack_f16x2(hi[SLOT][i].x), h1 = unpack_f16x2(hi[SLOT][i].y);
                xl = make_float4(h0.x, h0.y, h1.x, h1.y);
                if (lo_p) {
                    const float2 l0 = unpack_f16x2(lo[SLOT][i].x), l1 = unpack_f16x2(lo[SLOT][i].y);
                    xl.x += l0.x;
                    xl.y += l0.y;
                    xl.z += l1.x;
                    xl.w += l1.y;
                }
            }
            a.x = fmaf(lin_coef, xl.x, a.x * acc_coef);
            a.y = fmaf(lin_coef, xl.y, a.y * acc_coef);
            a.z = fmaf(lin_coef, xl.z, a.z * acc_coef);
            a.w = fmaf(lin_coef, xl.w, a.w * acc_coef);
            if (!in(i, c)) continue;
            const int row = r0 + 4 * i, col = c0 + 32 * c;
            if constexpr (kOut == kNext) {
                const long long o = static_cast<long long>(row) * ld + col;
                const uint2 h = make_uint2(pack_f16x2(a.x, a.y), pack_f16x2(a.z, a.w));
                *reinterpret_cast<uint2*>(next_hi + o) = h;
                if (next_lo) {
                    const float2 h0 = unpack_f16x2(h.x), h1 = unpack_f16x2(h.y);
                    *reinterpret_cast<uint2*>(next_lo + o) =
                        make_uint2(pack_f16x2(a.x - h0.x, a.y - h0.y),
                                   pack_f16x2(a.z - h1.x, a.w - h1.y));
                }
                if constexpr (kSplit) *reinterpret_cast<float4*>(x32 + o) = a;
            } else {
                const long long o = static_cast<long long>(row) * N + col;
                st4(out + o, a, col);
            }
        }
        if constexpr (kSlots == 2) {
            if (c + 2 < kChunks) fetch<SLOT>(c + 2);
        } else {
            if (c + 1 < kChunks) fetch<SLOT>(c + 1);
        }
        __syncwarp();
    }
};

// ---------------------------------------------------------------------------
// The pseudogradient G = g^T A of bf16 operands and the momentum: M <- mu M + G, U = G + mu M
// (nesterov) or M, both fp32 [M, N] (N a multiple of 8), and the sum of U's squares over the
// warp's part of the tile to part[matrix][tile][16 warps of the pair].  (A pass over G, M and U behind
// the library's EpiStoreGroupF32 took 97 us by itself for two 8192 x 2048 matrices.)
//
// M is a state in fp32, and the tensor core truncates its sums: with 4096 tokens in one accumulator
// M was 3.4e-6 off in norm, six times an fp32 product's error (all products positive: 1.4e-5).  So
// the accumulator is drained every 512 tokens: 4.8e-7 (7.1e-7) for any number of tokens, beside
// an fp32 product's 2e-7 to 1.5e-6.  The MMAs then run two runs ahead of an epilogue, where they
// were a whole tile ahead: two 4096 x 11008 layers 536 us, 476 without (of 5.3 ms), two 8192 x 2048
// of 2048 tokens 135 and 114 (of 1.16).
struct EpiMomentumBase {
    struct Params {
        float* M[kMaxGroups];
        float* U;             // [groups], u_stride apart
        long long u_stride;
        double* part;
        int rows, cols, m_blocks, n_blocks;
        float mu;
        bool nesterov;
    };
};

// Sum of 4 squares where fp32 neither overflows nor loses digits to underflow; else 0, and the
// fp64 sum is added to `exact`.
__device__ __forceinline__ float square_sum4(const float4& v, double& exact) {
    const float s = fmaf(v.x, v.x, fmaf(v.y, v.y, fmaf(v.z, v.z, v.w * v.w)));
    if (s >= 1e-30f && s <= 1e30f) return s;
    if (((__float_as_uint(v.x) | __float_as_uint(v.y) | __float_as_uint(v.z) |
          __float_as_uint(v.w)) << 1) != 0)
        exact += static_cast<double>(v.x) * v.x + static_cast<double>(v.y) * v.y +
                 static_cast<double>(v.z) * v.z + static_cast<double>(v.w) * v.w;
    return 0.f;
}

template <int BN>
struct EpiMomentum : EpiMomentumBase {
    using Maps = NsGradMaps;
    static constexpr bool kBf16 = true;
    static constexpr int kRun = 4;  // stages of 128 tokens
    static constexpr bool kRanges = false;
    static constexpr int kChunks = BN / 2 / 32;
    static constexpr int kAcc = 8;

    float *M, *U;      // (by value, as in EpiSym)
    double* slot;
    int r0, c0, rows, cols;
    float mu;
    bool nesterov;
    double squares;
    float4 m[kAcc];    // M of the next chunk

    __device__ __forceinline__ bool in(int i, int c) const {
        return r0 + 4 * i < rows && c0 + 32 * c < cols;
    }
    __device__ __forceinline__ long long at(int i, int c) const {
        return static_cast<long long>(r0 + 4 * i) * cols + c0 + 32 * c;
    }
    __device__ __forceinline__ void fetch(int c) {
#pragma unroll
        for (int i = 0; i < kAcc; ++i) {
            m[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (in(i, c)) m[i] = *reinterpret_cast<const float4*>(M + at(i, c));
        }
    }
    __device__ __forceinline__ EpiMomentum(const Params& p, int g, int row0, int col0, int lane, bool)
        : M(p.M[g]), U(p.U + g * p.u_stride), r0(row0 + lane / 8), c0(col0 + 4 * (lane % 8)),
          rows(p.rows), cols(p.cols), mu(p.mu), nesterov(p.nesterov), squares(0.0) {
        const int warps = 2 * kNsWarps;  // of a tile: 8 blocks of 32 rows x 2 halves of the columns
        const long long tile = (static_cast<long long>(g) * p.m_blocks + row0 / kPairBM) * p.n_blocks +
                               col0 / BN;
        slot = p.part + tile * warps + row0 % kPairBM / 32 * 2 + col0 % BN / (BN / 2);
        fetch(0);
    }
    template <int SLOT>
    __device__ __forceinline__ void chunk(const float (&v)[32], uint32_t buf, int lane, int c) {
        ns_stage(buf, lane, v);
        float run = 0.f;
#pragma unroll
        for (int i = 0; i < kAcc; ++i) {
            const float4 g = ld_shared_f4(ns_piece(buf, lane, i));
            float4 a = m[i];
            a.x = fmaf(mu, a.x, g.x);
            a.y = fmaf(mu, a.y, g.y);
            a.z = fmaf(mu, a.z, g.z);
            a.w = fmaf(mu, a.w, g.w);
            float4 u = a;
            if (nesterov) {
                u.x = fmaf(mu, a.x, g.x);
                u.y = fmaf(mu, a.y, g.y);
                u.z = fmaf(mu, a.z, g.z);
                u.w = fmaf(mu, a.w, g.w);
            }
            if (in(i, c)) {
                *reinterpret_cast<float4*>(M + at(i, c)) = a;
                *reinterpret_cast<float4*>(U + at(i, c)) = u;
                run += square_sum4(u, squares);
            }
        }
        squares += run;
        if (c + 1 < kChunks) fetch(c + 1);
        __syncwarp();
    }
    __device__ __forceinline__ void finish(int lane) {
        double t = squares;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        if (lane == 0) *slot = t;
        __syncwarp();
    }
};

// ---------------------------------------------------------------------------
template <int BN, bool A_MN, bool B_MN, bool kSplit, class Epi>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(ns_threads<BN, kSplit, Epi>(), 1)
    ns_gemm_kernel(const __grid_constant__ typename Epi::Maps maps,
                   const __grid_constant__ typename Epi::Params ep, const NsShape sh,
                   unsigned int* status, unsigned long long wait_limit_ns) {
    using L = NsSmem<BN>;
    constexpr int kStages = L::kStages;
    constexpr int kSub = kSplit ? 1 : 2;   // k-blocks (and full barriers) per stage
    constexpr int kRun = ns_run<kSplit, Epi>();
    constexpr bool kDrained = kRun > 0;
    constexpr uint32_t kIdesc = Epi::kBf16 ? idesc_bf16_f32(kPairBM, BN, A_MN, B_MN)
                                           : idesc_f16_f32(kPairBM, BN, A_MN, B_MN);
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
    const int tile_k = (sh.g.k_blocks + kSub - 1) / kSub;  // stages per tile
    const int splits = Epi::kRanges ? sh.splits : 1;
    const long long units = sh.g.tiles * splits;
    // first stage of a unit's range
    auto first_k = [&](long long u, int add) {
        if (splits == 1) return add * tile_k;
        return static_cast<int>((u % splits + add) * tile_k / splits);
    };

    const uint32_t bar0 = sbase + L::kBarOffset;
    constexpr int kFull = kStages * kSub, kAccs = ns_accs<kSplit, BN>();
    constexpr int kFirst = ns_first_warp<BN, kSplit, Epi>();
    auto full_bar = [&](int s, int j) { return bar0 + 8u * (s * kSub + j); };
    auto empty_bar = [&](int s) { return bar0 + 8u * (kFull + s); };
    auto tfull_bar = [&](int a) { return bar0 + 8u * (kFull + kStages + a); };
    auto tempty_bar = [&](int a) { return bar0 + 8u * (kFull + kStages + kAccs + a); };
    const uint32_t drain_bar = bar0 + 8u * (kFull + kStages + 2 * kAccs);
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
        for (int a = 0; a < kAccs; ++a) {
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
        tmem_alloc_pair<kAccs * BN>(smem_u32(tmem_holder));
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;
    grid_dependency_wait();

    const WaitGuard guard{abort_flag, status, wait_limit_ns};

    if (warp < kFirst) {
        if constexpr (kFirst == 4) ns_fewer_registers<kNsFewRegs>();
        if (warp == 0) {
            // ------------------------------------------------------- TMA producer (both CTAs)
            if (lane == 0) {
                int stage = 0;
                uint32_t phase = 0, issued = 0;
                bool ok = true;
                for (long long u = cluster; ok && u < units; u += n_clusters) {
                    int g, mb, nb;
                    ns_tile<BN>(u / splits, sh, g, mb, nb);
                    const int a_row = mb * kPairBM + 128 * static_cast<int>(rank);
                    const int b_row = nb * BN + (BN / 2) * static_cast<int>(rank);
                    const int k1 = first_k(u, 1);
                    for (int kb = first_k(u, 0); kb < k1; ++kb) {
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
                            ns_load<A_MN, 128>(maps.A(part, g), sa + j * L::kABox, fb, a_row, k0, maps.z(g));
                            ns_load<B_MN, BN / 2>(maps.B(part, g), sb + j * L::kBBox, fb, b_row, k0, maps.z(g));
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
                for (long long u = cluster; ok && u < units; u += n_clusters) {
                    const int k0 = first_k(u, 0), k1 = first_k(u, 1);
                    for (int kb = k0; kb < k1; ++kb) {
                        bool first = kb == k0, last = kb == k1 - 1;  // of an accumulator
                        if constexpr (kDrained) {
                            first = (kb - k0) % kRun == 0;
                            last = last || (kb - k0) % kRun == kRun - 1;
                        }
                        if (first) {
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
                                                     (!first || j != 0 || kk != 0) ? 1u : 0u);
                                issued_any = true;
                            }
                            if (!ok) break;
                        }
                        issued_any = true;
                        tc_commit_pair_multicast(empty_bar(stage), kBoth);
                        if (++stage == kStages) { stage = 0; phase ^= 1u; }
                        if (last) {
                            tc_commit_pair_multicast(tfull_bar(acc), kBoth);
                            if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
                        }
                    }
                }
                if (issued_any) {
                    tc_commit_pair_multicast(drain_bar, 0x1);
                    mbar_wait_cl_drain(drain_bar, 0, kDrainLimitNs);
                }
            }
            __syncwarp();
        }
    } else {
        if constexpr (kFirst == 4) ns_more_registers<kNsManyRegs>();
        // ------------------------------------------------------- epilogue (both CTAs)
        const int q = warp & 3;               // TMEM lanes [32 q, 32 q + 32)
        const int half = (warp - kFirst) / 4;
        constexpr int kWarpCols = BN / 2;     // columns [kWarpCols half, kWarpCols (half + 1))
        const uint32_t buf = sbase + L::kOutOffset + static_cast<uint32_t>(warp - kFirst) * kOutBufBytes;
        int acc = 0;
        uint32_t acc_phase = 0;
        // One answer for the warp, whose lanes poll one by one; it is together again after lane 0's
        // arrival, and at every load of the accumulator (tmem_ld_32x32b_x32).
        auto ready = [&] {
            const bool in_time = mbar_wait_cl(tfull_bar(acc), acc_phase, guard);
            if (!__all_sync(0xffffffffu, in_time)) return false;
            tc_fence_after();
            return true;
        };
        auto release = [&] {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_leader(tempty_bar(acc));
            __syncwarp();
            if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
        };
        auto t_row = [&] {
            return tmem_base + (static_cast<uint32_t>(q * 32) << 16) +
                   static_cast<uint32_t>(acc * BN + half * kWarpCols);
        };
        constexpr int kChunks = kWarpCols / 32;
        bool ok = true;
        for (long long u = cluster; ok && u < units; u += n_clusters) {
            const long long t = u / splits;
            int g, mb, nb;
            ns_tile<BN>(t, sh, g, mb, nb);
            const int row0 = mb * kPairBM + 128 * static_cast<int>(rank) + 32 * q;
            const int col0 = nb * BN + half * kWarpCols;
            const bool mirror = sh.tri && nb * BN / kPairBM != mb;
            if constexpr (kDrained) {
                // the sums of the unit's accumulators, a run of stages each, in registers
                float s[kChunks][32];
                auto drain = [&] {
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
#pragma unroll
                        for (int j = 0; j < 32; ++j) s[c][j] = 0.f;
                    const int k1 = first_k(u, 1);
                    for (int kb = first_k(u, 0); kb < k1; kb += kRun) {
                        if (!ready()) return false;
                        const uint32_t tr = t_row();
#pragma unroll
                        for (int c = 0; c < kChunks; ++c) {
                            float v[32];
                            tmem_ld_32x32b_x32(tr + 32 * c, v);
                            if (c == kChunks - 1) release();  // it is all in registers
#pragma unroll
                            for (int j = 0; j < 32; ++j) s[c][j] += v[j];
                        }
                    }
                    return true;
                };
                auto finish = [&](Epi& epi) {
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) epi.template chunk<0>(s[c], buf, lane, c);
                    epi.finish(lane);
                };
                if constexpr (!kSplit) {
                    Epi epi(ep, g, row0, col0, lane, mirror);  // (its first loads arrive meanwhile)
                    ok = drain();
                    if (!ok) break;
                    finish(epi);
                } else {
                    ok = drain();
                    if (!ok) break;
                    if constexpr (Epi::kRanges) {
                        if (splits > 1) {
                            constexpr int kWarpSums = kChunks * 32 * 32;
                            const int w = static_cast<int>(rank) * kNsWarps + warp - kFirst;
                            float* mine = sh.slots + (u * 2 * kNsWarps + w) * kWarpSums + lane;
#pragma unroll
                            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                                for (int j = 0; j < 32; ++j) mine[(c * 32 + j) * 32] = s[c][j];
                            __threadfence();
                            __syncwarp();
                            unsigned* count = sh.counts + t * 2 * kNsWarps + w;
                            unsigned before = 0;
                            if (lane == 0) before = atomicAdd(count, 1u);
                            before = __shfl_sync(0xffffffffu, before, 0);
                            if (before + 1 != static_cast<unsigned>(splits)) continue;
                            __threadfence();
                            if (lane == 0) *count = 0;
#pragma unroll
                            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                                for (int j = 0; j < 32; ++j) s[c][j] = 0.f;
                            const float* from =
                                sh.slots + (t * splits * 2 * kNsWarps + w) * kWarpSums + lane;
                            for (int r = 0; r < splits; ++r) {
#pragma unroll
                                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                                    for (int j = 0; j < 32; ++j)
                                        s[c][j] += __ldcg(from + (c * 32 + j) * 32);
                                from += 2 * kNsWarps * kWarpSums;
                            }
                        }
                    }
                    Epi epi(ep, g, row0, col0, lane, mirror);
                    finish(epi);
                }
            } else {
                Epi epi(ep, g, row0, col0, lane, mirror);
                ok = ready();
                if (!ok) break;
                const uint32_t tr = t_row();
#pragma unroll 1
                for (int c = 0; c < kChunks; c += 2) {
                    float v[32];
                    tmem_ld_32x32b_x32(tr + 32 * c, v);
                    epi.template chunk<0>(v, buf, lane, c);
                    tmem_ld_32x32b_x32(tr + 32 * c + 32, v);
                    if (c == kChunks - 2) release();
                    epi.template chunk<1>(v, buf, lane, c + 1);
                }
                epi.finish(lane);
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
        tmem_dealloc_pair<kAccs * BN>(tmem_base);
    }
}

// ---------------------------------------------------------------------------
// The whole iteration in one launch, for fp16 batches whose products have at most one 256 x 128
// tile per resident cluster: there a launch per product (15 of them) costs 7 us each, most of it
// set-up, the wait for the kernel before and the first operand's way in.  The roles walk the
// products ("phases": A, B, X of every step) with one counter in global memory between them:
// every block adds one when its stores of a phase are done, and the producers and epilogues of
// the next phase wait until all have.  A cooperative launch: every cluster is resident.  The
// waits are bounded like the barriers'.
struct NsChainStep {
    float a_acc;             // A = a_acc acc
    float b_lin, b_acc;      // B = b_lin A + b_acc acc
    float x_lin, x_acc;      // X' = x_lin X + x_acc acc
};
constexpr int kNsMaxSteps = 32;

template <int kOut>
struct NsChainParams {
    CUtensorMap map[3][2][2];  // operands of the phases: [A, B, X][X buffer][A operand, B operand]
    typename EpiApplyBase<false, kOut>::Params ap;  // of the last step (s unused)
    NsChainStep step[kNsMaxSteps];
    __half* A;
    __half* B;
    __half* hi[2];
    __half* lo[2];
    long long ms;            // elements of one A
    int m, ldm, steps, groups, rows, cols;
    bool tall;
    unsigned* count;         // zero at the start
};

__device__ __forceinline__ unsigned ld_acquire_u32(const unsigned* p) {
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// Until *count reaches `target` (one thread); false: given up.
__device__ __forceinline__ bool ns_wait_count(const unsigned* count, unsigned target,
                                              const WaitGuard& g) {
    if (ld_acquire_u32(count) >= target) return true;
    const uint64_t t0 = global_timer_ns();
    for (uint32_t i = 1;; ++i) {
        if (ld_acquire_u32(count) >= target) return true;
        if ((i & 31u) == 0) {
            if (*g.abort_flag) return false;
            if (global_timer_ns() - t0 > g.limit_ns) {
                *g.abort_flag = 1;
                if (g.status) atomicOr(g.status, kDevTimeout);
                return false;
            }
        }
    }
}

// Orders global-memory accesses of this thread through the generic proxy with those of TMA.
__device__ __forceinline__ void fence_proxy_async_global() {
    asm volatile("fence.proxy.async.global;" ::: "memory");
}

template <int kOut>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kNsThreads, 1)
    ns_chain_kernel(const __grid_constant__ NsChainParams<kOut> p, unsigned int* status,
                    unsigned long long wait_limit_ns) {
    constexpr int BN = 128;
    using L = NsSmem<BN>;
    constexpr int kStages = L::kStages;
    constexpr int kSub = 2;
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

    const uint32_t bar0 = sbase + L::kBarOffset;
    constexpr int kFull = kStages * kSub, kAccs = ns_accs<false>();
    auto full_bar = [&](int s, int j) { return bar0 + 8u * (s * kSub + j); };
    auto empty_bar = [&](int s) { return bar0 + 8u * (kFull + s); };
    auto tfull_bar = [&](int a) { return bar0 + 8u * (kFull + kStages + a); };
    auto tempty_bar = [&](int a) { return bar0 + 8u * (kFull + kStages + kAccs + a); };
    const uint32_t drain_bar = bar0 + 8u * (kFull + kStages + 2 * kAccs);
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
        for (int a = 0; a < kAccs; ++a) {
            mbar_init(tfull_bar(a), 1);
            mbar_init(tempty_bar(a), 2 * kNsWarps);
        }
        mbar_init(drain_bar, 1);
        *abort_flag = 0;
        *issued_word = 0;
        fence_mbar_init();
        for (int f = 0; f < 3; ++f)  // (1% of two 1024 x 1024)
            for (int k = 0; k < 4; ++k) tma_prefetch_desc(&p.map[f][k / 2][k % 2]);
    }
    if (warp == 1) {
        tmem_alloc_pair<kAccs * BN>(smem_u32(tmem_holder));
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;

    const WaitGuard guard{abort_flag, status, wait_limit_ns};

    // Phase f: 0 A, 1 B, 2 X of step f / 3.  (Closures hold copies of the parameters they use.)
    auto shape = [m = p.m, rows = p.rows, cols = p.cols, groups = p.groups, tall = p.tall](int f) {
        NsShape sh = {};
        const bool sym = f % 3 != 2;
        sh.tri = sym;
        sh.g.M = sym ? m : rows;
        sh.g.N = sym ? m : cols;
        sh.g.K = f % 3 == 0 ? (tall ? rows : cols) : m;
        sh.g.m_blocks = (sh.g.M + kPairBM - 1) / kPairBM;
        sh.g.n_blocks = (sh.g.N + BN - 1) / BN;
        sh.g.k_blocks = (sh.g.K + kBK - 1) / kBK;
        sh.g.groups = groups;
        sh.g.band = 16;
        sh.g.tiles = static_cast<long long>(groups) *
                     (sym ? sh.g.m_blocks * (sh.g.m_blocks + 1) / 2 * (kPairBM / BN)
                          : sh.g.m_blocks * sh.g.n_blocks);
        return sh;
    };
    const int phases = 3 * p.steps;
    const unsigned arrivals = gridDim.x;  // of a phase

    if (warp == 0) {
        // ------------------------------------------------------- TMA producer (both CTAs)
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, issued = 0;
            bool ok = true;
            for (int f = 0; ok && f < phases; ++f) {
                const NsShape sh = shape(f);
                if (cluster >= sh.g.tiles) continue;
                if (!ns_wait_count(p.count, f * arrivals, guard)) break;
                fence_proxy_async_global();
                const CUtensorMap(&mp)[2] = p.map[f % 3][(f / 3) & 1];
                const bool a_mn = f % 3 == 0 && p.tall;
                const bool b_mn = f % 3 == 0 ? p.tall : f % 3 == 2 && !p.tall;
                const int stages_k = (sh.g.k_blocks + kSub - 1) / kSub;
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
                            const uint32_t fb = mapa_shared(full_bar(stage, j), 0);
                            if (leader)
                                mbar_arrive_expect_tx(full_bar(stage, j),
                                                      2 * (L::kStageBytes / kSub));
                            const int k0 = (2 * kb + j) * kBK;
                            if (a_mn)
                                ns_load<true, 128>(&mp[0], sa + j * L::kABox, fb, a_row, k0, g);
                            else
                                ns_load<false, 128>(&mp[0], sa + j * L::kABox, fb, a_row, k0, g);
                            if (b_mn)
                                ns_load<true, BN / 2>(&mp[1], sb + j * L::kBBox, fb, b_row, k0, g);
                            else
                                ns_load<false, BN / 2>(&mp[1], sb + j * L::kBBox, fb, b_row, k0, g);
                        }
                        ++issued;
                        if (++stage == kStages) { stage = 0; phase ^= 1u; }
                    }
                }
            }
            *issued_word = issued;
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------- pair MMA (leader only)
        if (leader && lane == 0) {
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool ok = true, issued_any = false;
            // the MMAs of one stage (one k-block of it: j) with the operands' layouts
            auto stage_mmas = [&](auto amn, auto bmn, uint32_t d_tmem, uint32_t sa, uint32_t sb, int j,
                                  bool first) {
                constexpr bool A_MN = decltype(amn)::value, B_MN = decltype(bmn)::value;
                constexpr uint32_t kIdesc = idesc_f16_f32(kPairBM, BN, A_MN, B_MN);
#pragma unroll
                for (int kk = 0; kk < kBK / kUmmaK; ++kk)
                    tc_mma_bf16_pair(d_tmem, operand_desc<A_MN>(sa + j * L::kABox, kk),
                                     operand_desc<B_MN>(sb + j * L::kBBox, kk), kIdesc,
                                     (!first || kk != 0) ? 1u : 0u);
            };
            for (int f = 0; ok && f < phases; ++f) {
                const NsShape sh = shape(f);
                const int stages_k = (sh.g.k_blocks + kSub - 1) / kSub;
                const bool both_mn = f % 3 == 0 && p.tall, b_mn = f % 3 == 2 && !p.tall;
                for (long long t = cluster; ok && t < sh.g.tiles; t += n_clusters) {
                    for (int kb = 0; kb < stages_k; ++kb) {
                        if (kb == 0) {
                            if (!mbar_wait_cl(tempty_bar(acc), acc_phase ^ 1u, guard)) {
                                ok = false;
                                break;
                            }
                            tc_fence_after();
                        }
                        const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(acc * BN);
                        const uint32_t sa = sbase + stage * L::kStageBytes, sb = sa + 2 * L::kABox;
#pragma unroll
                        for (int j = 0; j < kSub; ++j) {
                            // (not mbar_wait_cl_poll: this wait spans the wait between phases)
                            if (!mbar_wait_cl(full_bar(stage, j), phase, guard)) { ok = false; break; }
                            tc_fence_after();
                            const bool first = kb == 0 && j == 0;
                            if (both_mn)
                                stage_mmas(std::true_type{}, std::true_type{}, d_tmem, sa, sb, j, first);
                            else if (b_mn)
                                stage_mmas(std::false_type{}, std::true_type{}, d_tmem, sa, sb, j, first);
                            else
                                stage_mmas(std::false_type{}, std::false_type{}, d_tmem, sa, sb, j, first);
                            issued_any = true;
                        }
                        if (!ok) break;
                        tc_commit_pair_multicast(empty_bar(stage), kBoth);
                        if (++stage == kStages) { stage = 0; phase ^= 1u; }
                        if (kb == stages_k - 1) {
                            tc_commit_pair_multicast(tfull_bar(acc), kBoth);
                            if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
                        }
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
        const int q = warp & 3;
        const int half = (warp - 2) / 4;
        constexpr int kWarpCols = BN / 2;
        constexpr int kChunks = kWarpCols / 32;
        const uint32_t buf = sbase + L::kOutOffset + static_cast<uint32_t>(warp - 2) * kOutBufBytes;
        int acc = 0;
        uint32_t acc_phase = 0;
        bool ok = true;
        auto release = [&] {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_leader(tempty_bar(acc));
            __syncwarp();
            if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
        };
        // the sums of one tile through `epi`
        auto tile = [&](auto&& epi) {
            auto t_row = [&] {
                return tmem_base + (static_cast<uint32_t>(q * 32) << 16) +
                       static_cast<uint32_t>(acc * BN + half * kWarpCols);
            };
            auto ready = [&] {  // (as in ns_gemm_kernel)
                const bool in_time = mbar_wait_cl(tfull_bar(acc), acc_phase, guard);
                if (!__all_sync(0xffffffffu, in_time)) return false;
                tc_fence_after();
                return true;
            };
            if (!ready()) return false;
            static_assert(kChunks == 2, "one chunk per slot");
            const uint32_t tr = t_row();
            float v[32];
            tmem_ld_32x32b_x32(tr, v);
            epi.template chunk<0>(v, buf, lane, 0);
            tmem_ld_32x32b_x32(tr + 32, v);
            release();
            epi.template chunk<1>(v, buf, lane, 1);
            return true;
        };
        // the 8 warps' own barrier; all of them reach it twice in every phase, also after giving up
        auto epilogue_sync = [&] {
            __syncwarp();
            asm volatile("bar.sync 1, %0;" ::"n"(32 * kNsWarps) : "memory");
        };
        for (int f = 0; f < phases; ++f) {
            const NsShape sh = shape(f);
            const int k = f / 3, cur = k & 1;
            const bool last = k == p.steps - 1;
            // one thread of the block polls (a failure is in the abort flag); every block waits
            // here, also one without a tile: none may count for a phase ahead of time
            if (warp == 2 && lane == 0 && ok) ns_wait_count(p.count, f * arrivals, guard);
            epilogue_sync();
            // (the flag may rise between the reads of two lanes: the warp goes on or gives up as one)
            ok = __all_sync(0xffffffffu, ok && !*abort_flag);
            for (long long t = cluster; ok && t < sh.g.tiles; t += n_clusters) {
                int g, mb, nb;
                ns_tile<BN>(t, sh, g, mb, nb);
                const int row0 = mb * kPairBM + 128 * static_cast<int>(rank) + 32 * q;
                const int col0 = nb * BN + half * kWarpCols;
                if (f % 3 != 2) {
                    typename EpiSymBase<false>::Params sp;
                    const bool gram = f % 3 == 0;
                    sp.lin[0] = gram ? nullptr : p.A;
                    sp.out[0] = gram ? p.A : p.B;
                    sp.stride = p.ms;
                    sp.M = p.m;
                    sp.ld = p.ldm;
                    sp.lin_coef = p.step[k].b_lin;
                    sp.acc_coef = gram ? p.step[k].a_acc : p.step[k].b_acc;
                    ok = tile(EpiSym<BN, false>(sp, g, row0, col0, lane, nb * BN / kPairBM != mb));
                } else {
                    NsApplyStep st;
                    st.hi = p.hi[cur];
                    st.lo = p.lo[cur];
                    st.next_hi = p.hi[cur ^ 1];
                    st.next_lo = k + 2 < p.steps ? p.lo[cur ^ 1] : nullptr;
                    st.lin_coef = p.step[k].x_lin;
                    st.acc_coef = p.step[k].x_acc;
                    st.lin_lo = !last;
                    if (last) {
                        ok = tile(EpiApply<BN, false, kOut>(p.ap, st, g, row0, col0, lane));
                    } else {
                        typename EpiApplyBase<false, kNext>::Params np;
                        np.stride = p.ap.stride;
                        np.M = p.rows;
                        np.N = p.cols;
                        np.ld = p.ap.ld;
                        ok = tile(EpiApply<BN, false, kNext>(np, st, g, row0, col0, lane));
                    }
                }
            }
            // the block's part of the phase is done, and visible to TMA
            fence_proxy_async_global();
            epilogue_sync();
            if (warp == 2 && lane == 0 && ok) {
                __threadfence();
                atomicAdd(p.count, 1u);
            }
            __syncwarp();
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
        tmem_dealloc_pair<kAccs * BN>(tmem_base);
    }
}

}  // namespace fpo
