// linear.cu -- the linear layer Y = act(X W^T + b) + R and its backward pass (bf16; the fp32
// products are in simt_f32.cu).
//
//   forward    Z = X W^T + b       M = T  N = N  K = K    A, B K-major
//   signal     dX = dZ W           M = T  N = K  K = N    A K-major, B MN-major
//   gradient   dW = dZ^T X         M = N  N = K  K = T    A, B MN-major
//
// Large batches run on the tiles of tc_gemm_pair.cuh, or where these are few of tc_gemm.cuh, with
// the epilogues of linear_epilogues.cuh.  Batches of at most kFewT tokens run on
// few_tokens_kernel, with the weights as the 128-row operand and the tokens along N, and forward
// with at most row_tokens on row_kernel.  What the layer's own activation does to the signal, and the
// bias gradient, are one pass over dY (signal_kernel).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <string.h>

#include "gemm_launch.cuh"
#include "internal.h"
#include "linear_epilogues.cuh"

namespace fpo {
namespace {

constexpr size_t kHead = 256;  // status word
size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// ------------------------------------------------------------------ few tokens
// Y^T = W X^T: 128 rows of the weights (features) by BT tokens per tile, one CTA each.  The
// tiles' k-steps, tile by tile, are one sequence of units that the CTAs share out evenly, so
// that every SM streams the same number of weight bytes whatever the number of tiles: CTA c has
// units [c U / C, (c + 1) U / C).  A tile that lies in one CTA's range goes from the accumulator
// to the output.  Of the others each CTA leaves its sums in scratch, and the warp that is the
// last of a tile's to do so (a counter per tile and quarter of its rows) adds them in CTA order,
// whichever it is: the sums do not depend on the order in which the CTAs finish, and no CTA
// waits for another.
//   warp 0      TMA producer: a k-step, two 64-deep k-blocks, of weights and tokens per stage
//   warp 1      TMEM, MMAs (128 x BT x 16)
//   warps 2..5  epilogue: one feature per lane
// Bound: the weights' bytes, with a fixed part of some 8 us; under that a CTA's own pace, some 540
// cycles for a k-block with a commit of its own however few columns it had, so that tiles which
// have an SM each are no faster for being narrow.  us on pair tiles and here, from
// memory, K 4096 to 11008 features and 11008 to 4096: 5 tokens 41.7 26.8, 38.4 25.2; 16 tokens 38.3
// 28.3, 34.9 25.8; 32 tokens 38.6 30.6, 35.2 27.9.  With 64 tokens 38.8 37.4, 36.6 32.8, but 1024 to
// 1024 features 15.3 16.4; with more the sums of the parts, one warp per 32 features, are slower
// than the whole product on pair tiles.
constexpr int kFewT = 32;

template <int BT>
struct FewSmem {
    static constexpr int kSub = 2;  // 64-deep k-blocks per stage
    static constexpr int kWBytes = kBM * kBK * 2;
    static constexpr int kXBytes = BT * kBK * 2;
    static constexpr int kStageBytes = kSub * (kWBytes + kXBytes);
    static constexpr int kFit = 221184 / kStageBytes;
    static constexpr int kStages = kFit < 12 ? kFit : 12;
    static constexpr int kBarOffset = kStages * kStageBytes;
    static constexpr int kNumBars = 2 * kStages + 5;
    static constexpr int kMiscOffset = kBarOffset + kNumBars * 8;
    static constexpr int kBytes = kMiscOffset + 16 + 1024;
};

struct FewShape {
    int T;               // tokens, at most BT
    int k_steps;
    long long units;     // tiles * k_steps
    float* scratch;      // [2 CTAs][BT][128]: slot 2 c + 1 has a tile's first k-steps
    unsigned* counters;  // [tiles][4], zero at the start
};

// CTA c's units, and the CTA of a unit.
__device__ __forceinline__ long long few_start(const FewShape& s, long long c, long long C) {
    return c * s.units / C;
}
__device__ __forceinline__ int few_owner(const FewShape& s, long long u, long long C) {
    return static_cast<int>(((u + 1) * C - 1) / s.units);
}

// One feature of the n tokens through the epilogue: consecutive lanes are consecutive
// features.  What it reads is loaded for all tokens before anything is stored (a load behind a store
// to memory that may be the same waits for itself alone: 128 tokens took 110 us instead of 35).
template <int kN>
__device__ __forceinline__ void few_load(const __nv_bfloat16* p, long long ld, int n, uint16_t (&u)[kN]) {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
    for (int j = 0; j < kN; ++j) u[j] = j < n ? q[j * ld] : 0;
}
__device__ __forceinline__ float bf16_bits(uint16_t u) {
    return __uint_as_float(static_cast<uint32_t>(u) << 16);
}
template <int kN>
__device__ __forceinline__ void few_out(const LinearOut& p, int feature, int n, float (&v)[kN]) {
    if (feature >= p.N) return;
    uint16_t r[kN];
    if (p.residual) few_load(p.residual + feature, p.ld, n, r);
    if (p.bias) {
        const float bias = __bfloat162float(p.bias[feature]);
#pragma unroll
        for (int j = 0; j < kN; ++j) v[j] += bias;
    }
    if (p.Z) {
#pragma unroll
        for (int j = 0; j < kN; ++j)
            if (j < n) p.Z[j * p.ld + feature] = __float2bfloat16_rn(v[j]);
    }
    with_act(p.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < kN; j += 2) {
            if (j >= n) break;
            const float2 y = act_value2<act.value>(make_float2(v[j], v[j + 1]));
            v[j] = y.x;
            v[j + 1] = y.y;
        }
    });
#pragma unroll
    for (int j = 0; j < kN; ++j)
        if (j < n) p.Y[j * p.ld + feature] = __float2bfloat16_rn(p.residual ? v[j] + bf16_bits(r[j]) : v[j]);
}
template <int kN>
__device__ __forceinline__ void few_out(const SlopeOut& p, int feature, int n, float (&v)[kN]) {
    if (feature >= p.N) return;
    if (p.z) {
        uint16_t z[kN];
        few_load(p.z + feature, p.ld, n, z);
        with_act(p.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < kN; j += 2) {
                if (j >= n) break;
                const float2 s = act_slope2<act.value>(make_float2(bf16_bits(z[j]), bf16_bits(z[j + 1])));
                v[j] *= s.x;
                v[j + 1] *= s.y;
            }
        });
    }
#pragma unroll
    for (int j = 0; j < kN; ++j)
        if (j < n) p.X[j * p.ld + feature] = __float2bfloat16_rn(v[j]);
}

template <int BT, bool W_MN, class Out>
__global__ void __launch_bounds__(192, 1)
    few_tokens_kernel(const __grid_constant__ CUtensorMap wmap,
                      const __grid_constant__ CUtensorMap xmap, const __grid_constant__ Out out,
                      const FewShape sh, unsigned* status, unsigned long long wait_limit_ns) {
    using L = FewSmem<BT>;
    constexpr int kStages = L::kStages, kSub = L::kSub;
    constexpr uint32_t kIdesc = idesc_bf16_f32(kBM, BT, W_MN, false);
    static_assert(BT <= 32, "one load of the accumulator");
    constexpr int kAccCols = 32;
    constexpr int kTmemCols = 2 * kAccCols;
    constexpr int kAhead = BT <= 16 ? 4 : 2;  // CTAs' sums in flight

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t pad = (1024u - (raw & 1023u)) & 1023u;
    uint8_t* smem = smem_raw + pad;
    const uint32_t sbase = raw + pad;
    const uint32_t bar0 = sbase + L::kBarOffset;
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
    auto tfull_bar = [&](int a) { return bar0 + 8u * (2 * kStages + a); };
    auto tempty_bar = [&](int a) { return bar0 + 8u * (2 * kStages + 2 + a); };
    const uint32_t drain_bar = bar0 + 8u * (2 * kStages + 4);
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem + L::kMiscOffset);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::kMiscOffset + 4);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull_bar(a), 1);
            mbar_init(tempty_bar(a), 4);
        }
        mbar_init(drain_bar, 1);
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&wmap);
        tma_prefetch_desc(&xmap);
    }
    if (warp == 1) {
        tmem_alloc<kTmemCols>(smem_u32(tmem_holder));
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;
    grid_dependency_wait();

    const WaitGuard guard{abort_flag, status, wait_limit_ns};
    const long long C = gridDim.x;
    const long long u0 = few_start(sh, blockIdx.x, C), u1 = few_start(sh, blockIdx.x + 1, C);
    const int tile0 = static_cast<int>(u0 / sh.k_steps), k0 = static_cast<int>(u0 % sh.k_steps);

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            uint32_t issued_mask = 0, issued_parity = 0;
            int tile = tile0, ks = k0;
            for (long long u = u0; u < u1; ++u) {
                if (!mbar_wait(empty_bar(stage), phase ^ 1u, guard)) break;
                const uint32_t sw = sbase + stage * L::kStageBytes, sx = sw + kSub * L::kWBytes;
                mbar_arrive_expect_tx(full_bar(stage), L::kStageBytes);
#pragma unroll
                for (int j = 0; j < kSub; ++j) {
                    const int k = (ks * kSub + j) * kBK;
                    load_operand<W_MN, kBM>(&wmap, sw + j * L::kWBytes, full_bar(stage),
                                            tile * kBM, k);
                    load_operand<false, BT>(&xmap, sx + j * L::kXBytes, full_bar(stage), 0, k);
                }
                issued_mask |= 1u << stage;
                issued_parity = (issued_parity & ~(1u << stage)) | (phase << stage);
                if (++stage == kStages) { stage = 0; phase ^= 1u; }
                if (++ks == sh.k_steps) { ks = 0; ++tile; }
            }
            grid_dependency_trigger();
            for (int s = 0; s < kStages; ++s)  // no copy lands in shared memory after exit
                if (issued_mask & (1u << s))
                    mbar_wait_drain(full_bar(s), (issued_parity >> s) & 1u, kDrainLimitNs);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool ok = true, issued_any = false;
            int ks = k0;
            for (long long u = u0; u < u1 && ok;) {
                const long long end = min(u1, u + sh.k_steps - ks);  // of this tile's segment
                if (!mbar_wait(tempty_bar(acc), acc_phase ^ 1u, guard)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(acc * kAccCols);
                bool first = true;
                for (; u < end; ++u) {
                    if (!mbar_wait(full_bar(stage), phase, guard)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sw = sbase + stage * L::kStageBytes, sx = sw + kSub * L::kWBytes;
#pragma unroll
                    for (int j = 0; j < kSub; ++j)
#pragma unroll
                        for (int kk = 0; kk < kBK / kUmmaK; ++kk)
                            tc_mma_bf16(d_tmem, operand_desc<W_MN>(sw + j * L::kWBytes, kk),
                                        operand_desc<false>(sx + j * L::kXBytes, kk), kIdesc,
                                        !first || j != 0 || kk != 0 ? 1u : 0u);
                    first = false;
                    issued_any = true;
                    tc_commit(empty_bar(stage));
                    if (++stage == kStages) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
                ks = 0;
                tc_commit(tfull_bar(acc));
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
            if (issued_any) {  // the MMAs issued end before TMEM and shared memory go away
                tc_commit(drain_bar);
                mbar_wait_drain(drain_bar, 0, kDrainLimitNs);
            }
        }
        __syncwarp();
    } else {
        const int q = warp & 3;  // TMEM lane quarter this warp may access
        int acc = 0;
        uint32_t acc_phase = 0;
        int tile = tile0, ks = k0;
        for (long long u = u0; u < u1;) {
            const long long end = min(u1, u + sh.k_steps - ks);
            const bool whole = ks == 0 && end - u == sh.k_steps;
            const int feature = tile * kBM + q * 32 + lane;
            const uint32_t t_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16) +
                                   static_cast<uint32_t>(acc * kAccCols);
            // one answer for the warp: its lanes wait, and run out of time, one by one
            auto ready = [&] {
                const bool in_time = mbar_wait(tfull_bar(acc), acc_phase, guard);
                if (!__all_sync(0xffffffffu, in_time)) return false;
                tc_fence_after();
                return true;
            };
            if (!ready()) break;
            float* slot = sh.scratch + static_cast<long long>(2 * blockIdx.x + (ks == 0)) * BT * kBM +
                          q * 32 + lane;
            float w[32], v[BT];
            tmem_ld_32x32b_x32(t_row, w);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(tempty_bar(acc));
#pragma unroll
            for (int j = 0; j < BT; ++j) v[j] = w[j];
            if (whole) {
                few_out(out, feature, sh.T, v);
            } else {
#pragma unroll
                for (int j = 0; j < BT; ++j)
                    if (j < sh.T) slot[j * kBM] = v[j];
                // the last of the tile's CTAs adds their sums
                const long long first_unit = static_cast<long long>(tile) * sh.k_steps;
                const int c0 = few_owner(sh, first_unit, C);
                const int c1 = few_owner(sh, first_unit + sh.k_steps - 1, C);
                __threadfence();
                __syncwarp();
                unsigned before = 0;
                if (lane == 0) before = atomicAdd(sh.counters + 4 * tile + q, 1u);
                before = __shfl_sync(0xffffffffu, before, 0);
                if (before == static_cast<unsigned>(c1 - c0)) {
                    __threadfence();
                    const float* part = sh.scratch + q * 32 + lane;
                    // (CTA c0 has the tile's first k-steps: its odd slot)
                    const float* s0 = part + static_cast<long long>(2 * c0 + 1) * BT * kBM;
#pragma unroll
                    for (int j = 0; j < BT; ++j) v[j] = j < sh.T ? __ldcg(s0 + j * kBM) : 0.f;
                    // several CTAs' loads in flight: one by one each waits for L2
#pragma unroll 1
                    for (int c = c0 + 1; c <= c1; c += kAhead) {
                        float x[kAhead][BT];
#pragma unroll
                        for (int i = 0; i < kAhead; ++i) {
                            const float* s = part + static_cast<long long>(2 * min(c + i, c1)) * BT * kBM;
#pragma unroll
                            for (int j = 0; j < BT; ++j) x[i][j] = j < sh.T ? __ldcg(s + j * kBM) : 0.f;
                        }
#pragma unroll
                        for (int i = 0; i < kAhead; ++i) {
                            if (c + i > c1) break;
#pragma unroll
                            for (int j = 0; j < BT; ++j) v[j] += x[i][j];
                        }
                    }
                    few_out(out, feature, sh.T, v);
                }
            }
            if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            u = end;
            ks = 0;
            ++tile;
        }
        __syncwarp();
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc<kTmemCols>(tmem_base);
    }
}

// The weights as an operand of few_tokens_kernel: 256 bytes of a row at a time from DRAM (two
// k-blocks, the second of which the same SM wants next).
bool map_weights(CUtensorMap* m, const void* W, int rows, int cols, int box_rows) {
    const EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    cuuint64_t strides[1] = {static_cast<cuuint64_t>(cols) * 2};
    cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)};
    cuuint32_t es[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(W), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int sm_count() {
    DevInfo di;
    return current_device_info(&di) ? di.sm_count : 152;
}

// The tiles and k-steps of a problem of M features, and its CTAs: one per SM while each has at
// least 2 k-steps.
struct FewPlan {
    int k_steps;
    long long tiles, units, ctas;
};
FewPlan few_plan(int M, int K) {
    FewPlan p;
    p.k_steps = (K + 2 * kBK - 1) / (2 * kBK);
    p.tiles = (M + kBM - 1) / kBM;
    p.units = p.tiles * p.k_steps;
    const long long most = (p.units + 1) / 2, sms = sm_count();
    p.ctas = most < sms ? most : sms;
    // A tile's parts are read by one CTA in turn, each in about a third of the time of a step: more than
    // sqrt(3.5 k_steps) of them take longer than they save.  20 tokens, 12216 to 488 features 18.5 us
    // (22.6 without this limit, 17.1 with half of it), 16384 to 128 18.5 (30.8, 17.8), 1024 to 1024
    // 10.5 (11.3, 13.7); 4096 and 11008 to 1024 and more the same
    const long long cap = p.tiles * static_cast<long long>(sqrt(3.5 * p.k_steps));
    if (p.ctas > cap) p.ctas = cap;
    return p;
}
int few_bt(int T) { return T <= 16 ? 16 : 32; }
size_t few_counter_bytes(int M) { return up256(static_cast<size_t>((M + kBM - 1) / kBM) * 16); }
size_t few_scratch_bytes(int M, int K, int T) {
    return static_cast<size_t>(2 * few_plan(M, K).ctas) * few_bt(T) * kBM * 4;
}

// W: [M, K] (K-major) or, W_MN, [K, M]; X [T, K].
template <int BT, bool W_MN, class Out>
cudaError_t run_few_bt(const void* W, const void* X, int M, int K, int T, const Out& out,
                       uint8_t* counters, float* scratch, unsigned* status, cudaStream_t st) {
    using L = FewSmem<BT>;
    constexpr auto kern = few_tokens_kernel<BT, W_MN, Out>;
    const cudaError_t e = set_smem_limit<kern>(L::kBytes);
    if (e != cudaSuccess) return e;
    CUtensorMap wmap, xmap;
    const bool ok = W_MN ? map_weights(&wmap, W, K, M, kBK) : map_weights(&wmap, W, M, K, kBM);
    if (!ok || !map_kmajor(&xmap, X, T, K, BT)) return cudaErrorInvalidValue;
    const FewPlan p = few_plan(M, K);
    FewShape sh;
    sh.T = T;
    sh.k_steps = p.k_steps;
    sh.units = p.units;
    sh.scratch = scratch;
    sh.counters = reinterpret_cast<unsigned*>(counters);
    return launch_chained(kern, dim3(static_cast<unsigned>(p.ctas)), 192, L::kBytes, st, wmap, xmap,
                          out, sh, status, wait_limit_ns());
}
template <bool W_MN, class Out>
cudaError_t run_few(const void* W, const void* X, int M, int K, int T, const Out& out,
                    uint8_t* counters, float* scratch, unsigned* status, cudaStream_t st) {
    if (few_bt(T) == 16)
        return run_few_bt<16, W_MN>(W, X, M, K, T, out, counters, scratch, status, st);
    return run_few_bt<32, W_MN>(W, X, M, K, T, out, counters, scratch, status, st);
}

// ------------------------------------------------------------------ a few rows of X
// Y = act(X W^T + b) + R for T <= row_tokens(dtype): a warp per feature, whose row of the weights the
// lanes read 16 bytes each (fp32 rows that are no multiple of that: 4), some loads ahead; X comes from
// L1, and a butterfly adds the lanes' sums.  Nothing has to be set up or added across blocks: one
// launch, which also clears the status word (no kernel of the call waits for anything).
// Bound: the weights' bytes.  bf16, 4096 to 11008 features 17.8 us (5.1 TB/s; few_tokens_kernel 28),
// to 44032 56 (6.4 TB/s).  8 and 16 loads ahead 19.2 and 20.3; 8 warps a block the same, and with four
// tokens 26.2 instead of 23.9.  fp32 goes to 16 tokens, since the 64-row tiles of the products that take
// over there cost the same down to one: 3000 to 3000 features, weights in L2, 1 token 5.9 us, 4 8.3, 8
// 13, 16 25, 17 (on tiles) 46; 767 to 1537 5.2, 5.8, 7.9, 9.5, 16.6.
constexpr int kRowWarps = 4;
constexpr int row_tokens(int dtype) { return dtype == 1 ? 4 : 16; }

template <typename T>
struct RowOut {
    const T* bias;
    const T* residual;
    T* Y;
    T* Z;
    int act;
};

// A vector of kV values as it is loaded, and acc + w (.) x over it.
template <typename T, int kV>
struct RowVec {  // 16 bytes
    static constexpr int kAhead = 4;
    uint4 u;
    __device__ __forceinline__ void load(const T* p) { u = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void load_stream(const T* p) {
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w)
                     : "l"(p));
    }
    __device__ __forceinline__ void zero() { u = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ float2 dot(const RowVec& x, float2 acc) const {
        if constexpr (kV == 8) {
            acc = fma2(unpack2(u.x), unpack2(x.u.x), acc);
            acc = fma2(unpack2(u.y), unpack2(x.u.y), acc);
            acc = fma2(unpack2(u.z), unpack2(x.u.z), acc);
            return fma2(unpack2(u.w), unpack2(x.u.w), acc);
        } else {
            acc = fma2(pair(u.x, u.y), pair(x.u.x, x.u.y), acc);
            return fma2(pair(u.z, u.w), pair(x.u.z, x.u.w), acc);
        }
    }
    static __device__ __forceinline__ float2 pair(uint32_t a, uint32_t b) {
        return make_float2(__uint_as_float(a), __uint_as_float(b));
    }
};
template <>
struct RowVec<float, 1> {
    static constexpr int kAhead = 8;
    float f;
    __device__ __forceinline__ void load(const float* p) { f = *p; }
    __device__ __forceinline__ void load_stream(const float* p) { f = __ldcs(p); }
    __device__ __forceinline__ void zero() { f = 0.f; }
    __device__ __forceinline__ float2 dot(const RowVec& x, float2 acc) const {
        return make_float2(fmaf(f, x.f, acc.x), 0.f);
    }
};

__device__ __forceinline__ float row_value(const float* p) { return *p; }
__device__ __forceinline__ float row_value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void row_store(float* p, float x) { *p = x; }
__device__ __forceinline__ void row_store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// kT >= tokens: those behind the last are read as it, and not written.
template <typename T, int kV, int kT>
__global__ void __launch_bounds__(32 * kRowWarps)
    row_kernel(const T* __restrict__ X, const T* __restrict__ W, int tokens, int N, int K,
               const __grid_constant__ RowOut<T> out, unsigned* status) {
    using Vec = RowVec<T, kV>;
    if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0u;
    const int lane = threadIdx.x % 32, feature = blockIdx.x * kRowWarps + threadIdx.x / 32;
    if (feature >= N) return;
    const int vecs = K / kV;
    const T* w = W + static_cast<long long>(feature) * K;
    float2 acc[kT];
#pragma unroll
    for (int t = 0; t < kT; ++t) acc[t] = make_float2(0.f, 0.f);
    for (int v0 = lane; v0 < vecs; v0 += 32 * Vec::kAhead) {
        Vec u[Vec::kAhead];
#pragma unroll
        for (int i = 0; i < Vec::kAhead; ++i) {
            u[i].zero();
            if (v0 + 32 * i < vecs) u[i].load_stream(w + static_cast<long long>(v0 + 32 * i) * kV);
        }
#pragma unroll
        for (int i = 0; i < Vec::kAhead; ++i) {
            if (v0 + 32 * i >= vecs) break;
#pragma unroll
            for (int t = 0; t < kT; ++t) {
                Vec x;
                x.load(X + static_cast<long long>(min(t, tokens - 1)) * K +
                       static_cast<long long>(v0 + 32 * i) * kV);
                acc[t] = u[i].dot(x, acc[t]);
            }
        }
    }
    float s = 0.f;  // lane t has token t's
#pragma unroll
    for (int t = 0; t < kT; ++t) {
        const float r = warp_sum_f32(acc[t].x + acc[t].y);
        if (lane == t) s = r;
    }
    if (lane >= tokens) return;
    const long long o = static_cast<long long>(lane) * N + feature;
    if (out.bias) s += row_value(out.bias + feature);
    if (out.Z) row_store(out.Z + o, s);
    with_act(out.act, [&](auto act) {
        if constexpr (std::is_same_v<T, float>)
            s = act_value<act.value>(s);
        else
            s = act_value2<act.value>(make_float2(s, 0.f)).x;
    });
    if (out.residual) s += row_value(out.residual + o);
    row_store(out.Y + o, s);
}

template <typename T, int kV, int kT>
cudaError_t run_rows_t(const LinearFwd& p, unsigned* status, cudaStream_t st) {
    const RowOut<T> out{static_cast<const T*>(p.bias), static_cast<const T*>(p.residual),
                        static_cast<T*>(p.Y), static_cast<T*>(p.Z), p.act};
    return launch_plain(row_kernel<T, kV, kT>, static_cast<unsigned>((p.N + kRowWarps - 1) / kRowWarps),
                        32 * kRowWarps, st, static_cast<const T*>(p.X), static_cast<const T*>(p.W), p.T, p.N,
                        p.K, out, status);
}
template <typename T, int kV>
cudaError_t run_rows_v(const LinearFwd& p, unsigned* status, cudaStream_t st) {
    if (p.T == 1) return run_rows_t<T, kV, 1>(p, status, st);
    if (p.T == 2) return run_rows_t<T, kV, 2>(p, status, st);
    if constexpr (std::is_same_v<T, float>) {
        if (p.T > 8) return run_rows_t<T, kV, 16>(p, status, st);
        if (p.T > 4) return run_rows_t<T, kV, 8>(p, status, st);
    } else {
        if (p.T == 3) return run_rows_t<T, kV, 3>(p, status, st);
    }
    return run_rows_t<T, kV, 4>(p, status, st);
}
cudaError_t run_rows(int dtype, const LinearFwd& p, unsigned* status, cudaStream_t st) {
    if (dtype == 1) return run_rows_v<__nv_bfloat16, 8>(p, status, st);
    return p.K % 4 == 0 ? run_rows_v<float, 4>(p, status, st) : run_rows_v<float, 1>(p, status, st);
}

// ------------------------------------------------------------------ pair tiles
// Clusters of the pair kernels at once (76 without a device: two SMs of 152 each).
int linear_clusters() {
    using L = GemmPairSmem<256, kPairStages, pair_ksub<256, false, false>()>;
    constexpr auto kern = tc_gemm_pair_kernel<256, false, false, kPairStages, 1, EpiLinear<256, kActNone>>;
    DevInfo di;
    if (current_device_info(&di)) {
        if (set_smem_limit<kern>(L::kBytes) == cudaSuccess)
            return resident_clusters<kern>(gemm_threads<EpiLinear<256, kActNone>>(), L::kBytes, di.sm_count, 2);
        cudaGetLastError();  // its own (one that the caller left pending stays)
    }
    return 76;
}

// How a product runs: on one CTA's tiles of 128 rows by `single` columns, on pair tiles of 128
// columns (half) or on those of 256, with k ranges of every tile (split), or of those of the last
// partial wave (tail), and the units of scratch.
struct PairPlan {
    int single = 0;
    bool half = false;
    int split = 0;
    SkPlan tail;
    long long units = 0;
};

// The cheapest by what was measured, in ns.  A 64-deep k-block of a 256 x 256 pair tile takes 325,
// where one wave has all tiles: pair tiles of 128 columns 300, one CTA's of 128 columns 355 and of 64
// columns 290, and a launch and its epilogue 9000 on pairs and 6000 on single CTAs, which have no
// partner to wait for.  (From L2 a single CTA's pace is its own, and not that of something the CTAs
// share: with 2, 8, 18, 38 and 76 CTAs a k-block of 64 columns took 291, 299, 288, 288 and 280 ns, one
// of 128 columns 256 to 258 with each; all 152 took 261 and, their operands beyond L2, 305.)  Split tiles
// add the store of the parts of a wave of units (2500), the fixup's launch (5000) and its read of a
// unit (100).
//   T x K x N, us: 200 x 256 x 384 12.3 on pairs, 8.3 on 64-column CTAs; 128 x 1024 x 1024 16.4,
//   12.3; 200 x 4096 x 4096 28.7, 26.7; 64 x 4096 x 11008 38.8, 28.9 on 128-column ones.  4096 x
//   11008 x 4096 (256 tiles on 76 clusters): the last 28 tiles whole 56, in 2 ranges 41, in the 5 that
//   fill the waves best 48 (the product 239).
PairPlan pair_plan(int M, int N, int K) {
    PairPlan p;
    const long long tiles = static_cast<long long>((M + 255) / 256) * ((N + 255) / 256);
    const int kb = (K + kBK - 1) / kBK;
    const long long clusters = linear_clusters(), sms = sm_count();
    const long long left = tiles < clusters ? tiles : tiles % clusters;
    if (left == 0) return p;
    double best = 9000.0 + kb * 325.0;
    if (2 * tiles <= clusters) {
        p.half = true;
        best = 9000.0 + kb * 300.0;
    }
    for (int S = 2; S <= 32 && kb / S >= 8 && left * S <= kTailWaves * clusters; ++S) {
        const double waves = static_cast<double>((left * S + clusters - 1) / clusters);
        const double cost =
            9000.0 + waves * (((kb + S - 1) / S) * 325.0 + 2500.0) + 5000.0 + left * S * 100.0;
        if (cost >= best) continue;
        best = cost;
        p.half = false;
        p.units = left * S;
        p.split = S;
    }
    if (tiles >= clusters) {
        if (p.units > 0) {
            p.tail.tail_tiles = left;
            p.tail.tail_split = p.split;
            p.split = 0;
        }
        return p;
    }
    for (int width : {128, 64}) {
        const long long n = static_cast<long long>((M + 127) / 128) * ((N + width - 1) / width);
        const double cost = 6000.0 + kb * (width == 128 ? 355.0 : 290.0);
        if (n > sms || cost >= best) continue;
        best = cost;
        p = PairPlan{};
        p.single = width;
    }
    return p;
}

size_t pair_scratch_bytes(int M, int N, int K) {
    return static_cast<size_t>(pair_plan(M, N, K).units) * kPairBM * 256 * sizeof(float);
}

template <class Out>
__global__ void __launch_bounds__(kFixupThreads)
    linear_fixup_kernel(const GemmShape sh, const float* scratch, const __grid_constant__ Out out) {
    grid_dependency_trigger();
    grid_dependency_wait();
    int row, n;
    float s4[4];
    if (!sk_tail_sum<256>(sh, scratch, row, n, s4)) return;
    out_row4(out, row * out.ld + n, n, s4);
}

bool out_maps(EpiLinear<256, kActAny>::Params* p) {
    return map_out_bf16(&p->ymap, p->o.Y, p->o.M, p->o.N) &&
           map_out_bf16(&p->zmap, p->o.Z ? p->o.Z : p->o.Y, p->o.M, p->o.N);
}
bool out_maps(EpiSlope<256, kActAny>::Params* p) {
    return map_out_bf16(&p->xmap, p->o.X, p->o.M, p->o.N);
}

// Parameters for another width or activation of an epilogue: the fields are the same.
template <class To, class From>
To params_as(const From& from) {
    static_assert(sizeof(To) == sizeof(From), "the same fields");
    To to;
    memcpy(&to, &from, sizeof(to));
    return to;
}

// C[M, N] = A B^T through Epi.  A_MN: A is [K, M], else [M, K]; B_MN: B is [K, N], else [N, K].
// kPlain: there is no activation (fewer kernels to compile).
template <bool A_MN, bool B_MN, bool kPlain, template <int, int> class Epi, class Out>
cudaError_t run_pair(const void* A, const void* B, int M, int N, int K, const Out& out, int act,
                     float* scratch, unsigned* status, cudaStream_t st) {
    constexpr int kAny = kPlain ? kActNone : kActAny;
    const PairPlan pp = pair_plan(M, N, K);
    GemmMaps<1> maps;
    bool ok = A_MN ? map_mnmajor(&maps.a[0], A, K, M) : map_kmajor(&maps.a[0], A, M, K, kBM);
    const int b_rows = pp.single ? pp.single : pp.half ? kHalfBN / 2 : 128;
    ok = ok && (B_MN ? map_mnmajor(&maps.b[0], B, K, N) : map_kmajor(&maps.b[0], B, N, K, b_rows));
    typename Epi<256, kActAny>::Params ep;
    ep.o = out;
    if (!ok || !out_maps(&ep)) return cudaErrorInvalidValue;
    if (pp.single == 64) {
        using E = Epi<64, kAny>;
        return run_gemm<64, A_MN, B_MN, 8, 1, E>(maps, params_as<typename E::Params>(ep),
                                                 make_shape(M, N, K, 64, 1, band_for(false)), status, st);
    }
    if (pp.single == 128) {
        using E = Epi<128, kAny>;
        return run_gemm<128, A_MN, B_MN, 6, 1, E>(maps, params_as<typename E::Params>(ep),
                                                  make_shape(M, N, K, 128, 1, band_for(false)), status, st);
    }
    if (pp.half) {
        using E = Epi<kHalfBN, kAny>;
        return run_gemm_pair<kHalfBN, A_MN, B_MN, kHalfStages, 1, E>(
            maps, params_as<typename E::Params>(ep),
            make_shape(M, N, K, kHalfBN, 1, band_for(true), kPairBM), status, st);
    }
    const GemmShape sh = make_shape(M, N, K, 256, 1, band_for(true), kPairBM);
    SkPlan plan;
    auto run = [&](auto a) {
        using E = Epi<256, decltype(a)::value>;
        return run_gemm_pair<256, A_MN, B_MN, kPairStages, 1, E>(
            maps, params_as<typename E::Params>(ep), sh, status, st, pp.units > 0 ? scratch : nullptr,
            &plan, pp.split, &pp.tail);
    };
    cudaError_t e;
    if constexpr (kPlain) {
        e = run(std::integral_constant<int, kActNone>{});
    } else {
        switch (act) {
            case kActRelu: e = run(std::integral_constant<int, kActRelu>{}); break;
            case kActGelu: e = run(std::integral_constant<int, kActGelu>{}); break;
            case kActGeluTanh: e = run(std::integral_constant<int, kActGeluTanh>{}); break;
            case kActSilu: e = run(std::integral_constant<int, kActSilu>{}); break;
            default: e = run(std::integral_constant<int, kActNone>{}); break;
        }
    }
    if (e != cudaSuccess || plan.tail_tiles <= 0) return e;
    return launch_chained(linear_fixup_kernel<Out>, sk_fixup_grid<256>(plan), kFixupThreads, 0, st,
                          sk_fixup_shape(plan, sh), static_cast<const float*>(scratch), out);
}

// ------------------------------------------------------------------ the signal at the layer's own output
// dZ = dY (.) act'(Z) (dZ and Z null: dY as it is) and the sums of its columns, before rounding,
// over a range of rows: part[range][N].  16 lanes to kV columns each and 16 rows at a time;
// a thread adds its rows in order, the block's 16 in order.
// Bound: HBM, one pass over dY and Z.
constexpr int kSigThreads = 256, kSigLanes = 16, kSigRows = kSigThreads / kSigLanes;

template <typename T, int kV>
__device__ __forceinline__ void sig_load(const T* p, float (&x)[kV]) {
    if constexpr (kV == 8) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        const float2 a = unpack2(u.x), b = unpack2(u.y), c = unpack2(u.z), d = unpack2(u.w);
        x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
        x[4] = c.x; x[5] = c.y; x[6] = d.x; x[7] = d.y;
    } else if constexpr (kV == 4) {
        const float4 u = *reinterpret_cast<const float4*>(p);
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
    } else {
        x[0] = p[0];
    }
}
template <typename T, int kV>
__device__ __forceinline__ void sig_store(T* p, const float (&x)[kV]) {
    if constexpr (kV == 8) {
        *reinterpret_cast<uint4*>(p) =
            make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                       pack_bf16x2(x[6], x[7]));
    } else if constexpr (kV == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
        p[0] = x[0];
    }
}

// status (or null): this kernel is the call's first and clears it and `clear_words` words behind it.
// With more ranges than one their sums are added in their order: without counters the ranges are the
// blocks of one cluster, whose first reads the others' shared memory; with them (zero at the start)
// by the last block of a column group to finish.
template <typename T, int kV>
__global__ void __launch_bounds__(kSigThreads)
    signal_kernel(const T* dY, const T* Z, int act, int rows, int N, int rows_per, T* dZ, float* part,
                  float* dbias, unsigned* counters, unsigned* status, int clear_words) {
    __shared__ float sums[kSigRows][kSigLanes * kV + 1];
    __shared__ bool last;
    grid_dependency_trigger();
    grid_dependency_wait();
    if (status && blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = threadIdx.x; i < clear_words; i += kSigThreads) status[i] = 0u;
    const int lane = threadIdx.x % kSigLanes, row_lane = threadIdx.x / kSigLanes;
    const int col = (blockIdx.x * kSigLanes + lane) * kV;
    const int r0 = blockIdx.y * rows_per, r1 = min(rows, r0 + rows_per);
    float s[kV];
#pragma unroll
    for (int k = 0; k < kV; ++k) s[k] = 0.f;
    if (col < N) {
        with_act(Z ? act : kActNone, [&](auto a) {
#pragma unroll 8
            for (int r = r0 + row_lane; r < r1; r += kSigRows) {
                const long long o = static_cast<long long>(r) * N + col;
                float x[kV];
                sig_load<T, kV>(dY + o, x);
                if constexpr (a.value != kActNone) {
                    float z[kV];
                    sig_load<T, kV>(Z + o, z);
                    if constexpr (kV == 8) {  // bf16
#pragma unroll
                        for (int k = 0; k < kV; k += 2) {
                            const float2 s2 = act_slope2<a.value>(make_float2(z[k], z[k + 1]));
                            x[k] *= s2.x;
                            x[k + 1] *= s2.y;
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < kV; ++k) x[k] *= act_slope<a.value>(z[k]);
                    }
                    sig_store<T, kV>(dZ + o, x);
                }
#pragma unroll
                for (int k = 0; k < kV; ++k) s[k] += x[k];
            }
        });
    }
    if (!dbias) return;
#pragma unroll
    for (int k = 0; k < kV; ++k) sums[row_lane][lane * kV + k] = s[k];
    __syncthreads();
    const int c = threadIdx.x, n = blockIdx.x * kSigLanes * kV + c;
    const bool mine = c < kSigLanes * kV && n < N;
    float t = 0.f;
    if (mine) {
#pragma unroll
        for (int r = 0; r < kSigRows; ++r) t += sums[r][c];
    }
    if (gridDim.y == 1) {
        if (mine) dbias[n] = t;
        return;
    }
    if (!counters) {
        __shared__ float total[kSigLanes * kV];
        if (mine) total[c] = t;
        __syncwarp();
        cluster_sync();
        if (mine && blockIdx.y == 0) {
            const uint32_t at = smem_u32(total + c);
            t = 0.f;
#pragma unroll 8
            for (unsigned r = 0; r < gridDim.y; ++r)
                t += __uint_as_float(ld_shared_cluster_u32(mapa_shared(at, r)));
            dbias[n] = t;
        }
        __syncwarp();
        cluster_sync();  // until the first has read this one's
        return;
    }
    if (mine) part[static_cast<long long>(blockIdx.y) * N + n] = t;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(counters + blockIdx.x, 1u) == gridDim.y - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (!mine) return;
    t = 0.f;
#pragma unroll 16
    for (int r = 0; r < static_cast<int>(gridDim.y); ++r)
        t += __ldcg(part + static_cast<long long>(r) * N + n);
    dbias[n] = t;
}

struct SignalPlan {
    int cols;      // column blocks
    int rows_per;  // rows of a range, a multiple of kSigRows
    int ranges;
    bool cluster;  // the ranges are a cluster's blocks (or one)
};
int sig_v(int dtype, int N) { return dtype == 1 ? 8 : N % 4 == 0 ? 4 : 1; }
// Up to 2048 rows, or 8192 without an activation to compute, the ranges are a cluster's blocks, one for
// every 64 or 256 rows begun and at most eight: no counters to clear and wait for.  us with 256 rows
// and counters, and so (fp32 with a slower gelu than now's, 4.5): 512 x 1024 fp32 gelu 18.5 and 5.9,
// bias sums alone 8.3 and 3.1; 2048 x 256 bf16 gelu 14.5 and 8.9, alone 8.6 and 3.2; 200 x 256 bf16 gelu (one range) 6.6 and 4.1.
// Above that eight blocks of a column group are too few: 4096 x 128 fp32 gelu 18.6 and 24.9, 8192 x 256
// bf16 14.4 and 27.8, alone 8.3 and 6.0; 16384 x 128 alone 8.5 and 9.7.
SignalPlan signal_plan(int dtype, int T, int N, int act) {
    const int per = kSigLanes * sig_v(dtype, N), least = act == kActNone ? 256 : 64;
    SignalPlan p;
    p.cols = (N + per - 1) / per;
    p.cluster = T <= (act == kActNone ? 8192 : 2048);
    const long long most = 4LL * sm_count() / p.cols;  // ranges
    long long ranges = p.cluster ? (T + least - 1) / least : (T + 255) / 256;
    if (p.cluster && ranges > 8) ranges = 8;
    if (ranges > most) ranges = most;
    if (ranges < 1) ranges = 1;
    p.rows_per = static_cast<int>((((T + ranges - 1) / ranges) + kSigRows - 1) / kSigRows * kSigRows);
    p.ranges = (T + p.rows_per - 1) / p.rows_per;
    if (p.ranges == 1) p.cluster = true;
    return p;
}

size_t signal_counter_bytes(const SignalPlan& p) {
    return p.cluster ? 0 : up256(static_cast<size_t>(p.cols) * sizeof(unsigned));
}

template <typename T, int kV>
cudaError_t run_signal_v(const LinearVjp& p, T* dZ, float* part, unsigned* counters, unsigned* status,
                         size_t clear_bytes, const SignalPlan& sp, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(sp.cols, sp.ranges, 1);
    cfg.blockDim = dim3(kSigThreads, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // as launch_chained
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 1;
    at[1].val.clusterDim.y = static_cast<unsigned>(sp.ranges);
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = sp.cluster && sp.ranges > 1 ? 2 : 1;
    note_launch();
    const cudaError_t e = cudaLaunchKernelEx(
        &cfg, signal_kernel<T, kV>, static_cast<const T*>(p.dY),
        static_cast<const T*>(p.act != kActNone ? p.Z : nullptr), p.act, p.T, p.N, sp.rows_per, dZ, part,
        p.dbias, sp.cluster ? nullptr : counters, status,
        static_cast<int>(clear_bytes / sizeof(unsigned)));
    if (e != cudaSuccess) cudaGetLastError();
    return e;
}

}  // namespace

size_t linear_clear_bytes(int dtype, int T, int N, int K) {
    if (T <= row_tokens(dtype)) return 0;  // the kernel does it
    return dtype == 1 && T <= kFewT ? kHead + few_counter_bytes(N) : sizeof(unsigned);
}
size_t linear_workspace_bytes(int dtype, int T, int N, int K) {
    if (dtype != 1 || T <= row_tokens(dtype)) return kHead;
    if (T <= kFewT) return kHead + few_counter_bytes(N) + few_scratch_bytes(N, K, T);
    return kHead + pair_scratch_bytes(T, N, K);
}

cudaError_t launch_linear(int dtype, const LinearFwd& p, void* workspace, cudaStream_t st) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    unsigned* status = reinterpret_cast<unsigned*>(ws);
    if (p.T <= row_tokens(dtype)) return run_rows(dtype, p, status, st);
    if (dtype == 0) return launch_linear_f32(p, st);
    LinearOut out;
    out.bias = static_cast<const __nv_bfloat16*>(p.bias);
    out.residual = static_cast<const __nv_bfloat16*>(p.residual);
    out.Y = static_cast<__nv_bfloat16*>(p.Y);
    out.Z = static_cast<__nv_bfloat16*>(p.Z);
    out.ld = p.N;
    out.M = p.T;
    out.N = p.N;
    out.act = p.act;
    if (p.T <= kFewT)
        return run_few<false>(p.W, p.X, p.N, p.K, p.T, out, ws + kHead,
                              reinterpret_cast<float*>(ws + kHead + few_counter_bytes(p.N)),
                              status, st);
    return run_pair<false, false, false, EpiLinear>(p.X, p.W, p.T, p.N, p.K, out, p.act,
                                                    reinterpret_cast<float*>(ws + kHead), status, st);
}

namespace {

// The backward pass's workspace: status word, counters of few_tokens_kernel and of signal_kernel,
// dZ (with an activation), the bias ranges' sums, scratch of the products' parts; dx, dw: whether those
// products run (the bias gradient's share does not depend on K).
struct VjpLayout {
    size_t few, sig, clear, dz, part, scratch, total;
};
VjpLayout vjp_layout(int dtype, int T, int N, int K, int act, bool dx, bool dw) {
    VjpLayout l;
    const SignalPlan sp = signal_plan(dtype, T, N, act);
    l.few = kHead;
    const bool few = dtype == 1 && T <= kFewT;
    l.sig = l.few + (few && dx ? few_counter_bytes(K) : 0);
    l.clear = l.dz = l.sig + signal_counter_bytes(sp);
    size_t off = l.dz;
    if (act != kActNone) off = up256(off + static_cast<size_t>(T) * N * (dtype == 1 ? 2 : 4));
    l.part = off;
    if (!sp.cluster) off = up256(off + static_cast<size_t>(sp.ranges) * N * sizeof(float));
    l.scratch = off;
    size_t scratch = 0;
    if (dtype == 1 && dw) scratch = pair_scratch_bytes(N, K, T);
    if (dtype == 1 && dx) {
        const size_t parts = few ? few_scratch_bytes(K, N, T) : pair_scratch_bytes(T, K, N);
        scratch = parts > scratch ? parts : scratch;
    }
    l.total = off + scratch;
    return l;
}

}  // namespace

size_t linear_vjp_workspace_bytes(int dtype, int T, int N, int K, int act, bool dx, bool dw) {
    return T == 0 ? kHead : vjp_layout(dtype, T, N, K, act, dx, dw).total;
}

cudaError_t launch_linear_vjp(int dtype, const LinearVjp& p, void* workspace, cudaStream_t st) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    unsigned* status = reinterpret_cast<unsigned*>(ws);
    const VjpLayout l = vjp_layout(dtype, p.T, p.N, p.K, p.act, p.dX != nullptr, p.dW != nullptr);
    const SignalPlan sp = signal_plan(dtype, p.T, p.N, p.act);
    float* part = reinterpret_cast<float*>(ws + l.part);
    float* scratch = reinterpret_cast<float*>(ws + l.scratch);
    const bool signal = p.act != kActNone || p.dbias;
    // no counters: signal_kernel clears what the products need.  That it may start before the kernel
    // in front of the call has ended is in its own wait's hands
    const bool clears = signal && sp.cluster;
    cudaError_t e = cudaSuccess;
    if (!clears) e = cudaMemsetAsync(ws, 0, l.clear, st);
    if (e != cudaSuccess) return e;
    const void* dZ = p.act != kActNone ? ws + l.dz : p.dY;
    if (signal) {
        void* to = p.act != kActNone ? ws + l.dz : nullptr;
        unsigned* counters = reinterpret_cast<unsigned*>(ws + l.sig);
        unsigned* first = clears ? status : nullptr;
        if (dtype == 1)
            e = run_signal_v<__nv_bfloat16, 8>(p, static_cast<__nv_bfloat16*>(to), part, counters,
                                               first, l.clear, sp, st);
        else if (sig_v(dtype, p.N) == 4)
            e = run_signal_v<float, 4>(p, static_cast<float*>(to), part, counters, first, l.clear, sp,
                                       st);
        else
            e = run_signal_v<float, 1>(p, static_cast<float*>(to), part, counters, first, l.clear, sp,
                                       st);
        if (e != cudaSuccess) return e;
    }
    if (dtype == 0) {
        const float* dzf = static_cast<const float*>(dZ);
        if (p.dX)
            e = launch_linear_dx_f32(p.T, p.N, p.K, dzf, static_cast<const float*>(p.W),
                                     static_cast<const float*>(p.act_in != kActNone ? p.Z_in : nullptr),
                                     p.act_in, static_cast<float*>(p.dX), st);
        if (e != cudaSuccess || !p.dW) return e;
        return launch_linear_dw_f32(p.T, p.N, p.K, dzf, static_cast<const float*>(p.X),
                                    static_cast<float*>(p.dW), st);
    }
    if (p.dX) {
        SlopeOut out;
        out.z = static_cast<const __nv_bfloat16*>(p.act_in != kActNone ? p.Z_in : nullptr);
        out.X = static_cast<__nv_bfloat16*>(p.dX);
        out.ld = p.K;
        out.M = p.T;
        out.N = p.K;
        out.act = p.act_in;
        e = p.T <= kFewT
                ? run_few<true>(p.W, dZ, p.K, p.N, p.T, out, ws + l.few, scratch, status, st)
                : run_pair<false, true, false, EpiSlope>(dZ, p.W, p.T, p.K, p.N, out, p.act_in, scratch,
                                                           status, st);
        if (e != cudaSuccess) return e;
    }
    if (!p.dW) return cudaSuccess;
    SlopeOut out;
    out.z = nullptr;
    out.X = static_cast<__nv_bfloat16*>(p.dW);
    out.ld = p.K;
    out.M = p.N;
    out.N = p.K;
    out.act = kActNone;
    return run_pair<true, true, true, EpiSlope>(dZ, p.X, p.N, p.K, p.T, out, kActNone, scratch, status, st);
}

}  // namespace fpo
