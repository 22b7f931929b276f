// linear_epilogues.cuh -- 8-warp epilogues (tc_gemm.cuh, RowChunk) of the linear layer's
// products: bias, activation and residual of the forward pass, the slope of the activation
// below in the backward pass.  What a chunk reads is loaded as one batch when the chunk before
// is done (epilogues.cuh says why).
#pragma once

#include "act_math.cuh"
#include "epilogues.cuh"

namespace fpo {

__device__ __forceinline__ void unpack4(uint2 u, float (&x)[4]) {
    x[0] = __uint_as_float(u.x << 16);
    x[1] = __uint_as_float(u.x & 0xffff0000u);
    x[2] = __uint_as_float(u.y << 16);
    x[3] = __uint_as_float(u.y & 0xffff0000u);
}
__device__ __forceinline__ uint2 pack4(const float (&x)[4]) {
    return make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
}

// z = v + bias; Z = z; Y = act(z) + residual.  Any of bias, residual and Z may be null; with
// none of them and no activation the plain product, rounded (the weight gradient).
struct LinearOut {
    const __nv_bfloat16* bias;      // [N]
    const __nv_bfloat16* residual;  // [M, N]
    __nv_bfloat16* Y;               // [M, N]
    __nv_bfloat16* Z;
    long long ld;
    int M, N, act;
};
// X = v act'(z), z null: v.
struct SlopeOut {
    const __nv_bfloat16* z;  // [M, N]
    __nv_bfloat16* X;        // [M, N]
    long long ld;
    int M, N, act;
};

// N summed values of a row at element offset o (columns from c) through the epilogue, for the
// kernels that sum the parts of split tiles.
template <int kN>
__device__ __forceinline__ void out_row(const LinearOut& p, long long o, int c, float (&v)[kN]) {
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        if (p.bias) v[k] += __bfloat162float(p.bias[c + k]);
        if (p.Z) p.Z[o + k] = __float2bfloat16_rn(v[k]);
    }
    with_act(p.act, [&](auto act) {
#pragma unroll
        for (int k = 0; k < kN; ++k) v[k] = act_value<act.value, true>(v[k]);
    });
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        if (p.residual) v[k] += __bfloat162float(p.residual[o + k]);
        p.Y[o + k] = __float2bfloat16_rn(v[k]);
    }
}
template <int kN>
__device__ __forceinline__ void out_row(const SlopeOut& p, long long o, int, float (&v)[kN]) {
    if (p.z) {
        float z[kN];
#pragma unroll
        for (int k = 0; k < kN; ++k) z[k] = __bfloat162float(p.z[o + k]);
        with_act(p.act, [&](auto act) {
#pragma unroll
            for (int k = 0; k < kN; ++k) v[k] *= act_slope<act.value, true>(z[k]);
        });
    }
#pragma unroll
    for (int k = 0; k < kN; ++k) p.X[o + k] = __float2bfloat16_rn(v[k]);
}
// 4 of them, 8-byte aligned.
__device__ __forceinline__ void out_row4(const LinearOut& p, long long o, int c, float (&v)[4]) {
    if (p.bias) {
        float b[4];
        unpack4(*reinterpret_cast<const uint2*>(p.bias + c), b);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += b[k];
    }
    if (p.Z) *reinterpret_cast<uint2*>(p.Z + o) = pack4(v);
    with_act(p.act, [&](auto act) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = act_value<act.value, true>(v[k]);
    });
    if (p.residual) {
        float r[4];
        unpack4(*reinterpret_cast<const uint2*>(p.residual + o), r);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += r[k];
    }
    *reinterpret_cast<uint2*>(p.Y + o) = pack4(v);
}
__device__ __forceinline__ void out_row4(const SlopeOut& p, long long o, int, float (&v)[4]) {
    if (p.z) {
        float z[4];
        unpack4(*reinterpret_cast<const uint2*>(p.z + o), z);
        with_act(p.act, [&](auto act) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] *= act_slope<act.value, true>(z[k]);
        });
    }
    *reinterpret_cast<uint2*>(p.X + o) = pack4(v);
}

template <int kCG>
struct EpiLinear {
    using Params = LinearOut;
    static constexpr int kWarps = 8, kColGroups = kCG;
    using R = RowChunk;
    RowPos<kCG> pos;
    uint2 b[kCG];      // bias of the lane's columns of each column group
    uint2 r[R::kAcc];  // residual of the next chunk

    __device__ __forceinline__ void load(const Params& p, int c) {
        if (!p.residual) return;
#pragma unroll
        for (int i = 0; i < R::kAcc; ++i)
            r[i] = *reinterpret_cast<const uint2*>(pos.src(p.residual, p.ld, R::kAcc * c + i));
    }

    __device__ __forceinline__ EpiLinear(const Params& p, int, int row0, int n0, int lane)
        : pos(p.M, p.N, p.ld, row0, n0, lane) {
#pragma unroll
        for (int k = 0; k < kCG; ++k) {
            const int c = n0 + k * R::kCols + 4 * (lane % R::kLanes);
            b[k] = p.bias && c < p.N ? *reinterpret_cast<const uint2*>(p.bias + c)
                                     : make_uint2(0u, 0u);
        }
        load(p, 0);
    }

    __device__ __forceinline__ void chunk(const Params& p, uint32_t buf, int lane, int c) {
        float bias[4];
        unpack4(c % kCG == 0 ? b[0] : b[kCG - 1], bias);
        with_act(p.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < R::kAcc; ++i) {
                const float4 v4 = R::read(buf, lane, i);
                float v[4] = {v4.x + bias[0], v4.y + bias[1], v4.z + bias[2], v4.w + bias[3]};
                const bool in = pos.in(R::kAcc * c + i);
                const long long o = pos.at(p.ld, R::kAcc * c + i);
                if (p.Z && in) *reinterpret_cast<uint2*>(p.Z + o) = pack4(v);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = act_value<act.value, true>(v[k]);
                if (p.residual) {
                    float q[4];
                    unpack4(r[i], q);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] += q[k];
                }
                if (in) *reinterpret_cast<uint2*>(p.Y + o) = pack4(v);
            }
        });
        if (c + 1 < pos.kChunks) load(p, c + 1);
    }

    __device__ __forceinline__ void finish(const Params&, int) {}
};

template <int kCG>
struct EpiSlope {
    using Params = SlopeOut;
    static constexpr int kWarps = 8, kColGroups = kCG;
    using R = RowChunk;
    RowPos<kCG> pos;
    uint2 zr[R::kAcc];  // pre-activations of the next chunk

    __device__ __forceinline__ void load(const Params& p, int c) {
        if (!p.z) return;
#pragma unroll
        for (int i = 0; i < R::kAcc; ++i)
            zr[i] = *reinterpret_cast<const uint2*>(pos.src(p.z, p.ld, R::kAcc * c + i));
    }

    __device__ __forceinline__ EpiSlope(const Params& p, int, int row0, int n0, int lane)
        : pos(p.M, p.N, p.ld, row0, n0, lane) {
        load(p, 0);
    }

    __device__ __forceinline__ void chunk(const Params& p, uint32_t buf, int lane, int c) {
        with_act(p.z ? p.act : kActNone, [&](auto act) {
#pragma unroll
            for (int i = 0; i < R::kAcc; ++i) {
                const float4 v4 = R::read(buf, lane, i);
                float v[4] = {v4.x, v4.y, v4.z, v4.w};
                if constexpr (act.value != kActNone) {
                    float z[4];
                    unpack4(zr[i], z);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] *= act_slope<act.value, true>(z[k]);
                }
                if (pos.in(R::kAcc * c + i))
                    *reinterpret_cast<uint2*>(p.X + pos.at(p.ld, R::kAcc * c + i)) = pack4(v);
            }
        });
        if (c + 1 < pos.kChunks) load(p, c + 1);
    }

    __device__ __forceinline__ void finish(const Params&, int) {}
};

}  // namespace fpo
