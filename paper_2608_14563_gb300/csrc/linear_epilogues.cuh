// linear_epilogues.cuh -- epilogues (tc_gemm.cuh) of the linear layer's products: bias, activation
// and residual of the forward pass, the slope of the activation below in the backward pass.
//
// One row per thread, 32 columns at a time, written through the warp's staging buffers by TMA.  What
// a row reads beside the accumulator (residual, pre-activation) is loaded one chunk ahead, 64 bytes
// of 32 rows, and its other half line is in L1 by then.  The 8-warp form of the other epilogues that
// read matrices (RowChunk: every global access 256 bytes of two rows, through shared memory twice)
// takes 2 to 3 times the instructions; these run beside the MMAs of a GPU at its power cap.
#pragma once

#include "act_math.cuh"
#include "epilogues.cuh"

namespace fpo {

__device__ __forceinline__ float2 unpack2(uint32_t u) {
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pack2(float2 x) { return pack_bf16x2(x.x, x.y); }

// z = v + bias; Z = z; Y = act(z) + residual.  Any of bias, residual and Z may be null.
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

// 4 summed values at element offset o (a multiple of 4; columns from c) through the epilogue, for
// the kernel that adds the parts of split tiles.
__device__ __forceinline__ void out_row4(const LinearOut& p, long long o, int c, const float (&v)[4]) {
    float2 a = make_float2(v[0], v[1]), b = make_float2(v[2], v[3]);
    if (p.bias) {
        const uint2 u = *reinterpret_cast<const uint2*>(p.bias + c);
        a = add2(a, unpack2(u.x));
        b = add2(b, unpack2(u.y));
    }
    if (p.Z) *reinterpret_cast<uint2*>(p.Z + o) = make_uint2(pack2(a), pack2(b));
    with_act(p.act, [&](auto act) {
        a = act_value2<act.value>(a);
        b = act_value2<act.value>(b);
    });
    if (p.residual) {
        const uint2 u = *reinterpret_cast<const uint2*>(p.residual + o);
        a = add2(a, unpack2(u.x));
        b = add2(b, unpack2(u.y));
    }
    *reinterpret_cast<uint2*>(p.Y + o) = make_uint2(pack2(a), pack2(b));
}
__device__ __forceinline__ void out_row4(const SlopeOut& p, long long o, int, const float (&v)[4]) {
    float2 a = make_float2(v[0], v[1]), b = make_float2(v[2], v[3]);
    if (p.z) {
        const uint2 u = *reinterpret_cast<const uint2*>(p.z + o);
        with_act(p.act, [&](auto act) {
            a = mul2(a, act_slope2<act.value>(unpack2(u.x)));
            b = mul2(b, act_slope2<act.value>(unpack2(u.y)));
        });
    }
    *reinterpret_cast<uint2*>(p.X + o) = make_uint2(pack2(a), pack2(b));
}

// 32 columns of a row, one chunk ahead.
struct RowAhead {
    uint4 u[4];
    // p: the row's first element, null for none; columns outside the matrix (N: a multiple of 8) are
    // zeros.
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int col, int N) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            u[q] = p && col + 8 * q < N ? *reinterpret_cast<const uint4*>(p + col + 8 * q)
                                        : make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ float2 at(int j) const {  // columns 2 j and 2 j + 1
        const uint4& q = u[j / 4];
        return unpack2(j % 4 == 0 ? q.x : j % 4 == 1 ? q.y : j % 4 == 2 ? q.z : q.w);
    }
};

// 32 columns of the thread's row into the left or right half of a staging buffer (64 columns; the
// layout of out_stage_row), so that no registers hold the left half while the right is formed.
__device__ __forceinline__ void stage_half(uint32_t buf, int r, bool right, const uint32_t (&w)[16]) {
    const uint32_t row = buf + static_cast<uint32_t>(r) * 128u;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint32_t piece = static_cast<uint32_t>(right ? c + 4 : c) ^ (static_cast<uint32_t>(r) & 7u);
        st_shared_v4(row + (piece << 4), w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
    }
}
// Before a left half is staged: the stores that read the buffers last have done so.
template <int kBuffers>
__device__ __forceinline__ void stage_ready(const EpiIO& io) {
    if (io.lane == 0) bulk_wait_group_read<2 - kBuffers>();
    __syncwarp();
}
__device__ __forceinline__ uint32_t stage_buf(const EpiIO& io, uint32_t ahead) {
    return io.out + ((io.count + ahead) & 1u) * kOutBufBytes;
}

template <int BN>
struct EpiLinear {
    static constexpr int kWarps = 4;
    struct Params {
        CUtensorMap ymap, zmap;  // Y and Z, boxes 64 x 32
        LinearOut o;
    };
    const __nv_bfloat16* res;
    RowAhead r;

    __device__ __forceinline__ EpiLinear(const Params& p, int, int row, int n0) {
        res = p.o.residual && row < p.o.M ? p.o.residual + row * p.o.ld : nullptr;
        if (p.o.residual) r.load(res, n0, p.o.N);
        // the tile's bias into L1 while the mainloop runs: each chunk's load of it would wait for L2
        const int c = n0 + 8 * static_cast<int>(threadIdx.x & 31);
        if (p.o.bias && c < n0 + BN && c < p.o.N) touch(p.o.bias + c);
    }

    static __device__ __forceinline__ void touch(const __nv_bfloat16* p) {
        uint32_t u;
        asm volatile("ld.global.u32 %0, [%1];" : "=r"(u) : "l"(p));
    }

    __device__ __forceinline__ void chunk(const Params& p, const float (&v)[32], int col0, int c0,
                                          EpiIO& io) {
        if (io.row0 >= p.o.M || (col0 & ~63) >= p.o.N) return;
        const bool right = (c0 & 32) != 0, two = p.o.Z != nullptr;
        float2 x[16];
        RowAhead b;
        if (p.o.bias) b.load(p.o.bias, col0, p.o.N);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            x[j] = make_float2(v[2 * j], v[2 * j + 1]);
            if (p.o.bias) x[j] = add2(x[j], b.at(j));
        }
        if (!right) {
            if (two)
                stage_ready<2>(io);
            else
                stage_ready<1>(io);
        }
        uint32_t w[16];
        if (two) {
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j] = pack2(x[j]);
            stage_half(stage_buf(io, 0), io.lane, right, w);
        }
        with_act(p.o.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] = act_value2<act.value>(x[j]);
        });
        if (p.o.residual) {
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] = add2(x[j], r.at(j));
            if (c0 + 32 < BN) r.load(res, col0 + 32, p.o.N);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] = pack2(x[j]);
        stage_half(stage_buf(io, two ? 1 : 0), io.lane, right, w);
        if (!right) return;
        if (two) out_commit(io, &p.zmap, stage_buf(io, 0), col0 - 32, io.row0);
        out_commit(io, &p.ymap, stage_buf(io, 0), col0 - 32, io.row0);
    }

    __device__ __forceinline__ void finish(const Params&, int) {}
};

template <int BN>
struct EpiSlope {
    static constexpr int kWarps = 4;
    struct Params {
        CUtensorMap xmap;  // X, boxes 64 x 32
        SlopeOut o;
    };
    const __nv_bfloat16* zrow;
    RowAhead r;

    __device__ __forceinline__ EpiSlope(const Params& p, int, int row, int n0) {
        zrow = p.o.z && row < p.o.M ? p.o.z + row * p.o.ld : nullptr;
        if (p.o.z) r.load(zrow, n0, p.o.N);
    }

    __device__ __forceinline__ void chunk(const Params& p, const float (&v)[32], int col0, int c0,
                                          EpiIO& io) {
        if (io.row0 >= p.o.M || (col0 & ~63) >= p.o.N) return;
        const bool right = (c0 & 32) != 0;
        uint32_t w[16];
        if (p.o.z) {
            with_act(p.o.act, [&](auto act) {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    w[j] = pack2(mul2(make_float2(v[2 * j], v[2 * j + 1]), act_slope2<act.value>(r.at(j))));
            });
            if (c0 + 32 < BN) r.load(zrow, col0 + 32, p.o.N);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j] = pack_bf16x2(v[2 * j], v[2 * j + 1]);
        }
        if (!right) stage_ready<1>(io);
        stage_half(stage_buf(io, 0), io.lane, right, w);
        if (right) out_commit(io, &p.xmap, stage_buf(io, 0), col0 - 32, io.row0);
    }

    __device__ __forceinline__ void finish(const Params&, int) {}
};

}  // namespace fpo
