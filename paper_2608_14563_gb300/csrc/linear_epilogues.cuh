// linear_epilogues.cuh -- epilogues (tc_gemm.cuh) of the linear layer's products: bias, activation
// and residual of the forward pass, the slope of the activation below in the backward pass.
//
// One row per thread, 32 columns at a time, written through the warp's staging buffers by TMA.  The
// 8-warp form of the other epilogues that read matrices (RowChunk: the accumulator through shared
// memory, every global access 256 bytes of two rows) takes 2 to 3 times the instructions; these run
// beside the MMAs of a GPU at its power cap.
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

// 32 columns of a row, those outside the matrix (N: a multiple of 8) zeros.
struct RowPiece {
    uint4 u[4];
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int col, int N) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            u[q] = col + 8 * q < N ? *reinterpret_cast<const uint4*>(p + col + 8 * q)
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
// 32 columns of the warp's 32 rows of a matrix, loaded one chunk ahead: four lanes to a row's 64
// bytes, so that a load touches 8 rows and not 32, and handed to the rows' threads through the half of
// the staging buffer that they are about to fill.
struct TileAhead : RowPiece {
    const __nv_bfloat16* p;  // the warp's first row, or null
    int rows;                // of the matrix from there on
    __device__ __forceinline__ void next(long long ld, int col, int N) {
        const int lane = threadIdx.x & 31, c = col + 8 * (lane & 3);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 8 * i + lane / 4;
            u[i] = r < rows && c < N ? *reinterpret_cast<const uint4*>(p + r * ld + c)
                                     : make_uint4(0u, 0u, 0u, 0u);
        }
    }
    // The thread's row of them (the buffer's half is free, and is the warp's).
    __device__ __forceinline__ void deal(uint32_t buf, int lane, bool right) {
        auto piece = [&](int r, int c) {
            const uint32_t ur = static_cast<uint32_t>(r);
            return buf + ur * 128u + (((right ? c + 4u : c) ^ (ur & 7u)) << 4);
        };
#pragma unroll
        for (int i = 0; i < 4; ++i)
            st_shared_v4(piece(8 * i + lane / 4, lane & 3), u[i].x, u[i].y, u[i].z, u[i].w);
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const float4 f = ld_shared_f4(piece(lane, c));
            u[c] = make_uint4(__float_as_uint(f.x), __float_as_uint(f.y), __float_as_uint(f.z),
                              __float_as_uint(f.w));
        }
    }
};

// The epilogues' warps: two share 32 rows and take half of the columns each, with one staging buffer
// (4 warps, with two, where half a tile is less than a buffer's 64 columns).  A warp's instructions
// follow one another at latencies that a second one on its scheduler hides.  kAct: the activation, or
// kActAny where it is looked up; it is known on 256-column tiles, where the branch of every chunk cost
// a tenth of a short tile's time.  12541 tokens, 144 to 12184 features (tiles of three k-blocks), 4
// warps, 8 warps, 8 with the activation known: plain 154, 141, 131 us; bias and relu 222, 169, 143;
// with a residual too, whose load by row touched 32 lines, 322, 263 and, by 8 rows, 218; with Z 254,
// 212 and 220.
constexpr int kActAny = -1;

template <int kAct, class F>
__device__ __forceinline__ void with_known_act(int act, F&& f) {
    if constexpr (kAct == kActAny)
        with_act(act, f);
    else
        f(std::integral_constant<int, kAct>{});
}

template <int BN>
struct RowWarps {
    static constexpr int kWarps = BN >= 128 ? 8 : 4;
    static constexpr int kCols = BN / (kWarps / 4);  // of a warp
    static constexpr int kBuffers = 8 / kWarps;
    static __device__ __forceinline__ uint32_t buf(const EpiIO& io, uint32_t ahead) {
        return kBuffers == 2 ? io.out + ((io.count + ahead) & 1u) * kOutBufBytes : io.out;
    }
    // Before the next `n` buffers are written: the stores that read them last have done so.
    template <int n>
    static __device__ __forceinline__ void ready(const EpiIO& io) {
        if (io.lane == 0) bulk_wait_group_read<kBuffers - n>();
        __syncwarp();
    }
    // Whether the warp's columns go on behind the chunk at offset c0 of the tile.
    static __device__ __forceinline__ bool more(int c0) { return (c0 & (kCols - 1)) + 32 < kCols; }
};

template <int BN, int kAct>
struct EpiLinear {
    using R = RowWarps<BN>;
    static constexpr int kWarps = R::kWarps;
    static constexpr bool kByRow = true;
    struct Params {
        CUtensorMap ymap, zmap;  // Y and Z, boxes 64 x 32
        LinearOut o;
    };
    TileAhead r;
    uint32_t left[16];  // with Z and one buffer: Y's left half, until Z has left

    __device__ __forceinline__ EpiLinear(const Params& p, int, int row, int n0) {
        const int lane = static_cast<int>(threadIdx.x & 31), row0 = row - lane;
        if (p.o.residual) {
            r.p = p.o.residual + row0 * p.o.ld;
            r.rows = p.o.M - row0;
            r.next(p.o.ld, n0, p.o.N);
        }
        // the columns' bias into L1 while the mainloop runs: each chunk's load of it would wait for L2
        const int c = n0 + 8 * lane;
        if (p.o.bias && c < n0 + R::kCols && c < p.o.N) touch(p.o.bias + c);
    }

    static __device__ __forceinline__ void touch(const __nv_bfloat16* p) {
        uint32_t u;
        asm volatile("ld.global.u32 %0, [%1];" : "=r"(u) : "l"(p));
    }

    __device__ __forceinline__ void chunk(const Params& p, const float (&v)[32], int col0, int c0,
                                          EpiIO& io) {
        if (io.row0 >= p.o.M || (col0 & ~63) >= p.o.N) return;
        const bool right = (c0 & 32) != 0, two = p.o.Z != nullptr;
        const bool wait = two && R::kBuffers == 1;  // Y waits for Z to leave the one buffer
        float2 x[16];
        RowPiece b;
        if (p.o.bias) b.load(p.o.bias, col0, p.o.N);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            x[j] = make_float2(v[2 * j], v[2 * j + 1]);
            if (p.o.bias) x[j] = add2(x[j], b.at(j));
        }
        if (!right) {
            if (two && R::kBuffers == 2)
                R::template ready<R::kBuffers>(io);
            else
                R::template ready<1>(io);
        }
        uint32_t w[16];
        if (two) {
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j] = pack2(x[j]);
            stage_half(R::buf(io, 0), io.lane, right, w);
            if (wait && right) out_commit(io, &p.zmap, R::buf(io, 0), col0 - 32, io.row0);
        }
        with_known_act<kAct>(p.o.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] = act_value2<act.value>(x[j]);
        });
        if (wait && right) R::template ready<1>(io);
        if (p.o.residual) {
            // (while Z's left half waits in the one buffer, its right half is free)
            r.deal(R::buf(io, two ? 1 : 0), io.lane, right || wait);
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] = add2(x[j], r.at(j));
            if (R::more(c0)) r.next(p.o.ld, col0 + 32, p.o.N);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] = pack2(x[j]);
        if (wait && !right) {
#pragma unroll
            for (int j = 0; j < 16; ++j) left[j] = w[j];
            __syncwarp();  // every row of the right half is read before Z's is staged there
            return;
        }
        if (wait) stage_half(R::buf(io, 0), io.lane, false, left);
        stage_half(R::buf(io, two ? 1 : 0), io.lane, right, w);
        if (!right) return;
        if (two && R::kBuffers == 2) out_commit(io, &p.zmap, R::buf(io, 0), col0 - 32, io.row0);
        out_commit(io, &p.ymap, R::buf(io, 0), col0 - 32, io.row0);
    }

    __device__ __forceinline__ void finish(const Params&, int) {}
};

template <int BN, int kAct>
struct EpiSlope {
    using R = RowWarps<BN>;
    static constexpr int kWarps = R::kWarps;
    static constexpr bool kByRow = true;
    struct Params {
        CUtensorMap xmap;  // X, boxes 64 x 32
        SlopeOut o;
    };
    TileAhead z;

    __device__ __forceinline__ EpiSlope(const Params& p, int, int row, int n0) {
        const int row0 = row - static_cast<int>(threadIdx.x & 31);
        if (kAct != kActNone && p.o.z) {
            z.p = p.o.z + row0 * p.o.ld;
            z.rows = p.o.M - row0;
            z.next(p.o.ld, n0, p.o.N);
        }
    }

    __device__ __forceinline__ void chunk(const Params& p, const float (&v)[32], int col0, int c0,
                                          EpiIO& io) {
        if (io.row0 >= p.o.M || (col0 & ~63) >= p.o.N) return;
        const bool right = (c0 & 32) != 0;
        if (!right) R::template ready<1>(io);
        uint32_t w[16];
        if (kAct != kActNone && p.o.z) {
            z.deal(R::buf(io, 0), io.lane, right);
            with_known_act<kAct>(p.o.act, [&](auto act) {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    w[j] = pack2(mul2(make_float2(v[2 * j], v[2 * j + 1]), act_slope2<act.value>(z.at(j))));
            });
            if (R::more(c0)) z.next(p.o.ld, col0 + 32, p.o.N);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j] = pack_bf16x2(v[2 * j], v[2 * j + 1]);
        }
        stage_half(R::buf(io, 0), io.lane, right, w);
        if (right) out_commit(io, &p.xmap, R::buf(io, 0), col0 - 32, io.row0);
    }

    __device__ __forceinline__ void finish(const Params&, int) {}
};

}  // namespace fpo
