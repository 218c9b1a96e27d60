// linear_gemm_f32.hip -- the dense layer's matrix products of fp32 operands, formed on the
// bf16 matrix cores from three parts of each value (bf16x3.h: six part products, the leading
// one and the five smaller ones in sums of their own).
//
// A workgroup of eight (64 x 64: four) waves computes a TM x TN tile of C, its K loop over
// chunks of 32. A chunk's values are loaded into registers at the end of the chunk before the
// last, split there while the last one is on the matrix cores, between its products, and
// written to the other of two LDS buffers as three bf16 tiles (linear_tile.h): one barrier a
// chunk. So 4 bytes a value come from L2, not the 6 of parts made beforehand, and no pass
// makes them (4,096 x 1,024 x 1,024 55 us, 66 with parts beforehand and their passes).
//
// Bound by the matrix cores and their power: 8,192 x 4,096 x 4,096 runs at 206 TFLOP/s, 1.24
// PFLOP/s of bf16 products, what the 16-bit tiles reach. Two chunks of loads ahead, three
// LDS buffers, the first operands of a chunk read before its barrier, and other shares of
// vector instructions between the products change 4,096 x 1,024 x 1,024 by 3 % at most.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "linear_tile.h"

namespace mlp {

constexpr int FK = 32;   // depth of a chunk

// 16 bytes at any float's address
struct __attribute__((packed, aligned(4))) Float4 {
    float e[4];
};

// One operand's chunks: TX values of x by FK of k, moved by NT threads, four values that
// are contiguous in memory at a time.
template <bool XC, int TX, int NT>
struct Operand32 : LdsTile<XC, TX, FK> {
    using L = LdsTile<XC, TX, FK>;
    using L::ROW;
    using L::swz;
    static constexpr int LOADS = TX * FK / 4 / NT;
    static constexpr int ELEMS = TX * FK;   // of a part
    static_assert(TX * FK / 4 % NT == 0, "every thread moves the same number of pieces");

    const char *base;        // XC: the start of the chunk's first row; else the tile's corner
    uint32_t off[LOADS];     // bytes from it
    int64_t step, ld;
    int end;                 // XC: columns from the row's start, else k from the chunk's to the row's end
    f4 v[LOADS];

    static __device__ __forceinline__ int row_of(int i) { return (i * NT + threadIdx.x) / (ROW / 4); }
    static __device__ __forceinline__ int col_of(int i) { return (i * NT + threadIdx.x) % (ROW / 4) * 4; }

    // o.p: fp32 rows of o.ld elements, o.len of them readable (four at least; what pads a row is
    // zero)
    bool edge;               // XC: the tile reaches past the rows' end
    __device__ __forceinline__ void init(const Operand &o, int64_t x0, int64_t xlim, int64_t k0) {
        const float *p = reinterpret_cast<const float *>(o.p);
        ld = 4 * o.ld;
        const int rows = (int)(xlim - x0 < TX ? xlim - x0 : TX);
        base = (const char *)(XC ? p + k0 * o.ld : p + x0 * o.ld + k0);
        step = XC ? FK * ld : 4 * FK;
        end = (int)(XC ? o.len : o.len - k0);
        edge = XC && x0 + TX > o.len;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            // rows past the matrix in x give sums that are not kept: the last one is read
            const int r = row_of(i);
            off[i] = XC ? (uint32_t)r * (uint32_t)ld + 4u * (uint32_t)((int)x0 + col_of(i))
                        : (uint32_t)(r < rows ? r : rows - 1) * (uint32_t)ld + 4u * (uint32_t)col_of(i);
        }
    }
    static __device__ __forceinline__ f4 get(const char *p) {
        const Float4 w = *reinterpret_cast<const Float4 *>(p);
        return f4{w.e[0], w.e[1], w.e[2], w.e[3]};
    }
    // four values `over` places past the last four of a row, those past its end 0
    static __device__ __forceinline__ f4 shifted(f4 w, int over) {
        w = over & 1 ? f4{w[1], w[2], w[3], 0.f} : w;
        w = over & 2 ? f4{w[2], w[3], 0.f, 0.f} : w;
        return over & ~3 ? f4{0.f, 0.f, 0.f, 0.f} : w;
    }
    // the chunk at base to the registers, base to the next; left: its k
    __device__ __forceinline__ void load(int64_t left) {
        if (left >= FK && !edge) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) v[i] = get(base + off[i]);
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                if constexpr (XC) {
                    const int x = (int)(off[i] - (uint32_t)row_of(i) * (uint32_t)ld) / 4, over = x > end - 4 ? x - (end - 4) : 0;
                    const int r = row_of(i) < left ? row_of(i) : (int)left - 1;
                    const f4 w = shifted(get(base + (r * ld + 4 * (x - over))), over);
                    v[i] = row_of(i) < left ? w : f4{0.f, 0.f, 0.f, 0.f};
                } else {
                    const int k = col_of(i), over = k > end - 4 ? k - (end - 4) : 0;
                    v[i] = shifted(get(base + off[i] - 4 * over), over);
                }
            }
        }
        base += step;
        if (!XC) end -= FK;
    }
    // load i's values, split, to the LDS tiles of the three parts at S
    __device__ __forceinline__ void stash(uint16_t *S, int i) const {
        uint32_t w[2][3];
        split_pair(v[i][0], v[i][1], w[0]);
        split_pair(v[i][2], v[i][3], w[1]);
        const int r = row_of(i), c = col_of(i), at = r * ROW + ((((c >> 3) ^ swz(r)) << 3) | (c & 4));
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<u2v *>(S + p * ELEMS + at) = u2v{w[0][p], w[1][p]};
    }
};

// The operands of 16 k for a wave's products, in parts.
template <int NJ, int MI>
struct Frags32 {
    u4v a[MI][3], b[NJ][3];
    template <class TA, class TB>
    __device__ __forceinline__ void fetch(const uint16_t *A, const uint16_t *B, int wm, int wn, int kk) {
#pragma unroll
        for (int p = 0; p < 3; ++p) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) b[j][p] = TB::frag(B + p * TB::ELEMS, wn + 32 * j, kk);
#pragma unroll
            for (int i = 0; i < MI; ++i) a[i][p] = TA::frag(A + p * TA::ELEMS, wm + 32 * i, kk);
        }
    }
    __device__ __forceinline__ void multiply(f16v (&acc)[NJ][MI], f16v (&lo)[NJ][MI]) const {
        constexpr int PA[5] = {2, 1, 0, 1, 0}, PB[5] = {0, 1, 2, 0, 1};
#pragma unroll
        for (int p = 0; p < 5; ++p)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int i = 0; i < MI; ++i) lo[j][i] = mfma_bf16_32(b[j][PB[p]], a[i][PA[p]], lo[j][i]);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int i = 0; i < MI; ++i) acc[j][i] = mfma_bf16_32(b[j][0], a[i][0], acc[j][i]);
    }
};

template <int OP, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_gemm_f32(const GemmArgs g) {
    constexpr int NT = 64 * WM * WN, MI = TM / WM / 32, NJ = TN / WN / 32;
    typedef Operand32<OP == GEMM_TN, TM, NT> TA;
    typedef Operand32<OP != GEMM_NT, TN, NT> TB;
    constexpr int STAGE = 3 * (TA::ELEMS + TB::ELEMS);
    static_assert(WM * WN * 32 * RESULT_STRIDE<NJ> * 4 <= 4 * STAGE, "the results fit where the chunks were");
    __shared__ __attribute__((aligned(16))) uint16_t lds[2 * STAGE];
    const int wave = threadIdx.x >> 6;
    const int wm = wave / WN * (TM / WM), wn = wave % WN * (TN / WN);
    const TileAt at(g, TM, TN);
    const int nk = (int)((at.ke - at.kb + FK - 1) / FK);
    f16v acc[NJ][MI], lo[NJ][MI];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[j][i][v] = lo[j][i][v] = 0.f;
    if (nk > 0) {
        TA a;
        TB b;
        a.init(g.A, at.m0, g.M, at.kb);
        b.init(g.B, at.n0, g.N, at.kb);
        int64_t left = at.ke - at.kb;   // k from the chunk to be loaded next to the end
        auto load = [&]() __attribute__((always_inline)) {
            if (left > 0) {
                a.load(left);
                b.load(left);
                left -= FK;
            }
        };
        auto stash = [&](uint16_t *S, int half) __attribute__((always_inline)) {
            if (half == 0) {
#pragma unroll
                for (int i = 0; i < TA::LOADS; ++i) a.stash(S, i);
            } else {
#pragma unroll
                for (int i = 0; i < TB::LOADS; ++i) b.stash(S + 3 * TA::ELEMS, i);
            }
        };
        load();
        stash(lds, 0);
        stash(lds, 1);
        load();
        uint16_t *now = lds, *next = lds + STAGE;
        for (int c = 0; c < nk; ++c) {
            // every wave has written chunk c, and read chunk c - 1, whose buffer c + 1 takes
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            constexpr int SETS = MI * NJ <= 2 ? 2 : 1;   // (with two, 256 x 128 spills)
            Frags32<NJ, MI> f[SETS];
#pragma unroll
            for (int kk = 0; kk < SETS; ++kk) f[kk].template fetch<TA, TB>(now, now + 3 * TA::ELEMS, wm, wn, kk);
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                if (kk >= SETS) f[0].template fetch<TA, TB>(now, now + 3 * TA::ELEMS, wm, wn, kk);
                stash(next, kk);   // (past the last chunk: values that nothing reads)
                f[kk % SETS].multiply(acc, lo);
#pragma unroll
                for (int e = 0; e < 6 * MI * NJ; ++e) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            load();
            uint16_t *t = now;
            now = next;
            next = t;
        }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < MI; ++i) acc[j][i] += lo[j][i];
    finish_tile<float>(g, at, wm, wn, acc, reinterpret_cast<float *>(lds));
}

template <int OP, int TM, int TN, int WM, int WN>
static hipError_t tiles_f32(GemmArgs g, int64_t part_floats, hipStream_t stream) {
    // (A chunk takes 0.5 us on 64 x 64 tiles, 1.3 on 128 x 128. Where many 64 x 64 tiles are
    // deep, two workgroups a compute unit: 700 x 16,384 x 300 196 us with one, 103 with two;
    // dW of 3,000 x 10,001 x 30 141 and 64; 1,024 x 1,024 x 1,024 22 and 27)
    const bool two = TM == 64 && g.K > 64 * FK && ceil_div(g.M, TM) * ceil_div(g.N, TN) >= 32;
    const unsigned grid = plan_tiles(g, TM, TN, FK, two ? 2 * CUS : CUS, TM == 64 ? 9 : 4, part_floats);
    hipLaunchKernelGGL((k_gemm_f32<OP, TM, TN, WM, WN>), dim3(grid), dim3(64 * WM * WN), 0, stream, g);
    if (hipError_t e = hipGetLastError()) return e;
    return join_splits<float>(g, stream);
}

// The tile by the number of tiles, 64 x 64 where larger ones would cover over 5/4 of what
// those do (65,536 x 64 x 1,024 on 64 x 64 84 us, on 128 x 128 144, 65,536 x 192 x 256 56 and
// 71):
// 256 x 128 where there are many (us, of outputs x depth: 4,096 x 2,048 x 2,048 191, on 128 x
// 128 205; 2,048 x 2,048 x 2,048 106 and 94; TN, which spills 29 registers, 4,096 x 4,096 x
// 8,192 1,586 and 1,645, 4,096 x 2,048 x 2,048 244 and 209);
// 128 x 128 where no split is needed (2,048 x 2,048 x 2,048 94, on 64 x 64 125) or the depth pays
// for the splits' joining (1,024 x 1,024 x 2,048 40 and 52, of 1,024 29 and 23).
template <int OP>
static hipError_t op_f32(const GemmArgs &g, int64_t part_floats, hipStream_t stream) {
    const int64_t mid = ceil_div(g.M, 128) * ceil_div(g.N, 128);
    if (16 * mid <= 5 * ceil_div(g.M, 64) * ceil_div(g.N, 64)) {
        if (mid >= (OP == GEMM_TN ? 1024 : 400)) return tiles_f32<OP, 256, 128, 4, 2>(g, part_floats, stream);
        if (mid > CUS / 2 || (mid >= 16 && g.K > 1024)) return tiles_f32<OP, 128, 128, 2, 4>(g, part_floats, stream);
    }
    return tiles_f32<OP, 64, 64, 2, 2>(g, part_floats, stream);
}

hipError_t launch_gemm_f32(int op, const GemmArgs &g, int64_t part_floats, hipStream_t stream) {
    switch (op) {
    case GEMM_NN: return op_f32<GEMM_NN>(g, part_floats, stream);
    case GEMM_NT: return op_f32<GEMM_NT>(g, part_floats, stream);
    default: return op_f32<GEMM_TN>(g, part_floats, stream);
    }
}

}  // namespace mlp
