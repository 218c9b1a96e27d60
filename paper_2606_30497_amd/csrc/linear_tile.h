// linear_tile.h -- what the dense layer's tile kernels (linear_gemm.hip, linear_gemm_f32.hip)
// share: operand tiles in LDS, the order of the tiles, and the way of a tile's results
// through the epilogue.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include <type_traits>

#include "linear_internal.h"

namespace mlp {

typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef short s4v __attribute__((ext_vector_type(4)));

// A tile of 16-bit operand values in LDS, TX values of x by BK of k. XC: as [k][x] (x is
// contiguous in memory), read by ds_read_b64_tr_b16, which hands each lane four consecutive
// k of its x; else as [x][k], read in 16-byte pieces. The pieces of a row are permuted by
// the row's number: LDS has 64 banks of 4 bytes, and the 16 rows that a 16-byte read meets
// at one piece, or the four rows that a transposing read meets at two pieces each, fall on
// all of them.
template <bool XC, int TX, int BK>
struct LdsTile {
    static constexpr int K = BK, ROW = XC ? TX : BK;   // elements of a row
    static constexpr int READS = XC ? 2 : 1;           // LDS reads of a fragment
    static __device__ __forceinline__ int swz(int row) {
        if constexpr (XC) return TX >= 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
        else return BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3;
    }
    // k in [16 kk, 16 kk + 16) of x in [x, x + 32), as an MFMA operand: lane l has x + l
    // % 32 and the eight k of its half l / 32
    static __device__ __forceinline__ u4v frag(const uint16_t *S, int x, int kk) {
        const int l = threadIdx.x & 63;
        if constexpr (XC) {
            // of 16 lanes, four read four x of one of four consecutive k each
            const int k = 16 * kk + 8 * (l >> 5) + ((l >> 2) & 3), xx = x + 16 * ((l >> 4) & 1) + 4 * (l & 3);
            const int at = (((xx >> 3) ^ swz(k)) << 3) | (xx & 7);
            typedef __attribute__((address_space(3))) s4v lds4;
            const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(uintptr_t)(S + k * ROW + at));
            const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(uintptr_t)(S + (k + 4) * ROW + at));
            const u2v a = __builtin_bit_cast(u2v, lo), b = __builtin_bit_cast(u2v, hi);
            return u4v{a[0], a[1], b[0], b[1]};
        } else {
            const int row = x + (l & 31), c = 2 * kk + (l >> 5);
            return *reinterpret_cast<const u4v *>(S + row * ROW + ((c ^ swz(row)) << 3));
        }
    }
};

// A wave's LDS writes before its lanes' reads of one another's (and the reverse).
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// f(0), f(1), ... f(N - 1), each with its number as a constant
template <int N, int I = 0, class F>
__device__ __forceinline__ void unrolled(F f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        unrolled<N, I + 1>(f);
    }
}

// The tile and split of this workgroup. Workgroups go round the eight XCDs in turn: each XCD
// takes consecutive tiles, eight rows of tiles at a time down a column, so that its L2
// keeps what they share.
struct TileAt {
    int split;
    int64_t m0, n0, kb, ke;   // its corner, its depth
    __device__ __forceinline__ TileAt(const GemmArgs &g, int TM, int TN) {
        const int tiles = g.tiles_m * g.tiles_n;
        int id = blockIdx.x;
        split = id / tiles;
        id -= split * tiles;
        const int per = tiles / 8, extra = tiles % 8, x = id % 8;
        id = x * per + (x < extra ? x : extra) + id / 8;
        const int band = 8 * g.tiles_n, b0 = id / band * 8;
        const int bh = g.tiles_m - b0 < 8 ? g.tiles_m - b0 : 8;
        const int in = id % band;
        m0 = (int64_t)(b0 + in % bh) * TM;
        n0 = (int64_t)(in / bh) * TN;
        kb = (int64_t)split * g.kc;
        ke = kb + g.kc < g.K ? kb + g.kc : g.K;
    }
};

// A wave's results (32 x 32 MFMA tiles of its 32 MI rows from wm on by 32 NJ columns from wn
// on, the columns the first operand), 32 rows at a time, through LDS (lds: 32 rows of
// RESULT_STRIDE floats for each wave): a lane's registers hold four columns here and there
// of one row, memory is read and written along the rows. A lane's columns are the same in
// all rows; the residual's rows are read ahead. FOLD: columns 8 to 15 are added to the first eight,
// which are all there are.
template <int NJ>
constexpr int RESULT_STRIDE = 32 * NJ + 4;

template <class T, bool FOLD = false, int NJ, int MI>
__device__ __forceinline__ void finish_tile(const GemmArgs &g, const TileAt &at, int wm, int wn,
                                            const f16v (&acc)[NJ][MI], float *lds) {
    constexpr int WTN = 32 * NJ, CS = RESULT_STRIDE<NJ>;
    const int lane = threadIdx.x & 63;
    __syncthreads();
    float *C = lds + (threadIdx.x >> 6) * 32 * CS;
    constexpr int GROUPS = WTN / 8, ROWS = 64 / GROUPS, ITERS = 32 / ROWS;
    const int lr = lane / GROUPS;
    const int64_t m1 = at.m0 + wm + lr, n = at.n0 + wn + 8 * (lane % GROUPS);
    const bool whole = g.splits == 1;
    Finish<T> fin;
    if (whole) fin.init(g.e, n, g.N);
#pragma unroll 1
    for (int i = 0; i < MI; ++i) {
#pragma unroll
        for (int ii = 0; ii < MI; ++ii)
            if (ii == i) {
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        f4 v;
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = acc[j][ii][4 * q + r];
                        *reinterpret_cast<f4 *>(C + (lane & 31) * CS + 32 * j + 8 * q + 4 * (lane >> 5)) = v;
                    }
            }
        const int64_t m = m1 + 32 * i;
        Oct<T> res[ITERS];
        if (whole && g.e.R) {
#pragma unroll
            for (int k = 0; k < ITERS; ++k)
                if (m + k * ROWS < g.M && n < g.N) res[k] = fetch8((const T *)g.e.R + (m + k * ROWS) * g.e.ldr, n, g.N);
        }
        wave_sync();
#pragma unroll
        for (int k = 0; k < ITERS; ++k) {
            const int64_t r = m + k * ROWS;
            if (r >= g.M || n >= g.N) continue;
            float v[8];
            const f4 *c = reinterpret_cast<const f4 *>(C + (lr + k * ROWS) * CS + 8 * (lane % GROUPS));
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] = c[x / 4][x % 4];
            if constexpr (FOLD) {
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] += c[2 + x / 4][x % 4];
            }
            if (!whole) store8(g.part + ((int64_t)at.split * g.M + r) * g.N, n, g.N, v);
            else fin.finish(g.e, r, n, g.N, v, res[k]);
        }
        wave_sync();
    }
}

constexpr int CUS = 256;

// The launch plan of TM x TN tiles and chunks of BK: splits of the depth where the tiles
// are fewer than `most` workgroups, of four chunks at least, as far as there is room, and
// where they spare a tile at least `worth` chunks, the time of the splits' joining (a launch
// and the sums' way through memory: 4 to 5 us).
inline unsigned plan_tiles(GemmArgs &g, int TM, int TN, int BK, int most, int worth, int64_t part_floats) {
    g.tiles_m = (int)ceil_div(g.M, TM);
    g.tiles_n = (int)ceil_div(g.N, TN);
    const int64_t tiles = (int64_t)g.tiles_m * g.tiles_n, chunks = ceil_div(g.K, BK);
    int64_t splits = tiles < most ? most / tiles : 1;
    if (splits > chunks / 4) splits = chunks / 4;
    if (splits > part_floats / (g.M * g.N)) splits = part_floats / (g.M * g.N);
    if (splits < 1 || chunks - ceil_div(chunks, splits) < worth) splits = 1;
    g.kc = ceil_div(chunks, splits) * BK;
    g.splits = g.K > 0 ? (int)ceil_div(g.K, g.kc) : 1;
    return (unsigned)(tiles * g.splits);
}

}  // namespace mlp
