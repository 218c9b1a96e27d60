// linear_gemm.hip -- the dense layer's matrix products on the matrix cores (gfx950):
// bf16 and fp16 operands as they are, fp32 ones as three bf16 parts (bf16x3.h: six part
// products each, the leading one and the five smaller ones in sums of their own).
//
// A workgroup computes a TM x TN tile of C; its K loop runs over chunks of BK staged in
// LDS, in three to five stages: a chunk's loads go straight to LDS while the chunks before
// it are on the matrix cores, one barrier a chunk. The products are v_mfma_f32_32x32x16 with
// B as the first operand, so that four of a lane's results in a row lie along a row of C.
//
// An operand whose k is contiguous lies in LDS as [x][k], read in 16-byte pieces; one
// whose x is contiguous as [k][x], read by ds_read_b64_tr_b16, which hands each lane
// four consecutive k of its x. The 16-byte pieces of a row are permuted by the row's
// number, by way of the addresses they are loaded from, to spread reads over the banks.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <type_traits>

#include "linear_internal.h"

namespace mlp {

typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef short s4v __attribute__((ext_vector_type(4)));

template <class T>
__device__ __forceinline__ f16v mma(u4v a, u4v b, f16v c);
template <>
__device__ __forceinline__ f16v mma<bf16>(u4v a, u4v b, f16v c) {
    return mfma_bf16_32(a, b, c);
}
template <>
__device__ __forceinline__ f16v mma<f16>(u4v a, u4v b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8v, a), __builtin_bit_cast(h8v, b), c, 0, 0, 0);
}

// Where lanes with nothing to load (past the end of K) load from.
static __device__ __attribute__((aligned(16))) uint32_t g_zeros[4] = {0, 0, 0, 0};

__device__ __forceinline__ void to_lds(const void *g, void *l) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)(uintptr_t)g,
                                     (__attribute__((address_space(3))) uint32_t *)(uintptr_t)l, 16, 0, 0);
}

// One operand's chunks: TX values of x by BK of k, NP parts, moved by NT threads.
// XC: x is contiguous in memory (P[k][x]), else k is (P[x][k]).
template <bool XC, int TX, int BK, int NP, int NT>
struct Tile {
    static constexpr int K = BK, PARTS = NP;
    static constexpr int ROW = XC ? TX : BK;              // elements of an LDS row
    static constexpr int PIECES = TX * BK / 8;            // 16-byte pieces of a part
    static constexpr int LOADS = PIECES / NT;
    static constexpr int READS = XC ? 2 : 1;              // LDS reads of a fragment
    static constexpr int ELEMS = NP * TX * BK;
    static_assert(PIECES % NT == 0, "every thread moves the same number of pieces");

    const char *base;        // the current chunk's corner, uniform
    uint32_t off[LOADS];     // bytes from it
    int64_t step, plane;     // bytes to the next chunk, to the next part

    // The permutation of a row's pieces: LDS has 64 banks of 4 bytes, and the 16 rows
    // that a 16-byte read meets at one piece, or the four rows that a transposing read
    // meets at two pieces each, fall on all of them.
    static __device__ __forceinline__ int swz(int row) {
        if constexpr (XC) return TX >= 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
        else return BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3;
    }
    __device__ __forceinline__ void init(const Operand &o, int64_t x0, int64_t xlim, int64_t k0) {
        base = (const char *)(o.p + (XC ? k0 * o.ld + x0 : x0 * o.ld + k0));
        step = 2 * (XC ? BK * o.ld : (int64_t)BK);
        plane = 2 * o.plane;
        // what lies past the matrix in x gives sums that are not kept: any value will
        // do, the last row or piece of the matrix is read in its place
        const int last = (int)(xlim - x0 < TX ? xlim - x0 : TX) - 1;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int q = i * NT + threadIdx.x, row = q / (ROW / 8), c = (q % (ROW / 8)) ^ swz(row);
            const int at = XC ? (c < last / 8 ? c : last / 8) : c, r = XC ? row : (row < last ? row : last);
            off[i] = 2u * (uint32_t)(r * (uint32_t)o.ld + 8u * at);
        }
    }
    // one of the NP * LOADS loads of the chunk at base to the LDS tile S; TAIL: only k <
    // left is there, zeros take the place of the rest
    template <bool TAIL>
    __device__ __forceinline__ void load(uint16_t *S, int n, int left) const {
        const int p = n / LOADS, i = n % LOADS;
        uint16_t *d = S + p * (TX * BK) + 8 * (i * NT + (threadIdx.x & ~63u));
        const char *g = base + p * plane + off[i];
        if constexpr (TAIL) {
            const int q = i * NT + threadIdx.x, row = q / (ROW / 8);
            const int k = XC ? row : 8 * ((q % (ROW / 8)) ^ swz(row));
            if (k >= left) g = (const char *)g_zeros;
        }
        to_lds(g, d);
    }
    // k in [16 kk, 16 kk + 16) of x in [x, x + 32), as an MFMA operand: lane l has x + l
    // % 32 and the eight k of its half l / 32
    static __device__ __forceinline__ u4v frag(const uint16_t *S, int x, int kk, int p) {
        const int l = threadIdx.x & 63;
        S += p * (TX * BK);
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

template <int NP, int NJ, int MI>
struct Sums {
    f16v acc[NJ][MI], lo[NP == 3 ? NJ : 1][NP == 3 ? MI : 1];
};

// Loads [n0, n1) of a chunk of both operands (the A tile's, then the B tile's).
template <bool TAIL, int N0, int N1, class TA, class TB>
__device__ __forceinline__ void load_some(const TA &a, const TB &b, uint16_t *An, uint16_t *Bn, int left) {
    constexpr int NA = TA::PARTS * TA::LOADS;
#pragma unroll
    for (int n = N0; n < N1; ++n) {
        if (n < NA) a.template load<TAIL>(An, n, left);
        else b.template load<TAIL>(Bn, n - NA, left);
    }
}

// Every wave has loaded its pieces but for the last N loads it issued, and is done with
// what it read before.
template <int N>
__device__ __forceinline__ void loaded_all_but() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The operands of 16 k for a wave's products.
template <int NP, int NJ, int MI>
struct Frags {
    u4v a[MI][NP], b[NJ][NP];
    template <class TA, class TB>
    __device__ __forceinline__ void fetch(const uint16_t *A, const uint16_t *B, int wm, int wn, int kk) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) b[j][p] = TB::frag(B, wn + 32 * j, kk, p);
#pragma unroll
            for (int i = 0; i < MI; ++i) a[i][p] = TA::frag(A, wm + 32 * i, kk, p);
        }
    }
    // the products of row j of the wave's tiles
    template <class T>
    __device__ __forceinline__ void multiply(Sums<NP, NJ, MI> &s, int j) const {
        if constexpr (NP == 3) {
            constexpr int PA[5] = {2, 1, 0, 1, 0}, PB[5] = {0, 1, 2, 0, 1};
#pragma unroll
            for (int p = 0; p < 5; ++p)
#pragma unroll
                for (int i = 0; i < MI; ++i) s.lo[j][i] = mfma_bf16_32(b[j][PB[p]], a[i][PA[p]], s.lo[j][i]);
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            if constexpr (NP == 3) s.acc[j][i] = mfma_bf16_32(b[j][0], a[i][0], s.acc[j][i]);
            else s.acc[j][i] = mma<T>(b[j][0], a[i][0], s.acc[j][i]);
        }
    }
};

// One chunk (at Ac, Bc) on the matrix cores, while a later one is loaded (to An, Bn): each
// 16 k are read from LDS while the 16 before are multiplied; f[0] holds the chunk's first.
// AHEAD (three stages or more): the first of the chunk that follows (at Af, Bf) are read
// too. The buffers are restrict parameters of a function of its own: only so does the
// compiler know that the loads to LDS in flight do not write what is read here, and does
// not wait for them first. The loads are spread over the products, since a wave that
// issues them in a row waits for the address unit, which takes 16 cycles for each (TN of
// 8,192 x 8,192 x 8,192 in bf16 1,218 us in a row, 870 us spread); with two stages over
// the first three eighths of the chunk (NT 875 us; over five eighths 911, over all 934).
template <bool TAIL, bool AHEAD, class T, int NP, int NJ, int MI, class TA, class TB>
__device__ __forceinline__ void chunk_step(const TA &a, const TB &b, Sums<NP, NJ, MI> &sum,
                                           Frags<NP, NJ, MI> (&f)[2], uint16_t *__restrict__ An,
                                           uint16_t *__restrict__ Bn, const uint16_t *__restrict__ Ac,
                                           const uint16_t *__restrict__ Bc, const uint16_t *__restrict__ Af,
                                           const uint16_t *__restrict__ Bf, int left, int wm, int wn) {
    constexpr int KK = TA::K / 16, SLOTS = AHEAD ? KK * NJ : (3 * KK * NJ + 7) / 8;
    constexpr int ALL = TA::PARTS * TA::LOADS + TB::PARTS * TB::LOADS;
    constexpr int MFMAS = MI * (NP == 3 ? 6 : 1);
    constexpr int EACH = 2;   // LDS reads after a product
    static_assert(KK % 2 == 0, "the next chunk's first operands go to f[0]");
    unrolled<KK>([&](auto kkc) __attribute__((always_inline)) {
        constexpr int kk = decltype(kkc)::value;
        if constexpr (kk + 1 < KK) f[(kk + 1) & 1].template fetch<TA, TB>(Ac, Bc, wm, wn, kk + 1);
        else if constexpr (AHEAD) f[0].template fetch<TA, TB>(Af, Bf, wm, wn, 0);
        unrolled<NJ>([&](auto jc) __attribute__((always_inline)) {
            constexpr int j = decltype(jc)::value, slot = kk * NJ + j;
            if constexpr (slot < SLOTS)
                load_some<TAIL, ALL * slot / SLOTS, ALL *(slot + 1) / SLOTS>(a, b, An, Bn, left);
            f[kk & 1].template multiply<T>(sum, j);
#pragma unroll
            for (int n = 0; n < MFMAS; ++n) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
            }
        });
        __builtin_amdgcn_sched_barrier(0);
    });
}

// TM x TN outputs, WM x WN waves, each TM / WM x TN / WN outputs as 32 x 32 MFMA tiles.
// T: the type of C; NP = 3: fp32 operands in parts. S: LDS stages, each a chunk of both
// operands.
template <class T, int OP, int TM, int TN, int BK, int S, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_gemm_tile(const GemmArgs g) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1, NT = 64 * WM * WN;
    constexpr int MI = TM / WM / 32, NJ = TN / WN / 32;
    typedef Tile<OP == GEMM_TN, TM, BK, NP, NT> TA;
    typedef Tile<OP != GEMM_NT, TN, BK, NP, NT> TB;
    constexpr int WTN = TN / WN, CS = WTN + 4;   // a wave's columns; row stride of its results in LDS
    static_assert(WM * WN * 32 * CS * 4 <= 2 * S * (TA::ELEMS + TB::ELEMS), "the results fit where the chunks were");
    constexpr int STAGE = TA::ELEMS + TB::ELEMS;
    __shared__ __attribute__((aligned(16))) uint16_t lds[S * STAGE];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave / WN * (TM / WM), wn = wave % WN * (TN / WN);

    // Workgroups go round the eight XCDs in turn: each XCD takes consecutive tiles, eight
    // rows of tiles at a time down a column, so that its L2 keeps what they share.
    const int tiles = g.tiles_m * g.tiles_n;
    int id = blockIdx.x;
    const int split = id / tiles;
    id -= split * tiles;
    {
        const int per = tiles / 8, extra = tiles % 8, x = id % 8;
        id = x * per + (x < extra ? x : extra) + id / 8;
    }
    const int band = 8 * g.tiles_n, b0 = id / band * 8;
    const int bh = g.tiles_m - b0 < 8 ? g.tiles_m - b0 : 8;
    const int in = id % band;
    const int64_t m0 = (int64_t)(b0 + in % bh) * TM, n0 = (int64_t)(in / bh) * TN;

    const int64_t kb = (int64_t)split * g.kc, ke = kb + g.kc < g.K ? kb + g.kc : g.K;
    const int nk = (int)((ke - kb + BK - 1) / BK);
    Sums<NP, NJ, MI> sum;
    auto &acc = sum.acc;
    auto &lo = sum.lo;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                acc[j][i][v] = 0.f;
                if constexpr (NP == 3) lo[j][i][v] = 0.f;
            }

    if (nk > 0) {
        TA a;
        TB b;
        a.init(g.A, m0, g.M, kb);
        b.init(g.B, n0, g.N, kb);
        // S - 1 chunks are on their way before the first is used. At chunk c's barrier
        // every wave has loaded chunks c and c + 1 and read all of chunk c - 1, whose
        // stage chunk c + S - 1 takes. (Past the last chunk zeros are loaded, so that the
        // waits stay the same.)
        constexpr bool AHEAD = S > 2;
        constexpr int PER = TA::PARTS * TA::LOADS + TB::PARTS * TB::LOADS;
        int64_t left = ke - kb;   // k from the chunk to be loaded next to the end
        Frags<NP, NJ, MI> f[2];
#pragma unroll
        for (int s = 0; s < S - 1; ++s) {
            uint16_t *d = lds + s * STAGE;
            if (left >= BK) load_some<false, 0, PER>(a, b, d, d + TA::ELEMS, BK);
            else load_some<true, 0, PER>(a, b, d, d + TA::ELEMS, (int)left);
            a.base += a.step;
            b.base += b.step;
            left -= BK;
        }
        if constexpr (AHEAD) {
            loaded_all_but<PER *(S - 2)>();
            f[0].template fetch<TA, TB>(lds, lds + TA::ELEMS, wm, wn, 0);
        }
        int now = 0;
        auto chunk = [&](auto tail) __attribute__((always_inline)) {
            loaded_all_but<AHEAD ? PER *(S - 3) : 0>();
            if constexpr (!AHEAD) f[0].template fetch<TA, TB>(lds + now, lds + now + TA::ELEMS, wm, wn, 0);
            const int last = now == 0 ? (S - 1) * STAGE : now - STAGE;
            const int next = now == (S - 1) * STAGE ? 0 : now + STAGE;
            chunk_step<decltype(tail)::value, AHEAD, T>(a, b, sum, f, lds + last, lds + last + TA::ELEMS, lds + now,
                                                 lds + now + TA::ELEMS, lds + next, lds + next + TA::ELEMS,
                                                 (int)left, wm, wn);
            now = next;
            a.base += a.step;
            b.base += b.step;
            left -= BK;
        };
        int c = 0;
        for (; left >= BK; ++c) chunk(std::false_type());
        for (; c < nk; ++c) chunk(std::true_type());
    }

    // The results, 32 rows of a wave at a time, through LDS: a lane's registers hold four
    // columns here and there of one row, memory is read and written along the rows. A
    // lane's columns are the same in all rows; the residual's rows are read ahead.
    __syncthreads();
    float *C = reinterpret_cast<float *>(lds) + wave * 32 * CS;
    constexpr int GROUPS = WTN / 8, ROWS = 64 / GROUPS, ITERS = 32 / ROWS;
    const int lr = lane / GROUPS;
    const int64_t m1 = m0 + wm + lr, n = n0 + wn + 8 * (lane % GROUPS);
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
                        for (int r = 0; r < 4; ++r) {
                            v[r] = acc[j][ii][4 * q + r];
                            if constexpr (NP == 3) v[r] += lo[j][ii][4 * q + r];
                        }
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
            if (!whole) store8(g.part + ((int64_t)split * g.M + r) * g.N, n, g.N, v);
            else fin.finish(g.e, r, n, g.N, v, res[k]);
        }
        wave_sync();
    }
}

// The splits' sums, in order, through the epilogue.
template <class T>
__global__ __launch_bounds__(256) void k_gemm_join(const GemmArgs g) {
    const int64_t blocks = (g.N + 7) / 8, total = g.M * blocks, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
        const int64_t m = i / blocks, n = (i - m * blocks) * 8;
        Finish<T> fin;
        fin.init(g.e, n, g.N);
        Oct<T> res;
        if (g.e.R) res = fetch8((const T *)g.e.R + m * g.e.ldr, n, g.N);
        float v[8];
        load8(g.part + m * g.N, n, g.N, v);
#pragma unroll 4
        for (int s = 1; s < g.splits; ++s) {
            float w[8];
            load8(g.part + (s * g.M + m) * g.N, n, g.N, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += w[j];
        }
        fin.finish(g.e, m, n, g.N, v, res);
    }
}

template <class T, int OP, int TM, int TN, int BK, int S, int WM, int WN>
static hipError_t gemm_tiles(GemmArgs g, int64_t part_floats, hipStream_t stream) {
    constexpr int64_t CUS = 256;
    g.tiles_m = (int)ceil_div(g.M, TM);
    g.tiles_n = (int)ceil_div(g.N, TN);
    const int64_t tiles = (int64_t)g.tiles_m * g.tiles_n, chunks = ceil_div(g.K, BK);
    int64_t splits = tiles < CUS ? CUS / tiles : 1;
    if (splits > chunks / 4) splits = chunks / 4;
    if (splits > part_floats / (g.M * g.N)) splits = part_floats / (g.M * g.N);
    if (splits < 1) splits = 1;
    g.kc = ceil_div(chunks, splits) * BK;
    g.splits = g.K > 0 ? (int)ceil_div(g.K, g.kc) : 1;
    hipLaunchKernelGGL((k_gemm_tile<T, OP, TM, TN, BK, S, WM, WN>), dim3((unsigned)(tiles * g.splits)),
                       dim3(64 * WM * WN), 0, stream, g);
    if (hipError_t e = hipGetLastError()) return e;
    if (g.splits > 1) {
        const int64_t need = ceil_div(g.M * ceil_div(g.N, 8), 256);
        hipLaunchKernelGGL(k_gemm_join<T>, dim3((unsigned)(need < 4096 ? need : 4096)), dim3(256), 0, stream, g);
    }
    return hipGetLastError();
}

template <class T, int OP>
static hipError_t gemm_op(const GemmArgs &g, int64_t part_floats, hipStream_t stream) {
    const int64_t big = ceil_div(g.M, 256) * ceil_div(g.N, 256), mid = ceil_div(g.M, 128) * ceil_div(g.N, 128);
    if constexpr (sizeof(T) == 2) {
        constexpr bool TN = OP == GEMM_TN;
        if (big >= 200) return gemm_tiles<T, OP, 256, 256, TN ? 32 : 64, TN ? 5 : 2, 2, 4>(g, part_floats, stream);
        if constexpr (!TN)
            if (mid >= 400) return gemm_tiles<T, OP, 128, 128, 64, 2, 2, 2>(g, part_floats, stream);
        if (mid >= 32) return gemm_tiles<T, OP, 128, 128, TN ? 32 : 64, 4, 2, TN ? 2 : 4>(g, part_floats, stream);
        return gemm_tiles<T, OP, 64, 64, 64, 4, 2, 2>(g, part_floats, stream);
    } else {
        if (mid >= 400) return gemm_tiles<T, OP, 256, 128, 32, 2, 4, 2>(g, part_floats, stream);
        if (mid >= 32) return gemm_tiles<T, OP, 128, 128, 32, 2, 2, 4>(g, part_floats, stream);
        return gemm_tiles<T, OP, 64, 64, 32, 4, 2, 2>(g, part_floats, stream);
    }
}

template <class T>
static hipError_t gemm_type(int op, const GemmArgs &g, int64_t part_floats, hipStream_t stream) {
    switch (op) {
    case GEMM_NN: return gemm_op<T, GEMM_NN>(g, part_floats, stream);
    case GEMM_NT: return gemm_op<T, GEMM_NT>(g, part_floats, stream);
    default: return gemm_op<T, GEMM_TN>(g, part_floats, stream);
    }
}

hipError_t launch_gemm(int op, int32_t dtype, const Operand &A, const Operand &B, int64_t M, int64_t N,
                       int64_t K, const Epilogue &e, float *part, int64_t part_floats, hipStream_t stream) {
    GemmArgs g{};
    g.A = A;
    g.B = B;
    g.M = M;
    g.N = N;
    g.K = K;
    g.part = part;
    g.e = e;
    switch (dtype) {
    case MLP_F32: return gemm_type<float>(op, g, part_floats, stream);
    case MLP_BF16: return gemm_type<bf16>(op, g, part_floats, stream);
    default: return gemm_type<f16>(op, g, part_floats, stream);
    }
}

}  // namespace mlp
