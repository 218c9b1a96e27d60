// linear_gemm.hip -- the dense layer's matrix products of bf16 and fp16 operands on the
// matrix cores (gfx950), and what joins the splits of a product's depth.
//
// A workgroup computes a TM x TN tile of C; its K loop runs over chunks of BK staged in
// LDS, in two to five stages: a chunk's loads go straight to LDS while the chunks before
// it are on the matrix cores, one barrier a chunk. The products are v_mfma_f32_32x32x16 with
// B as the first operand, so that four of a lane's results in a row lie along a row of C.
// The pieces of an LDS row are permuted (linear_tile.h) by way of the addresses they are
// loaded from.
//
// What bounds the larger tiles: a compute unit takes in 38 bytes a nanosecond from L2 (its
// lines in flight over their latency; 64 KB a chunk of 64 k of a 256 x 256 tile), and the
// matrix cores' power (8,192 x 8,192 x 8,192 in bf16: 1.25 PFLOP/s of Gaussian values, 1.47
// of zeros). Chunks of 64 k where k is contiguous, so that rows are whole lines of L2.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "linear_tile.h"

namespace mlp {

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

// One operand's chunks: TX values of x by BK of k, moved by NT threads.
template <bool XC, int TX, int BK, int NT>
struct Tile : LdsTile<XC, TX, BK> {
    using L = LdsTile<XC, TX, BK>;
    using L::ROW;
    using L::swz;
    static constexpr int PIECES = TX * BK / 8;            // of 16 bytes
    static constexpr int LOADS = PIECES / NT;
    static constexpr int ELEMS = TX * BK;
    static_assert(PIECES % NT == 0, "every thread moves the same number of pieces");

    const char *base;        // the current chunk's corner, uniform
    uint32_t off[LOADS];     // bytes from it
    int64_t step;            // bytes to the next chunk

    __device__ __forceinline__ void init(const Operand &o, int64_t x0, int64_t xlim, int64_t k0) {
        base = (const char *)((const uint16_t *)o.p + (XC ? k0 * o.ld + x0 : x0 * o.ld + k0));
        step = 2 * (XC ? BK * o.ld : (int64_t)BK);
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
    // one of the LOADS loads of the chunk at base to the LDS tile S; TAIL: only k < left is
    // there, zeros take the place of the rest
    template <bool TAIL>
    __device__ __forceinline__ void load(uint16_t *S, int i, int left) const {
        uint16_t *d = S + 8 * (i * NT + (threadIdx.x & ~63u));
        const char *g = base + off[i];
        if constexpr (TAIL) {
            const int q = i * NT + threadIdx.x, row = q / (ROW / 8);
            const int k = XC ? row : 8 * ((q % (ROW / 8)) ^ swz(row));
            if (k >= left) g = (const char *)g_zeros;
        }
        to_lds(g, d);
    }
};

// Loads [n0, n1) of a chunk of both operands (the A tile's, then the B tile's).
template <bool TAIL, int N0, int N1, class TA, class TB>
__device__ __forceinline__ void load_some(const TA &a, const TB &b, uint16_t *An, uint16_t *Bn, int left) {
    constexpr int NA = TA::LOADS;
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
template <int NJ, int MI>
struct Frags {
    u4v a[MI], b[NJ];
    template <class TA, class TB>
    __device__ __forceinline__ void fetch(const uint16_t *A, const uint16_t *B, int wm, int wn, int kk) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) b[j] = TB::frag(B, wn + 32 * j, kk);
#pragma unroll
        for (int i = 0; i < MI; ++i) a[i] = TA::frag(A, wm + 32 * i, kk);
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
template <bool TAIL, bool AHEAD, class T, int NJ, int MI, class TA, class TB>
__device__ __forceinline__ void chunk_step(const TA &a, const TB &b, f16v (&acc)[NJ][MI],
                                           Frags<NJ, MI> (&f)[2], uint16_t *__restrict__ An,
                                           uint16_t *__restrict__ Bn, const uint16_t *__restrict__ Ac,
                                           const uint16_t *__restrict__ Bc, const uint16_t *__restrict__ Af,
                                           const uint16_t *__restrict__ Bf, int left, int wm, int wn) {
    constexpr int KK = TA::K / 16, SLOTS = AHEAD ? KK * NJ : (3 * KK * NJ + 7) / 8;
    constexpr int ALL = TA::LOADS + TB::LOADS;
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
#pragma unroll
            for (int i = 0; i < MI; ++i) acc[j][i] = mma<T>(f[kk & 1].b[j], f[kk & 1].a[i], acc[j][i]);
#pragma unroll
            for (int n = 0; n < MI; ++n) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
            }
        });
        __builtin_amdgcn_sched_barrier(0);
    });
}

// TM x TN outputs, WM x WN waves, each TM / WM x TN / WN outputs as 32 x 32 MFMA tiles. T: the
// type of C. S: LDS stages, each a chunk of both operands. FOLD: fewer than eight columns,
// B's rows hold two values of each, eight apart.
template <class T, int OP, int TM, int TN, int BK, int S, int WM, int WN, bool FOLD>
__global__ __launch_bounds__(64 * WM * WN) void k_gemm_tile(const GemmArgs g) {
    constexpr int NT = 64 * WM * WN, MI = TM / WM / 32, NJ = TN / WN / 32;
    typedef Tile<OP == GEMM_TN, TM, BK, NT> TA;
    typedef Tile<OP != GEMM_NT, TN, BK, NT> TB;
    constexpr int STAGE = TA::ELEMS + TB::ELEMS;
    static_assert(WM * WN * 32 * RESULT_STRIDE<NJ> * 4 <= 2 * S * STAGE, "the results fit where the chunks were");
    __shared__ __attribute__((aligned(16))) uint16_t lds[S * STAGE];
    const int wave = threadIdx.x >> 6;
    const int wm = wave / WN * (TM / WM), wn = wave % WN * (TN / WN);
    const TileAt at(g, TM, TN);
    const int nk = (int)((at.ke - at.kb + BK - 1) / BK);
    f16v acc[NJ][MI];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[j][i][v] = 0.f;

    if (nk > 0) {
        TA a;
        TB b;
        a.init(g.A, at.m0, g.M, at.kb);
        b.init(g.B, at.n0, FOLD ? 16 : g.N, at.kb);
        // S - 1 chunks are on their way before the first is used. At chunk c's barrier
        // every wave has loaded chunks c and c + 1 and read all of chunk c - 1, whose
        // stage chunk c + S - 1 takes. (Past the last chunk zeros are loaded, so that the
        // waits stay the same.)
        constexpr bool AHEAD = S > 2;
        constexpr int PER = TA::LOADS + TB::LOADS;
        int64_t left = at.ke - at.kb;   // k from the chunk to be loaded next to the end
        Frags<NJ, MI> f[2];
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
            chunk_step<decltype(tail)::value, AHEAD, T>(a, b, acc, f, lds + last, lds + last + TA::ELEMS, lds + now,
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
        loaded_all_but<0>();   // no load to LDS is under way when the results take its place
    }

    finish_tile<T, FOLD>(g, at, wm, wn, acc, reinterpret_cast<float *>(lds));
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
        auto add = [&](const Oct<float> &w) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += w.e[j];
        };
        const float *p = g.part + m * g.N;
        int s = 1;
        // sixteen loads under way at a time: few outputs have many splits (dW of 65,536 x 64 x
        // 64 in bf16 35 us in all, 40 with four)
        for (; s + 16 <= g.splits; s += 16) {
            Oct<float> w[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) w[q] = fetch8(p + (s + q) * g.M * g.N, n, g.N);
#pragma unroll
            for (int q = 0; q < 16; ++q) add(w[q]);
        }
#pragma unroll 4
        for (; s < g.splits; ++s) add(fetch8(p + s * g.M * g.N, n, g.N));
        fin.finish(g.e, m, n, g.N, v, res);
    }
}

template <class T>
hipError_t join_splits(const GemmArgs &g, hipStream_t stream) {
    if (g.splits <= 1) return hipSuccess;
    const int64_t need = ceil_div(g.M * ceil_div(g.N, 8), 256);
    hipLaunchKernelGGL(k_gemm_join<T>, dim3((unsigned)(need < 4096 ? need : 4096)), dim3(256), 0, stream, g);
    return hipGetLastError();
}
template hipError_t join_splits<float>(const GemmArgs &, hipStream_t);

template <class T, int OP, int TM, int TN, int BK, int S, int WM, int WN, bool FOLD = false>
static hipError_t gemm_tiles(GemmArgs g, int64_t part_floats, hipStream_t stream) {
    // (a chunk of 64 takes 0.28 us on 64 x 64 tiles, 0.5 on 128 x 128, 1 and more on 256 x 256)
    constexpr int WORTH = (TM == 64 ? 1024 : TM == 128 ? 576 : 256) / BK;
    const unsigned grid = plan_tiles(g, TM, TN, BK, CUS, WORTH, part_floats);
    hipLaunchKernelGGL((k_gemm_tile<T, OP, TM, TN, BK, S, WM, WN, FOLD>), dim3(grid), dim3(64 * WM * WN), 0, stream, g);
    if (hipError_t e = hipGetLastError()) return e;
    return join_splits<T>(g, stream);
}

// The tile by the number of tiles (us in bf16, of outputs x depth):
// 256 x 256 where there are more than half as many as compute units, which run one each, and
// they cover at most 5/4 of what 128 x 128 would (3,328 x 3,328 x 1,024 33, on 128 x 128 38; 2,816 x
// 2,816 x 1,024, split in two, 49 and 24; 131,072 x 128 x 256 37 and 25);
// 128 x 128 of two stages, two workgroups a compute unit, where there are more than units
// (2,304 x 2,304 x 2,048 34, of four stages 40; 2,048 x 2,048 x 2,048 34 and 24; TN's stages
// are half as deep, and two workgroups run with four of them);
// 128 x 128 of four stages where no split is needed (1,536 x 1,536 x 1,536 18, on 64 x 64 22),
// or the depth pays for the splits' joining (1,024 x 1,024 x 16,384 58 and 76, of 1,024 23 and
// 8.6; TN, whose 64 x 64 tiles are slower, of 4,096 27 and 36, of 2,048 22 and 14).
template <class T, int OP, bool FOLD = false>
static hipError_t gemm_op(const GemmArgs &g, int64_t part_floats, hipStream_t stream) {
    constexpr bool TN = OP == GEMM_TN;
    const int64_t big = ceil_div(g.M, 256) * ceil_div(g.N, 256), mid = ceil_div(g.M, 128) * ceil_div(g.N, 128);
    if constexpr (!FOLD)   // (a column of tiles never covers so little)
        if (big > CUS / 2 && 16 * big <= 5 * mid)
            return gemm_tiles<T, OP, 256, 256, TN ? 32 : 64, TN ? 5 : 2, 2, 4>(g, part_floats, stream);
    if constexpr (!TN)
        if (mid > CUS) return gemm_tiles<T, OP, 128, 128, 64, 2, 2, 2>(g, part_floats, stream);
    if (mid > CUS / 2 || (mid >= 16 && g.K > (TN ? 2048 : 4096)))
        return gemm_tiles<T, OP, 128, 128, TN ? 32 : 64, 4, 2, TN ? 2 : 4, FOLD>(g, part_floats, stream);
    return gemm_tiles<T, OP, 64, 64, 64, 4, 2, 2, FOLD>(g, part_floats, stream);
}

template <class T>
static hipError_t gemm_type(int op, const GemmArgs &g, int64_t part_floats, hipStream_t stream) {
    switch (op) {
    case GEMM_NN: return gemm_op<T, GEMM_NN>(g, part_floats, stream);
    case GEMM_NT: return gemm_op<T, GEMM_NT>(g, part_floats, stream);
    default: return gemm_op<T, GEMM_TN>(g, part_floats, stream);
    }
}

hipError_t launch_gemm_fold(int32_t dtype, const Operand &A, const Operand &B, int64_t M, int64_t N, int64_t K,
                            const Epilogue &e, float *part, int64_t part_floats, hipStream_t stream) {
    GemmArgs g{};
    g.A = A;
    g.B = B;
    g.M = M;
    g.N = N;
    g.K = K;
    g.part = part;
    g.e = e;
    if (dtype == MLP_BF16) return gemm_op<bf16, GEMM_TN, true>(g, part_floats, stream);
    return gemm_op<f16, GEMM_TN, true>(g, part_floats, stream);
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
    case MLP_F32: return launch_gemm_f32(op, g, part_floats, stream);
    case MLP_BF16: return gemm_type<bf16>(op, g, part_floats, stream);
    default: return gemm_type<f16>(op, g, part_floats, stream);
    }
}

}  // namespace mlp
