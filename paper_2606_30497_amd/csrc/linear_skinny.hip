// linear_skinny.hip -- the dense layer's matrix products that are bound by W or by latency:
// of few rows (single tokens, small batches), and small ones in fp32.
//
// k_skinny, y = x W and dX = g W^T: W goes from memory straight to the registers of the
// matrix cores, 128 outputs and 32 (fp32: 16) of the depth a wave and step, two steps
// ahead, at any alignment; a workgroup takes 16 or 32 rows, and nothing is shared, so LDS
// has no part in it. The waves of a workgroup and `splits` workgroups share the depth; a
// workgroup adds its waves' sums in LDS, and the last of the splits to arrive adds theirs,
// in order, and finishes the rows. The products are v_mfma_f32_16x16x32 of 16-bit values,
// v_mfma_f32_16x16x4f32 of fp32 ones (plain fp32 products), W as the first operand: its row
// r of product t is output 8 r + t, so that a lane's results of the eight products are
// eight columns in a row. Where W's rows lie along the outputs, a lane loads eight
// outputs of eight (fp32: four) k and the pairs of k are put together by v_perm.
//
// k_outer, dW = X^T g of few rows: the same products with X read across its rows; a wave
// takes 16 x 128 values of dW, bound by writing them.
//
// k_narrow, y = x W of fewer than eight outputs and a deep row: no matrix instruction, whose
// columns would be idle; bound by reading X.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <type_traits>

#include "linear_internal.h"

namespace mlp {

typedef _Float16 h8v __attribute__((ext_vector_type(8)));

constexpr int SKINNY_N = 128;   // outputs of a workgroup

struct SkinnyArgs {
    const void *X, *W;
    int64_t low;           // LOW: elements from X to what its rounding left (the same ld)
    int64_t ldx, ldw, M, N, K;
    int splits;
    int64_t kw;            // depth of a wave (a multiple of the step)
    float *part;           // [splits][M][N rounded up to SKINNY_N]
    uint32_t *arrived;     // [row tiles][output tiles], zero between calls
    Epilogue e;
};

template <class T>
__device__ __forceinline__ f4 mma16(u4v a, u4v b, f4 c) {
    if constexpr (std::is_same<T, bf16>::value) return mfma_bf16(a, b, c);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8v, a), __builtin_bit_cast(h8v, b), c, 0, 0, 0);
}

// 16 bytes at any element's address
template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Piece {
    uint32_t w[4];
    __device__ __forceinline__ u4v get() const { return u4v{w[0], w[1], w[2], w[3]}; }
};

// One step of a wave's depth: W for 128 outputs, X for 16 MT rows.
// 16-bit: w[i] = outputs 8 r .. + 7 of k 8 g + i (OUT: W's rows lie along the outputs), or k
// 8 g .. + 7 of output 8 r + i. fp32: w[2 s + h] = outputs 8 r + 4 h .. + 3 of k 4 g + s, or
// w[i] = k 4 g .. + 3 of output 8 r + i. (Lane l: r = l % 16, g = l / 16.)
// LOW: X comes as two values of the type, the second what the first one's rounding left.
template <class T, bool OUT, int MT, bool LOW = false>
struct Step {
    static constexpr int PER = 16 / sizeof(T), K = 4 * PER;   // elements of a piece, depth
    u4v w[8], x[MT], y[LOW ? MT : 1];   // y: X's second values

    static __device__ __forceinline__ u4v piece(const char *p, uint32_t off) {
        return reinterpret_cast<const Piece<T> *>(p + off)->get();
    }
    // elements [at, at + PER) of a row of `len` >= PER, its first at row + off, those past
    // its end 0: its last PER elements moved down, so that one load at a valid address does
    static __device__ __forceinline__ u4v end_piece(const char *row, uint32_t off, int at, int len) {
        const int from = at < len - PER ? at : len - PER, d = (at - from < PER ? at - from : PER) * (int)sizeof(T);
        u4v v = piece(row, off + (uint32_t)(from * (int)sizeof(T)));
        if (sizeof(T) == 2) {   // by bytes: 2, 4, 8, 16
            const uint32_t up[4] = {v[1], v[2], v[3], 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = d & 2 ? __builtin_amdgcn_alignbit(up[i], v[i], 16) : v[i];
        }
        v = d & 4 ? u4v{v[1], v[2], v[3], 0} : v;
        v = d & 8 ? u4v{v[2], v[3], 0, 0} : v;
        return d & 16 ? u4v{0, 0, 0, 0} : v;
    }
    // The step at depth k0 (uniform) of the outputs from n0 on. EDGE: the tile reaches past
    // the outputs (what is computed of those is not used); TAIL: the step reaches past the
    // depth, where W and X count as 0.
    template <bool EDGE, bool TAIL>
    __device__ __forceinline__ void load(const void *W, int64_t ld, int64_t N, int64_t depth_all, int64_t n0, int64_t k0) {
        const int l = threadIdx.x & 63, r = l & 15, g = l >> 4;
        const uint32_t ES = sizeof(T), ldw = (uint32_t)ld * ES;
        const int kl = (int)(depth_all - k0 < K ? depth_all - k0 : K);   // depth of the step
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (OUT) {
                const int kd = sizeof(T) == 2 ? i : i / 2, k = PER * g + kd;
                const int n = 8 * r + (sizeof(T) == 2 ? 0 : 4 * (i & 1));
                const char *row = (const char *)W + k0 * ld * ES;
                uint32_t off = (uint32_t)(PER * g) * ldw;
                if constexpr (TAIL) off = (uint32_t)(k < kl ? k : kl - 1) * ldw;
                else row += kd * (int64_t)ldw;
                if constexpr (EDGE) w[i] = end_piece(row, off, (int)n0 + n, (int)N);
                else w[i] = piece(row + n0 * ES, off + n * ES);
                if (TAIL && k >= kl) w[i] = u4v{0, 0, 0, 0};
            } else {
                const char *row = (const char *)W + n0 * ld * ES;
                uint32_t off = (uint32_t)(8 * r) * ldw;
                if constexpr (EDGE) off = (uint32_t)(n0 + 8 * r + i < N ? 8 * r + i : (int)(N - n0) - 1) * ldw;
                else row += i * (int64_t)ldw;
                if constexpr (TAIL) w[i] = end_piece(row, off, (int)k0 + PER * g, (int)depth_all);
                else w[i] = piece(row + k0 * ES, off + PER * g * ES);
            }
        }
    }
    // X's rows at xp (one for each 16 rows), k contiguous
    template <bool TAIL>
    __device__ __forceinline__ void load_x(const char *const (&xp)[MT], int64_t low, int64_t depth_all, int64_t k0) {
        const int g = (threadIdx.x & 63) >> 4;
        auto get = [&](const char *p) __attribute__((always_inline)) {
            if constexpr (TAIL) return end_piece(p, 0, (int)k0 + PER * g, (int)depth_all);
            else return piece(p + k0 * (int64_t)sizeof(T), PER * g * (uint32_t)sizeof(T));
        };
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            x[t] = get(xp[t]);
            if constexpr (LOW) y[t] = get(xp[t] + low * (int64_t)sizeof(T));
        }
    }
    // X's columns at xp, k down them, `pitch` bytes apart
    template <bool TAIL>
    __device__ __forceinline__ void load_across(const char *const (&xp)[MT], int64_t pitch, int64_t depth_all,
                                                int64_t k0) {
        const int g = (threadIdx.x & 63) >> 4, kl = (int)(depth_all - k0 < K ? depth_all - k0 : K);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            union {
                T e[PER];
                u4v v;
            } o;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int k = PER * g + j;
                const T e = *reinterpret_cast<const T *>(xp[t] + (k0 + (TAIL && k >= kl ? kl - 1 : k)) * pitch);
                o.e[j] = TAIL && k >= kl ? (T)0.0f : e;
            }
            x[t] = o.v;
        }
    }
    __device__ __forceinline__ void multiply(f4 (&acc)[MT][8]) const {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            if constexpr (sizeof(T) == 2) {
                u4v f = w[t];
                if constexpr (OUT) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        f[q] = __builtin_amdgcn_perm(w[2 * q + 1][t >> 1], w[2 * q][t >> 1], t & 1 ? 0x07060302 : 0x05040100);
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    if constexpr (LOW) acc[m][t] = mma16<T>(f, y[m], acc[m][t]);
                    acc[m][t] = mma16<T>(f, x[m], acc[m][t]);
                }
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const float f = __uint_as_float(OUT ? w[2 * s + (t >> 2)][t & 3] : w[t][s]);
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(f, __uint_as_float(x[m][s]), acc[m][t], 0, 0, 0);
                }
            }
        }
    }
};

template <class T, bool OUT, int MT, bool LOW, bool EDGE>
__device__ __forceinline__ void skinny_sums(const SkinnyArgs &a, int64_t m0, int64_t n0, int64_t kb, f4 (&acc)[MT][8]) {
    typedef Step<T, OUT, MT, LOW> S;
    const int64_t ke = kb + a.kw < a.K ? kb + a.kw : a.K;
    const int full = ke > kb ? (int)((ke - kb) / S::K) : 0;
    const char *xp[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int64_t m = m0 + 16 * t + (threadIdx.x & 15);
        xp[t] = (const char *)a.X + (m < a.M ? m : a.M - 1) * a.ldx * (int64_t)sizeof(T);
    }
    auto load = [&](S &s, int i) __attribute__((always_inline)) {
        const int64_t k0 = kb + i * (int64_t)S::K;
        s.template load<EDGE, false>(a.W, a.ldw, a.N, a.K, n0, k0);
        s.template load_x<false>(xp, a.low, a.K, k0);
    };
    {
        S s[2];
        if (full > 0) load(s[0], 0);
        if (full > 1) load(s[1], 1);
        int i = 0;
        for (; i + 2 <= full; i += 2) {
            s[0].multiply(acc);
            if (i + 2 < full) load(s[0], i + 2);
            s[1].multiply(acc);
            if (i + 3 < full) load(s[1], i + 3);
        }
        if (i < full) s[0].multiply(acc);
    }
    if (kb + (int64_t)full * S::K < ke) {
        S s;
        s.template load<EDGE, true>(a.W, a.ldw, a.N, a.K, n0, kb + (int64_t)full * S::K);
        s.template load_x<true>(xp, a.low, a.K, kb + (int64_t)full * S::K);
        s.multiply(acc);
    }
}

template <class T, bool OUT, int MT, bool LOW>
__global__ __launch_bounds__(512, 2) void k_skinny(const SkinnyArgs a) {
    constexpr int WAVES = 8, NT = 512, CS = SKINNY_N + 4;
    __shared__ __attribute__((aligned(16))) float sums[WAVES][16 * MT][CS];
    __shared__ uint32_t before;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
    const int64_t n0 = (int64_t)tile * SKINNY_N, m0 = (int64_t)blockIdx.y * (16 * MT);
    const int rows = (int)(a.M - m0 < 16 * MT ? a.M - m0 : 16 * MT);
    const int64_t kb = ((int64_t)split * WAVES + wave) * a.kw;
    f4 acc[MT][8];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < 8; ++t) acc[m][t] = f4{0.f, 0.f, 0.f, 0.f};
    if (n0 + SKINNY_N <= a.N) skinny_sums<T, OUT, MT, LOW, false>(a, m0, n0, kb, acc);
    else skinny_sums<T, OUT, MT, LOW, true>(a, m0, n0, kb, acc);

    // register v of product t: row l % 16, column 8 (4 (l / 16) + v) + t
#pragma unroll
    for (int m = 0; m < MT; ++m)
        if (16 * m + (lane & 15) < rows) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f4 w{acc[m][4 * h][v], acc[m][4 * h + 1][v], acc[m][4 * h + 2][v], acc[m][4 * h + 3][v]};
                    *reinterpret_cast<f4 *>(&sums[wave][16 * m + (lane & 15)][8 * (4 * (lane >> 4) + v) + 4 * h]) = w;
                }
        }
    __syncthreads();
    const int64_t pitch = (a.N + SKINNY_N - 1) / SKINNY_N * SKINNY_N;
    if (a.splits > 1) {
        for (int i = threadIdx.x; i < rows * SKINNY_N; i += NT) {
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) s += sums[w][i / SKINNY_N][i % SKINNY_N];
            __hip_atomic_store(a.part + ((int64_t)split * a.M + m0 + i / SKINNY_N) * pitch + n0 + i % SKINNY_N, s,
                               __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        // The sums are stored and read device-coherently, past the XCDs' own L2s, so their
        // completion before the arrival is counted is all the order they need (a release
        // at device scope would write back the whole L2: 45 us a call of 1 x 4,096 x 4,096
        // with it, 8 without).
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        uint32_t *arrived = a.arrived + (int64_t)blockIdx.y * (pitch / SKINNY_N) + tile;
        if (threadIdx.x == 0)
            before = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (before != (uint32_t)a.splits - 1) return;
        if (threadIdx.x == 0) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    for (int i = threadIdx.x; i < rows * (SKINNY_N / 8); i += NT) {
        const int r = i / (SKINNY_N / 8), c = i % (SKINNY_N / 8) * 8;
        const int64_t n = n0 + c, m = m0 + r;
        if (n >= a.N) continue;
        Finish<T> fin;
        fin.init(a.e, n, a.N);
        Oct<T> res;
        if (a.e.R) res = fetch8((const T *)a.e.R + m * a.e.ldr, n, a.N);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        if (a.splits > 1) {
#pragma unroll 4
            for (int s = 0; s < a.splits; ++s) {
                const uint64_t *p = reinterpret_cast<const uint64_t *>(a.part + ((int64_t)s * a.M + m) * pitch + n);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint64_t w = __hip_atomic_load(p + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    v[2 * j] += __uint_as_float((uint32_t)w);
                    v[2 * j + 1] += __uint_as_float((uint32_t)(w >> 32));
                }
            }
        } else {
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += sums[w][r][c + j];
        }
        fin.finish(a.e, m, n, a.N, v, res);
    }
}

template <class T, bool OUT, int MT, bool LOW>
static hipError_t skinny(SkinnyArgs a, int64_t part_floats, int64_t arrived_words, hipStream_t stream) {
    constexpr int64_t STEP = Step<T, OUT, MT>::K;
    const int64_t tiles = ceil_div(a.N, SKINNY_N), row_tiles = ceil_div(a.M, 16 * MT), pitch = tiles * SKINNY_N;
    // A workgroup for each compute unit, of at least two steps a wave (one, where the
    // workgroups are fewer all the same). (With 512 of them
    // half wait for the other half, whose eight waves' registers fill the unit: fp32 1 x
    // 4,096 x 4,096 16 us with 256, 22 with 512, 20 with 128.)
    const int64_t most = ceil_div(a.K, STEP * 8);
    int64_t splits = tiles * row_tiles * most <= 256 ? most : ceil_div(a.K, 2 * STEP * 8);
    if (splits > 256 / (tiles * row_tiles)) splits = 256 / (tiles * row_tiles);
    if (splits > part_floats / (a.M * pitch)) splits = part_floats / (a.M * pitch);
    if (splits < 1 || tiles * row_tiles > arrived_words) splits = 1;
    a.kw = ceil_div(ceil_div(a.K, splits * 8), STEP) * STEP;
    a.splits = (int)ceil_div(a.K, a.kw * 8);
    hipLaunchKernelGGL((k_skinny<T, OUT, MT, LOW>), dim3((unsigned)(tiles * a.splits), (unsigned)row_tiles), dim3(512), 0,
                       stream, a);
    return hipGetLastError();
}

template <class T, bool OUT, bool LOW = false>
static hipError_t skinny_rows(const SkinnyArgs &a, int64_t part_floats, int64_t arrived_words, hipStream_t stream) {
    // 16 rows a workgroup, and W read again for every 16, from the caches, but 32 where W has
    // too many elements for that or the workgroups are more than enough. y of 24 rows, W from
    // memory, us with 16 rows and with 32, d_in x d_out, bf16: 8,192 x 1,024 14.4 and 23.6,
    // 8,192 x 2,048 15.1 and 19.0, 8,192 x 4,096 20.5 and 22.4, 8,192 x 5,120 25.6 and 23.4, 8,192 x
    // 8,192 33 and 31; fp32: 8,192 x 2,048 25 and 28, 8,192 x 4,096 40 and 42, 8,192 x 6,144 74 and
    // 59. Where W's rows do not start at 16 bytes from half as many on (bf16: 8,191 x 2,050 19.1
    // and 20.0, 6,143 x 4,098 24.3 and 22.2, 8,191 x 6,145 61 and 38), and for dX from a quarter
    // (bf16: 8,192 x 1,024 10.7 and 10.6, 8,192 x 2,048 15.7 and 15.1, 8,192 x 4,096 28 and 25;
    // fp32: 8,192 x 1,024 17.7 and 17.1, 8,192 x 2,048 30 and 28, 6,144 x 4,096 46 and 36).
    const bool whole = OUT && ((uintptr_t)a.W & 15u) == 0 && a.ldw * (int64_t)sizeof(T) % 16 == 0;
    if (a.M <= 16 || (a.N * a.K <= (whole ? 1 << 25 : OUT ? 1 << 24 : 1 << 23) &&
                      ceil_div(a.M, 16) * ceil_div(a.N, SKINNY_N) <= 256))
        return skinny<T, OUT, 1, LOW>(a, part_floats, arrived_words, stream);
    return skinny<T, OUT, 2, LOW>(a, part_floats, arrived_words, stream);
}

template <class T>
static hipError_t skinny_type(int op, const SkinnyArgs &a, int64_t part_floats, int64_t arrived_words,
                              hipStream_t stream) {
    if (op == GEMM_NN) return skinny_rows<T, true>(a, part_floats, arrived_words, stream);
    if constexpr (sizeof(T) == 2)
        if (a.low) return skinny_rows<T, false, true>(a, part_floats, arrived_words, stream);
    return skinny_rows<T, false>(a, part_floats, arrived_words, stream);
}

hipError_t launch_skinny(int op, int32_t dtype, const void *X, int64_t ldx, int64_t low, const void *W,
                         int64_t ldw, int64_t M, int64_t N, int64_t K, const Epilogue &e, float *part,
                         int64_t part_floats, uint32_t *arrived, int64_t arrived_words, hipStream_t stream) {
    const SkinnyArgs a{X, W, low, ldx, ldw, M, N, K, 1, 0, part, arrived, e};
    switch (dtype) {
    case MLP_F32: return skinny_type<float>(op, a, part_floats, arrived_words, stream);
    case MLP_BF16: return skinny_type<bf16>(op, a, part_floats, arrived_words, stream);
    default: return skinny_type<f16>(op, a, part_floats, arrived_words, stream);
    }
}

// Element v of lane group g (of 16 lanes) and element g of group v change places.
__device__ __forceinline__ void trade(f4 &x) {
    uint32_t w[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) w[v] = __float_as_uint(x[v]);
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const auto p = __builtin_amdgcn_permlane32_swap(w[v], w[v + 2], false, false);
        w[v] = p[0];
        w[v + 2] = p[1];
    }
#pragma unroll
    for (int v = 0; v < 4; v += 2) {
        const auto p = __builtin_amdgcn_permlane16_swap(w[v], w[v + 1], false, false);
        w[v] = p[0];
        w[v + 1] = p[1];
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) x[v] = __uint_as_float(w[v]);
}

struct OuterArgs {
    const void *X, *G;
    void *dW;
    int64_t low;   // LOW: elements from G to what its rounding left
    int64_t ldx, ldg, M, K, N;
    int tiles;     // tiles of 16 k a wave
    float scale;   // of the sums
};

template <class T, bool LOW, bool EDGE>
__device__ __forceinline__ void outer(const OuterArgs &a, int64_t k0, int64_t n0) {
    typedef Step<T, true, 1> S;
    const int lane = threadIdx.x & 63;
    const int64_t pitch = a.ldx * (int64_t)sizeof(T);
    const T *low = (const T *)a.G + a.low;
    const bool once = a.M <= S::K;   // G's rows stay in the registers for all tiles
    S s, y;                          // y: the second values of G
    if (once && a.M > 0) {
        s.template load<EDGE, true>(a.G, a.ldg, a.N, a.M, n0, 0);
        if constexpr (LOW) y.template load<EDGE, true>(low, a.ldg, a.N, a.M, n0, 0);
    }
#pragma unroll 1
    for (int i = 0; i < a.tiles && k0 < a.K; ++i, k0 += 16) {
        const int64_t k = k0 + (lane & 15);
        const char *xp[1] = {(const char *)a.X + (k < a.K ? k : a.K - 1) * (int64_t)sizeof(T)};
        f4 acc[1][8];
#pragma unroll
        for (int t = 0; t < 8; ++t) acc[0][t] = f4{0.f, 0.f, 0.f, 0.f};
        auto product = [&](auto tail, int64_t m) __attribute__((always_inline)) {
            constexpr bool TAIL = decltype(tail)::value;
            s.template load_across<TAIL>(xp, pitch, a.M, m);
            if constexpr (LOW) {
                if (!once) y.template load<EDGE, TAIL>(low, a.ldg, a.N, a.M, n0, m);
                y.x[0] = s.x[0];
                y.multiply(acc);
            }
            if (!once) s.template load<EDGE, TAIL>(a.G, a.ldg, a.N, a.M, n0, m);
            s.multiply(acc);
        };
        int64_t m = 0;
        if (!once)
            for (; m + S::K <= a.M; m += S::K) product(std::false_type(), m);
        if (m < a.M) product(std::true_type(), m);
        // Register v of lane group g is piece 4 g + v of the row: traded among the four
        // groups, piece 4 v + g, so that a store's four lanes of a row write side by side.
#pragma unroll
        for (int t = 0; t < 8; ++t) trade(acc[0][t]);
        if (k < a.K) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int64_t n = n0 + 8 * (4 * v + (lane >> 4));
                float w[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) w[t] = acc[0][t][v] * a.scale;
                if (n < a.N) store8((T *)a.dW + k * a.N, n, a.N, w);
            }
        }
    }
}

template <class T, bool LOW>
__global__ __launch_bounds__(256) void k_outer(const OuterArgs a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * SKINNY_N, k0 = ((int64_t)blockIdx.y * 4 + wave) * (16 * a.tiles);
    if (n0 + SKINNY_N <= a.N) outer<T, LOW, false>(a, k0, n0);
    else outer<T, LOW, true>(a, k0, n0);
}

hipError_t launch_outer(int32_t dtype, const void *X, int64_t ldx, const void *G, int64_t ldg, int64_t low,
                        int64_t M, int64_t K, int64_t N, float scale, void *dW, hipStream_t stream) {
    // about 1,024 workgroups of four waves
    const int64_t across = ceil_div(N, SKINNY_N), tiles = ceil_div(ceil_div(K, 64) * across, 1024);
    const OuterArgs a{X, G, dW, low, ldx, ldg, M, K, N, (int)(tiles < 16 ? tiles : 16), scale};
    const dim3 grid((unsigned)across, (unsigned)ceil_div(K, 64 * a.tiles));
#define OUTER(T, LOW) hipLaunchKernelGGL((k_outer<T, LOW>), grid, dim3(256), 0, stream, a)
    switch (dtype) {
    case MLP_F32: OUTER(float, false); break;
    case MLP_BF16:
        if (low) OUTER(bf16, true);
        else OUTER(bf16, false);
        break;
    default:
        if (low) OUTER(f16, true);
        else OUTER(f16, false);
        break;
    }
#undef OUTER
    return hipGetLastError();
}

// N outputs of eight rows: a workgroup's lanes share the depth, eight k a lane and step (W's
// 8 N values of those are contiguous), fp32 sums joined over the lanes and, in LDS, the waves.
template <class T, int N>
__global__ __launch_bounds__(512) void k_narrow(const T *X, int64_t ldx, const T *W, int64_t M, int64_t K, const Epilogue e) {
    constexpr int R = 8, WAVES = 8;
    __shared__ float sums[WAVES][R][N];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m0 = (int64_t)blockIdx.x * R;
    float acc[R][N];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[r][j] = 0.0f;
    for (int64_t k = 8 * (int64_t)threadIdx.x; k < K; k += 8 * 512) {
        Oct<T> x[R], w[N];
#pragma unroll
        for (int r = 0; r < R; ++r) x[r] = fetch8(X + (m0 + r < M ? m0 + r : M - 1) * ldx, k, K);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = fetch8(W, k * N + 8 * i, K * N);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float f = up(w[(i * N + j) / 8].e[(i * N + j) % 8]);
#pragma unroll
                for (int r = 0; r < R; ++r) acc[r][j] = fmaf(up(x[r].e[i]), f, acc[r][j]);
            }
    }
    // over the lanes: half of them take half of the rows, and so on (10 N exchanges)
#pragma unroll
    for (int h = 4, s = 32; h > 0; h >>= 1, s >>= 1)
#pragma unroll
        for (int r = 0; r < h; ++r)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float lo = acc[r][j], hi = acc[r + h][j];
                acc[r][j] = (lane & s ? hi : lo) + __shfl_xor(lane & s ? lo : hi, s);
            }
#pragma unroll
    for (int j = 0; j < N; ++j) {
#pragma unroll
        for (int s = 4; s > 0; s >>= 1) acc[0][j] += __shfl_xor(acc[0][j], s);
        if ((lane & 7) == 0) sums[wave][(lane >> 3 & 1) + 2 * (lane >> 4 & 1) + 4 * (lane >> 5)][j] = acc[0][j];
    }
    __syncthreads();
    const int r = threadIdx.x;
    if (r >= R || m0 + r >= M) return;
    float v[8] = {};
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v[j] += sums[w][r][j];
    Finish<T> fin;
    fin.init(e, 0, N);
    Oct<T> res;
    if (e.R) res = fetch8((const T *)e.R + (m0 + r) * e.ldr, 0, N);
    fin.finish(e, m0 + r, 0, N, v, res);
}

template <class T>
static hipError_t narrow_type(const void *X, int64_t ldx, const void *W, int64_t M, int64_t N, int64_t K,
                              const Epilogue &e, hipStream_t stream) {
    const dim3 grid((unsigned)ceil_div(M, 8));
#define NARROW(n) \
    case n: hipLaunchKernelGGL((k_narrow<T, n>), grid, dim3(512), 0, stream, (const T *)X, ldx, (const T *)W, M, K, e); break
    switch (N) {
        NARROW(1);
        NARROW(2);
        NARROW(3);
        NARROW(4);
        NARROW(5);
        NARROW(6);
        NARROW(7);
    default: return hipErrorInvalidValue;
    }
#undef NARROW
    return hipGetLastError();
}

hipError_t launch_narrow(int32_t dtype, const void *X, int64_t ldx, const void *W, int64_t M, int64_t N, int64_t K,
                         const Epilogue &e, hipStream_t stream) {
    switch (dtype) {
    case MLP_F32: return narrow_type<float>(X, ldx, W, M, N, K, e, stream);
    case MLP_BF16: return narrow_type<bf16>(X, ldx, W, M, N, K, e, stream);
    default: return narrow_type<f16>(X, ldx, W, M, N, K, e, stream);
    }
}

}  // namespace mlp
