// linear.hip -- a dense layer: z = X W + b, y = r + dropout(a(z)), and its gradients
//   g = dropout(dY) a'(z);  dX = g W^T;  dW = X^T g;  db = column sums of g
// for any widths, row strides and the three types of mlp_dtype.
#include <hip/hip_runtime.h>

#include <initializer_list>
#include <new>
#include <stdint.h>
#include <type_traits>

#include "layer.h"
#include "linear_internal.h"

namespace mlp {

constexpr int64_t LINEAR_MAX_WIDTH = 1 << 20;
constexpr int COL_CHUNKS = 256;                   // most row chunks of the column sums
constexpr int64_t ARRIVED_WORDS = 16384;
constexpr int64_t FEW_ROWS = 2048;                // most rows of a small product (few_rows)
constexpr int64_t REST_ROWS = 64;                 // most rows whose g comes in two 16-bit values (linear_backward)
constexpr int64_t TILE_ROWS = 32;                 // up to here, at widths of eight and more, no tiles at all
constexpr int64_t PART_TILES = 256 * 128 * 128;   // partial sums of 256 workgroups' split tiles, 128 x 128 at most
constexpr int64_t PART_FEW = 256 * 32 * 128;      // and of k_skinny's 256 workgroups

struct LinearCtx {
    int32_t dtype = 0, act = 0;
    int64_t d_in = 0, d_out = 0, max_rows = 0;
    const void *W = nullptr, *bias = nullptr;
    // workspace: operands as the matrix products take them (Operand): the gradient in z,
    // and X and W where the caller's are not laid out so
    void *g = nullptr, *x = nullptr, *w = nullptr;
    float *col = nullptr;       // [grad_chunks x d_out], partial column sums of g
    float *part = nullptr;      // partial sums of the products
    int64_t part_floats = 0;
    uint32_t *arrived = nullptr;   // the few-row products' arrival counts, zero between calls
    int64_t arrived_words = 0;
    hipStream_t stream = nullptr;
    int device = 0;
};

static int64_t pad8(int64_t n) { return (n + 7) / 8 * 8; }

// Matrices of rows x cols to be laid out as operands: rows of pad8(cols) elements, what pads
// them zero; each row 2^twice times. Read and written once, bound by memory; one launch for
// all of a call's.
struct PackArgs {
    struct Job {
        const void *P;
        void *out;
        int64_t ld, rows, cols;   // rows: of the output
        int twice;
    } job[3];
    int64_t groups[3];   // of workgroups, up to and with each job's
    int jobs;
};

template <class T>
__global__ __launch_bounds__(256) void k_pack(const PackArgs a) {
    int j = 0;
    while (j + 1 < a.jobs && blockIdx.x >= a.groups[j]) ++j;
    const int64_t first = j ? a.groups[j - 1] : 0, step = (a.groups[j] - first) * 256;
    const T *P = (const T *)a.job[j].P;
    T *out = (T *)a.job[j].out;
    const int64_t ld = a.job[j].ld, cols = a.job[j].cols;
    const int twice = a.job[j].twice;
    const int64_t blocks = (cols + 7) / 8, total = a.job[j].rows * blocks;
    for (int64_t i = ((int64_t)blockIdx.x - first) * 256 + threadIdx.x; i < total; i += step) {
        const int64_t r = i / blocks, c = (i - r * blocks) * 8;
        float v[8];
        load8(P + (r >> twice) * ld, c, cols, v);
        store8(out + r * blocks * 8, c, blocks * 8, v);
    }
}

// g = dropout(dY) a'(z) and its partial column sums: a workgroup takes a chunk of rows
// and 8 * groups columns, a thread eight columns of every 256 / groups rows, the next row's
// on their way. Bound by memory and the derivative's arithmetic (8,192 x 4,096 in bf16,
// GELU: 65 us, 3.1 TB/s).
struct GradArgs {
    const void *Z, *dY;
    void *G;                  // nullable, an operand of rows of pad8(N) elements, ldg apart
    int64_t ldg, low;         // low: 0, or elements from G to what its rounding to a 16-bit type left
    float shrink;             // what G holds is g times this (fp16; else 1)
    float *col;               // nullable [chunks x N]
    void *db;                 // nullable [N], of a single chunk
    int64_t ldz, lddy, M, N, chunk;   // chunk: rows of a workgroup
    int groups;               // a power of two up to 32
    int act;
    Drop drop;
};

template <class T>
__global__ __launch_bounds__(256) void k_linear_grad(const GradArgs a) {
    __shared__ float part[256][9];
    const int t = threadIdx.x;
    const int64_t c = ((int64_t)blockIdx.y * a.groups + t % a.groups) * 8;
    const int64_t r0 = (int64_t)blockIdx.x * a.chunk;
    const int64_t r1 = r0 + a.chunk < a.M ? r0 + a.chunk : a.M, padded = (a.N + 7) / 8 * 8;
    DropState st;
    if (a.drop.rng) st.init(a.drop, a.N);
    float sum[8] = {};
    if (c < a.N) {
        const int64_t step = 256 / a.groups;
        int64_t r = r0 + t / a.groups;
        const T *dY = (const T *)a.dY + r * a.lddy, *Z = (const T *)a.Z + r * a.ldz;
        Oct<T> dy, z;
        auto fetch = [&]() __attribute__((always_inline)) {
            dy = fetch8(dY, c, a.N);
            if (a.act != MLP_ACT_NONE) z = fetch8(Z, c, a.N);
            dY += step * a.lddy;
            Z += step * a.ldz;
        };
        if (r < r1) fetch();
        for (; r < r1; r += step) {
            float v[8], zf[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = up(dy.e[j]);
                zf[j] = up(z.e[j]);
            }
            if (r + step < r1) fetch();   // the next row's, ahead of this one's work
            if (a.act != MLP_ACT_NONE) activate_back8(a.act, zf, v);
            if (a.drop.rng) drop8(st.bits(r, c), a.drop.threshold, a.drop.scale, v);
            if (c + 8 > a.N) {   // what pads a row is 0
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = c + j < a.N ? v[j] : 0.0f;
            }
            if (a.G) {
                T *G = (T *)a.G + r * a.ldg;
                float w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = std::is_same<T, f16>::value ? v[j] * a.shrink : v[j];
                if (a.low) {   // (an infinity goes to the second value: of two, inf - inf would be left)
                    constexpr float MOST = std::is_same<T, f16>::value ? 65504.0f : 3.38953139e38f;
                    float rest[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float first = fminf(fmaxf(w[j], -MOST), MOST);
                        rest[j] = w[j] - up((T)first);
                        w[j] = first;
                    }
                    store8(G + a.low, c, padded, rest);
                }
                store8(G, c, padded, w);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += v[j];
        }
    }
    if (!a.col && !a.db) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) part[t][j] = sum[j];
    __syncthreads();
    for (int s = 128; s >= a.groups; s >>= 1) {
        if (t < s) {
#pragma unroll
            for (int j = 0; j < 8; ++j) part[t][j] += part[t + s][j];
        }
        __syncthreads();
    }
    if (t < a.groups) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (c + j >= a.N) continue;
            if (a.db) ((T *)a.db)[c + j] = (T)part[t][j];
            else a.col[(int64_t)blockIdx.x * a.N + c + j] = part[t][j];
        }
    }
}

// db[n] = the sum of the chunks' column sums: 32 columns a workgroup, each by eight
// threads that take every eighth chunk, summed in order.
template <class T>
__global__ __launch_bounds__(256) void k_column_sums(const float *col, int64_t chunks, int64_t N, T *db) {
    __shared__ float part[8][33];
    const int t = threadIdx.x & 31, q = threadIdx.x >> 5;
    const int64_t n = (int64_t)blockIdx.x * 32 + t;
    float s = 0.0f;
    if (n < N)
#pragma unroll 4
        for (int64_t i = q; i < chunks; i += 8) s += col[i * N + n];
    part[q][t] = s;
    __syncthreads();
    if (q == 0 && n < N) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += part[i][t];
        db[n] = (T)s;
    }
}

// The context's device, current for the length of a call.
struct OnDevice {
    int before = -1;
    bool ok;
    explicit OnDevice(int device) {
        ok = hipGetDevice(&before) == hipSuccess;
        if (!ok || before == device) before = -1;
        else ok = hipSetDevice(device) == hipSuccess;
    }
    ~OnDevice() {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

static size_t pad256(size_t b) { return (b + 255) / 256 * 256; }

static bool linear_shape_ok(int32_t dtype, int64_t d_in, int64_t d_out, int64_t max_rows) {
    return dtype_valid(dtype) && d_in >= 1 && d_in <= LINEAR_MAX_WIDTH && d_out >= 1 &&
           d_out <= LINEAR_MAX_WIDTH && max_rows >= 1 && max_rows <= MLP_MAX_BATCH;
}

// Whether a width is below what linear_skinny.hip takes.
static bool any_narrow(const LinearCtx &c) { return c.d_in < SKINNY_WIDTH || c.d_out < SKINNY_WIDTH; }

// Columns of a workgroup of k_linear_grad, in eights (few rows: as many rows at a time as there
// are, and fewer columns), and the most chunks of rows it takes a call's in: about four
// workgroups a compute unit; up to 64 rows in one chunk, which gives db by itself.
static int grad_groups(int64_t M, int64_t N) {
    const int most = M > 32 && M <= 64 ? 4 : M > 16 && M <= 32 ? 8 : M > 8 && M <= 16 ? 16 : 32;
    int groups = 1;
    while (groups < most && groups * 8 < N) groups *= 2;
    return groups;
}
static int64_t grad_chunks(int64_t M, int64_t N) {
    if (M <= 64) return 1;
    const int64_t want = ceil_div(1024, ceil_div(N, 8 * grad_groups(M, N)));
    return want < COL_CHUNKS ? want : COL_CHUNKS;
}

// Floats that the partial sums of a product of M x N outputs take at most: splits of a depth
// of 128 at least (four chunks of a tile, or a step of the eight waves of k_skinny, whose
// rows of outputs are whole tiles), for up to 256 workgroups (512 of 64 x 64 tiles).
static int64_t part_room(int64_t M, int64_t N, int64_t depth, int64_t most) {
    const int64_t splits = ceil_div(depth, 128), all = M * (ceil_div(N, 128) * 128) * splits;
    return splits <= 1 ? 0 : all < most ? all : most;
}

// Workspace (ws null: its size alone): the arrival counts, at the start and as many whatever
// the shape, so that contexts may share it (what else is there no call keeps); the operands g,
// X and W (of 16-bit types with room for the second values of g, and for X and W twice where
// narrow products need that; X and W only where there are tiles), the partial column sums, the
// partial products.
static size_t linear_carve(LinearCtx *c, char *ws) {
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = ws ? ws + at : nullptr;
        at += pad256(bytes);
        return p;
    };
    const size_t element = dtype_bytes(c->dtype);
    const int64_t M = c->max_rows, K = c->d_in, N = c->d_out;
    const int64_t more = element == 4 ? 0 : M < REST_ROWS || N < SKINNY_WIDTH ? M : REST_ROWS;
    const bool twice = element == 2 && any_narrow(*c);
    c->arrived_words = ARRIVED_WORDS;
    c->arrived = (uint32_t *)take(sizeof(uint32_t) * (size_t)c->arrived_words);
    c->g = take(element * (M + more) * pad8(N));
    const bool tiles = M > TILE_ROWS || any_narrow(*c);
    c->x = take(tiles ? element * (M + (twice && N >= SKINNY_WIDTH ? more : 0)) * pad8(K) : 0);
    c->w = take(tiles ? element * (twice ? 2 * K : K) * pad8(N) : 0);
    c->col = (float *)take(M > 64 ? sizeof(float) * grad_chunks(M, N) * (size_t)N : 0);
    c->part_floats = 0;
    const int64_t most = tiles ? PART_TILES : PART_FEW;
    for (const int64_t n : {part_room(M, N, K, most), part_room(M, K, N, most), part_room(K, N, M, most)})
        if (n > c->part_floats) c->part_floats = n;
    c->part = (float *)take(sizeof(float) * (size_t)c->part_floats);
    return at;
}

// Operands of a call's products.
struct Operands {
    const LinearCtx &c;
    PackArgs a{};
    explicit Operands(const LinearCtx &ctx) : c(ctx) {}
    // The matrix [rows x cols] at P: as it is where its layout is an operand's (and its rows
    // close enough for 32-bit offsets within a tile), else packed at `room` by launch(); twice:
    // each row two times, packed.
    template <class T>
    Operand get(const void *P, int64_t ld, int64_t rows, int64_t cols, void *room, bool twice = false) {
        if (rows <= 1) ld = pad8(cols);
        const bool fits = sizeof(T) == 4 ? cols >= 4 : ((uintptr_t)P & 15u) == 0 && ld % 8 == 0 && cols % 8 == 0;
        if (fits && ld < (1 << 22) && !twice) return Operand{P, ld, cols};
        if (twice) rows *= 2;
        if (rows > 0) {
            const int64_t need = ceil_div(rows * (pad8(cols) / 8), 256);
            a.job[a.jobs] = PackArgs::Job{P, room, ld, rows, cols, twice};
            a.groups[a.jobs] = (a.jobs ? a.groups[a.jobs - 1] : 0) + (need < 4096 ? need : 4096);
            ++a.jobs;
        }
        return Operand{room, pad8(cols), pad8(cols)};
    }
    template <class T>
    hipError_t launch() {
        if (a.jobs == 0) return hipSuccess;
        hipLaunchKernelGGL(k_pack<T>, dim3((unsigned)a.groups[a.jobs - 1]), dim3(256), 0, c.stream, a);
        a.jobs = 0;
        return hipGetLastError();
    }
};

// Whether the products of M rows with W go to linear_skinny.hip: those of a few rows, and
// small ones, the deep ones among them up to a larger size, since on tiles their depth is
// split over many (us here and on tiles; y in bf16: 1,024 x 512 x 512 5.8 and 6.4, with 2^29
// products, 2,048 x 512 x 512, 6.8 and 6.7; in fp32: 128 x 1,024 x 1,024 10 and 13, 512 x 1,024 x
// 1,024 21 and 19, 100 x 16,384 x 300 30 and 52; dX in fp32: 512 x 512 x 512 11 and 13, 256 x
// 1,024 x 1,024 16 and 15, 100 x 300 x 16,384 32 and 37; in bf16: 64 x 1,024 x 1,024 8.4 and 8.4,
// 256 x 1,024 x 1,024 10.2 and 8.5, 100 x 30 x 10,001 14 and 28).
static bool few_rows(const LinearCtx &c, int64_t M, bool back) {
    if (any_narrow(c)) return false;
    const bool f32 = c.dtype == MLP_F32, deep = (back ? c.d_out : c.d_in) > 4096;
    const int64_t rows = back && !f32 && !deep ? 64 : FEW_ROWS;
    const int64_t size = !f32 ? 1 << 28 : deep ? 1 << 29 : back ? 1 << 27 : 1 << 28;
    return M <= (f32 ? 64 : TILE_ROWS) || (M <= rows && M * c.d_in * c.d_out <= size);
}

// Whether y of fewer than eight outputs goes to k_narrow (us there and on tiles, rows x depth x
// outputs; fp32: 64 x 256 x 7 6.0 and 11, 3,000 x 256 x 7 10.4 and 11, 65,536 x 256 x 1 32 and
// 33, 65,536 x 1,024 x 3 56 and 107, 65,536 x 1,024 x 7 154 and 105, 3,000 x 16,384 x 3 38 and 93; bf16,
// whose values take an instruction more each and half of the bytes: 64 x 1,024 x 7 7.4 and
// 10.5, 64 x 256 x 7 7.6 and 7.0, 3,000 x 4,097 x 7 29 and 31, 65,536 x 1,024 x 1 68 and 29).
static bool narrow(const LinearCtx &c, int64_t M) {
    if (c.d_out >= SKINNY_WIDTH) return false;
    if (c.dtype != MLP_F32) return M <= 2048 && c.d_in >= 128 * c.d_out;
    return c.d_in >= (M <= 1024 ? 128 : 256 * c.d_out);
}

template <class T>
static hipError_t linear_forward(const LinearCtx &c, const void *X, int64_t ldx, int64_t rows, const Epilogue &e) {
    if (few_rows(c, rows, false))
        return launch_skinny(GEMM_NN, c.dtype, X, ldx, 0, c.W, c.d_out, rows, c.d_out, c.d_in, e, c.part,
                             c.part_floats, c.arrived, c.arrived_words, c.stream);
    if (narrow(c, rows))
        return launch_narrow(c.dtype, X, ldx, c.W, rows, c.d_out, c.d_in, e, c.stream);
    Operands o(c);
    const Operand x = o.get<T>(X, ldx, rows, c.d_in, c.x), w = o.get<T>(c.W, c.d_out, c.d_in, c.d_out, c.w);
    if (hipError_t s = o.launch<T>()) return s;
    return launch_gemm(GEMM_NN, c.dtype, x, w, rows, c.d_out, c.d_in, e, c.part, c.part_floats, c.stream);
}

// The power of two that |g| / |dY| stays below: fp16 has no room for a'(z) > 1 and dropout's
// 1 / q next to a dY of a loss that was scaled up, so g is kept divided by this, and the sums
// are multiplied with it. (The smallest step of g grows with it, to at most twice what dY's own
// smallest step makes in g.)
static float headroom(int act, const Drop &drop) {
    const float most = (act == MLP_ACT_NONE || act == MLP_ACT_RELU ? 1.0f : 1.13f) * (drop.rng ? drop.scale : 1.0f);
    float s = 1.0f;
    while (s < most) s *= 2.0f;
    return s;
}

struct BackwardArgs {
    const void *X, *Z, *dY;
    int64_t ldx, ldz, lddy, rows;
    Drop drop;
    void *dX, *dW, *db;
    int64_t lddx;
};

template <class T>
static hipError_t linear_backward(const LinearCtx &c, const BackwardArgs &b) {
    const int64_t M = b.rows, N = c.d_out, K = c.d_in;
    const bool products = M > 0 && (b.dX || b.dW), as_is = c.act == MLP_ACT_NONE && !b.drop.rng;
    const bool few = few_rows(c, M, true);
    // The products take g rounded to a 16-bit type, a rounding more than their result's own.
    // Of up to 64 rows, where it would show (an element of g is in every value of a row of
    // dX) and W or latency is the bound, what it left goes along as a second value, behind
    // the first ones of the row; and of fewer than eight outputs, whose second values take
    // columns of the tiles that are idle (both gradients in bf16, us with and without: 65,536 x
    // 4,096 x 1 343 and 344, 3,000 x 16,384 x 3 63 and 63). Few rows of fewer than eight inputs
    // pay a few us (64 x 1 x 4,096 27 and 23, 64 x 7 x 1,000 22 and 19). Large products of 33
    // to 64 rows do without (64 x 4,096 x 4,096 50 and 35), as more rows do, whose matrix
    // instructions would be twice as many (456 of the 530 us of 8,192 x 4,096 x 4,096, for an
    // error of dX and dW of 1.65e-3, their own rounding's, in place of 2.34e-3).
    const bool fold = sizeof(T) == 2 && !as_is && N < SKINNY_WIDTH;
    const bool rest = fold || (sizeof(T) == 2 && !as_is && M <= REST_ROWS && (few || any_narrow(c)));
    // g that is dY itself: dY is the operand (of few rows, where 32-bit offsets reach over
    // the depth of a step)
    const bool same = as_is && (!few || b.lddy < (1 << 24));
    // what goes to linear_skinny.hip: dX of few_rows, and dW of 32 rows (us there and on
    // tiles, 4,096 x 4,096: bf16 12.5 and 14.6, fp32 33 and 33) or, for the second values, 64
    const bool outer = few && M <= (sizeof(T) == 4 ? TILE_ROWS : REST_ROWS);
    // Second values on tiles: (g, low) by (w, w) along the depth of dX; for dW as columns of
    // their own, which are folded, or by x in the row of g and in that of low, which alternate.
    const bool twice = rest && !few;
    const float scale = std::is_same<T, f16>::value && !as_is ? headroom(c.act, b.drop) : 1.0f;
    const int64_t low = rest ? pad8(N) : 0, ldg = pad8(N) + low;
    Operands o(c);
    Operand x{}, w{c.W, N, N}, g{c.g, ldg, ldg};
    if (same && products) {
        if (few && (outer || !b.dW)) g = Operand{b.dY, b.lddy, N};
        else g = o.get<T>(b.dY, b.lddy, M, N, c.g);
    }
    // (16-bit rows that start at odd elements load slowly: where many rows of g read W, it is
    // laid out first for k_skinny too: 700 x 30 x 10,001 in bf16 29 us, 20 so)
    if (b.dX && M > 0 && (!few || (sizeof(T) == 2 && M > 128 && N % 2))) w = o.get<T>(c.W, N, K, N, c.w, twice);
    if (b.dW && !outer) x = o.get<T>(b.X, b.ldx, M, K, c.x, twice && !fold);
    if (hipError_t e = o.launch<T>()) return e;
    int64_t chunks = 0;
    if (M > 0 && (b.db || (products && !same))) {
        GradArgs a;
        a.groups = grad_groups(M, N);
        const int64_t step = 256 / a.groups;
        a.chunk = M <= 64 ? M : ceil_div(ceil_div(M, grad_chunks(M, N)), step) * step;
        chunks = ceil_div(M, a.chunk);
        a.Z = b.Z;
        a.dY = b.dY;
        a.G = products && !same ? c.g : nullptr;
        a.ldg = ldg;
        a.low = low;
        a.shrink = 1.0f / scale;
        a.col = b.db && chunks > 1 ? c.col : nullptr;
        a.db = chunks == 1 ? b.db : nullptr;
        a.ldz = b.ldz;
        a.lddy = b.lddy;
        a.M = M;
        a.N = N;
        a.act = c.act;
        a.drop = b.drop;
        hipLaunchKernelGGL(k_linear_grad<T>, dim3((unsigned)chunks, (unsigned)ceil_div(N, 8 * a.groups)),
                           dim3(256), 0, c.stream, a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (b.db && chunks != 1) {
        hipLaunchKernelGGL(k_column_sums<T>, dim3((unsigned)ceil_div(N, 32)), dim3(256), 0, c.stream, c.col,
                           chunks, N, (T *)b.db);
        if (hipError_t e = hipGetLastError()) return e;
    }
    Epilogue e{};
    e.scale = scale;
    if (b.dX && M > 0) {
        e.Y = b.dX;
        e.ldy = b.lddx;
        if (twice) w.ld = w.len = ldg;
        const hipError_t s =
            few ? launch_skinny(GEMM_NT, c.dtype, g.p, g.ld, low, w.p, w.ld, M, K, N, e, c.part, c.part_floats, c.arrived,
                                c.arrived_words, c.stream)
                : launch_gemm(GEMM_NT, c.dtype, g, w, M, K, twice ? ldg : N, e, c.part, c.part_floats, c.stream);
        if (s != hipSuccess) return s;
    }
    if (!b.dW) return hipSuccess;
    if (outer) return launch_outer(c.dtype, b.X, b.ldx, g.p, g.ld, low, M, K, N, scale, b.dW, c.stream);
    e.Y = b.dW;
    e.ldy = N;
    if (fold)
        return launch_gemm_fold(c.dtype, x, g, K, N, M, e, c.part, c.part_floats, c.stream);
    if (twice) g.ld = g.len = low;
    return launch_gemm(GEMM_TN, c.dtype, x, g, K, N, twice ? 2 * M : M, e, c.part, c.part_floats, c.stream);
}

__global__ __launch_bounds__(256) void k_clear(uint32_t *p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

}  // namespace mlp

using namespace mlp;

struct mlp_linear_ctx : mlp::LinearCtx {};

extern "C" size_t mlp_linear_workspace_bytes(int32_t dtype, int64_t d_in, int64_t d_out, int64_t max_rows) {
    if (!linear_shape_ok(dtype, d_in, d_out, max_rows)) return 0;
    LinearCtx c;
    c.dtype = dtype;
    c.d_in = d_in;
    c.d_out = d_out;
    c.max_rows = max_rows;
    return linear_carve(&c, nullptr);
}

extern "C" mlp_status mlp_linear_init(mlp_linear_t *out, int32_t dtype, int64_t d_in, int64_t d_out,
                                      int32_t activation, int64_t max_rows, const void *W,
                                      const void *bias, void *workspace, size_t ws_bytes, void *stream) {
    if (!out || !W || !workspace) return MLP_ERR_INVALID_ARG;
    if (!linear_shape_ok(dtype, d_in, d_out, max_rows) || activation < MLP_ACT_NONE || activation > MLP_ACT_SILU)
        return MLP_ERR_UNSUPPORTED;
    const size_t need = mlp_linear_workspace_bytes(dtype, d_in, d_out, max_rows);
    if (ws_bytes < need || ((uintptr_t)workspace & 255u)) return MLP_ERR_WORKSPACE;
    mlp_linear_ctx *c = new (std::nothrow) mlp_linear_ctx();
    if (!c) return MLP_ERR_HIP;
    c->dtype = dtype;
    c->act = activation;
    c->d_in = d_in;
    c->d_out = d_out;
    c->max_rows = max_rows;
    c->W = W;
    c->bias = bias;
    c->stream = (hipStream_t)stream;
    linear_carve(c, (char *)workspace);
    hipError_t e = hipGetDevice(&c->device);
    if (e == hipSuccess) {
        hipLaunchKernelGGL(k_clear, dim3((unsigned)ceil_div(c->arrived_words, 256)), dim3(256), 0, c->stream,
                           c->arrived, c->arrived_words);
        e = hipGetLastError();
    }
    if (e != hipSuccess) {
        delete c;
        return MLP_ERR_HIP;
    }
    *out = c;
    return MLP_OK;
}

extern "C" mlp_status mlp_linear_set_stream(mlp_linear_t c, void *stream) {
    if (!c) return MLP_ERR_INVALID_ARG;
    c->stream = (hipStream_t)stream;
    return MLP_OK;
}

extern "C" void mlp_linear_destroy(mlp_linear_t c) { delete c; }

// a stride of a [rows x cols] matrix whose last offset stays far from 64 bits
static bool stride_ok(int64_t ld, int64_t rows, int64_t cols) {
    return rows <= 1 || (ld >= cols && ld < ((int64_t)1 << 46) / rows);
}

#define MLP_BY_TYPE(c, call)                              \
    ((c)->dtype == MLP_F32    ? call<float>              \
     : (c)->dtype == MLP_BF16 ? call<bf16>               \
                              : call<f16>)

extern "C" mlp_status mlp_linear_forward(mlp_linear_t c, const void *X, int64_t ldx, int64_t rows,
                                         const void *residual, int64_t ldr, float p, const uint64_t *rng,
                                         void *Y, int64_t ldy, void *Z, int64_t ldz) {
    Epilogue e{};
    if (!c || rows < 0 || rows > c->max_rows || !make_drop(p, rng, &e.drop)) return MLP_ERR_INVALID_ARG;
    if (rows == 0) return MLP_OK;
    if (!X || !Y || X == Y || Z == Y || Z == X || Y == c->W || Z == c->W || Y == c->bias ||
        (Z && (Z == residual || Z == c->bias)) || (residual == Y && ldr != ldy))
        return MLP_ERR_INVALID_ARG;
    if (!stride_ok(ldx, rows, c->d_in) || !stride_ok(ldy, rows, c->d_out) ||
        (residual && !stride_ok(ldr, rows, c->d_out)) || (Z && !stride_ok(ldz, rows, c->d_out)))
        return MLP_ERR_INVALID_ARG;
    e.bias = c->bias;
    e.R = residual;
    e.ldr = ldr;
    e.Z = Z;
    e.ldz = ldz;
    e.Y = Y;
    e.ldy = ldy;
    e.act = c->act;
    OnDevice dev(c->device);
    if (!dev.ok) return MLP_ERR_HIP;
    return MLP_BY_TYPE(c, linear_forward)(*c, X, ldx, rows, e) == hipSuccess ? MLP_OK : MLP_ERR_HIP;
}

extern "C" mlp_status mlp_linear_backward(mlp_linear_t c, const void *X, int64_t ldx, const void *Z,
                                          int64_t ldz, const void *dY, int64_t lddy, int64_t rows, float p,
                                          const uint64_t *rng, void *dX, int64_t lddx, void *dW,
                                          void *dbias) {
    BackwardArgs b;
    if (!c || rows < 0 || rows > c->max_rows || !make_drop(p, rng, &b.drop)) return MLP_ERR_INVALID_ARG;
    for (const void *o : {(const void *)dX, (const void *)dW, (const void *)dbias})
        if (o && (o == X || o == Z || o == dY || o == c->W || o == c->bias)) return MLP_ERR_INVALID_ARG;
    if ((dX && (dX == dW || dX == dbias)) || (dW && dW == dbias)) return MLP_ERR_INVALID_ARG;
    if (rows > 0) {
        if (!dY || (dW && !X) || (c->act != MLP_ACT_NONE && !Z)) return MLP_ERR_INVALID_ARG;
        if (!stride_ok(lddy, rows, c->d_out) || (dW && !stride_ok(ldx, rows, c->d_in)) ||
            (c->act != MLP_ACT_NONE && !stride_ok(ldz, rows, c->d_out)) ||
            (dX && !stride_ok(lddx, rows, c->d_in)))
            return MLP_ERR_INVALID_ARG;
    }
    b.X = X;
    b.ldx = ldx;
    b.Z = Z;
    b.ldz = ldz;
    b.dY = dY;
    b.lddy = lddy;
    b.rows = rows;
    b.dX = dX;
    b.lddx = lddx;
    b.dW = dW;
    b.db = dbias;
    OnDevice dev(c->device);
    if (!dev.ok) return MLP_ERR_HIP;
    return MLP_BY_TYPE(c, linear_backward)(*c, b) == hipSuccess ? MLP_OK : MLP_ERR_HIP;
}
