// linear.hip -- a dense layer: z = X W + b, y = r + dropout(a(z)), and its gradients
//   g = dropout(dY) a'(z);  dX = g W^T;  dW = X^T g;  db = column sums of g
// for any widths, row strides and the three types of mlp_dtype.
#include <hip/hip_runtime.h>

#include <new>
#include <stdint.h>

#include "layer.h"

namespace mlp {

constexpr int64_t LINEAR_MAX_WIDTH = 1 << 20;

struct LinearCtx {
    int32_t dtype = 0, act = 0;
    int64_t d_in = 0, d_out = 0, max_rows = 0;
    const void *W = nullptr, *bias = nullptr;
    void *g = nullptr;          // [max_rows x ldg], the gradient in z
    int64_t ldg = 0;
    float *col = nullptr;       // [COL_CHUNKS x d_out], partial column sums of g
    hipStream_t stream = nullptr;
    int device = 0;
};

constexpr int COL_CHUNKS = 256;

// A matrix product's epilogue: what becomes of the fp32 sums of one row's eight columns.
struct Epilogue {
    const void *bias, *R;
    void *Z, *Y;
    int64_t ldr, ldz, ldy;
    int act;
    Drop drop;
};

template <class T>
__device__ __forceinline__ void finish8(const Epilogue &e, const DropState &st, int64_t r, int64_t c,
                                        int64_t n, float (&v)[8]) {
    if (e.bias) {
        float b[8];
        load8((const T *)e.bias, c, n, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += b[j];
    }
    if (e.Z) store8((T *)e.Z + r * e.ldz, c, n, v);
    if (e.act != MLP_ACT_NONE) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = activate(e.act, v[j]);
    }
    if (e.drop.rng) drop8(st.bits(r, c), e.drop.threshold, e.drop.scale, v);
    if (e.R) {
        float q[8];
        load8((const T *)e.R + r * e.ldr, c, n, q);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += q[j];
    }
    store8((T *)e.Y + r * e.ldy, c, n, v);
}

// C[m][n] = sum_k a(m, k) b(k, n), a(m, k) = A[m sam + k sak], b(k, n) = B[k sbk + n sbn],
// then the epilogue. 64 x 64 outputs a workgroup, K in chunks of 16 staged in LDS, two
// rows of eight columns a thread on the vector units.
struct ProductArgs {
    const void *A, *B;
    int64_t sam, sak, sbk, sbn, M, N, K;
    Epilogue e;
};

template <class T>
__global__ __launch_bounds__(256) void k_product(const ProductArgs a) {
    __shared__ float As[16][65], Bs[16][65];
    const int t = threadIdx.x;
    const int64_t m0 = (int64_t)blockIdx.x * 64, n0 = (int64_t)blockIdx.y * 64;
    const T *A = (const T *)a.A, *B = (const T *)a.B;
    const int tr = t >> 3, tc = (t & 7) * 8;
    float acc[2][8] = {};
    for (int64_t k0 = 0; k0 < a.K; k0 += 16) {
        for (int i = t; i < 1024; i += 256) {
            // the faster index along the operand's contiguous direction
            const int ak = a.sak == 1 ? i & 15 : i >> 6, am = a.sak == 1 ? i >> 4 : i & 63;
            const int bk = a.sbk == 1 ? i & 15 : i >> 6, bn = a.sbk == 1 ? i >> 4 : i & 63;
            As[ak][am] = m0 + am < a.M && k0 + ak < a.K ? up(A[(m0 + am) * a.sam + (k0 + ak) * a.sak]) : 0.0f;
            Bs[bk][bn] = n0 + bn < a.N && k0 + bk < a.K ? up(B[(k0 + bk) * a.sbk + (n0 + bn) * a.sbn]) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[i][j] += As[k][tr + 32 * i] * Bs[k][tc + j];
        __syncthreads();
    }
    DropState st;
    if (a.e.drop.rng) st.init(a.e.drop, a.N);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t m = m0 + tr + 32 * i;
        if (m < a.M && n0 + tc < a.N) finish8<T>(a.e, st, m, n0 + tc, a.N, acc[i]);
    }
}

// g = dropout(dY) a'(z) and its partial column sums: a workgroup takes a chunk of rows
// and 8 * groups columns.
struct GradArgs {
    const void *Z, *dY;
    void *G;
    float *col;               // nullable [chunks x N]
    int64_t ldz, lddy, ldg, M, N, chunk;   // chunk: rows of a workgroup
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
    const int64_t r1 = r0 + a.chunk < a.M ? r0 + a.chunk : a.M;
    DropState st;
    if (a.drop.rng) st.init(a.drop, a.N);
    float sum[8] = {};
    if (c < a.N) {
        for (int64_t r = r0 + t / a.groups; r < r1; r += 256 / a.groups) {
            float v[8];
            load8((const T *)a.dY + r * a.lddy, c, a.N, v);
            if (a.act != MLP_ACT_NONE) {
                float z[8];
                load8((const T *)a.Z + r * a.ldz, c, a.N, z);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = activate_back(a.act, z[j], v[j]);
            }
            if (a.drop.rng) drop8(st.bits(r, c), a.drop.threshold, a.drop.scale, v);
            store8((T *)a.G + r * a.ldg, c, a.ldg, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += v[j];
        }
    }
    if (!a.col) return;
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
        for (int j = 0; j < 8; ++j)
            if (c + j < a.N) a.col[(int64_t)blockIdx.x * a.N + c + j] = part[t][j];
    }
}

// db[n] = sum over the chunks, in order
template <class T>
__global__ __launch_bounds__(256) void k_column_sums(const float *col, int64_t chunks, int64_t N, T *db) {
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= N) return;
    float s = 0.0f;
    for (int64_t i = 0; i < chunks; ++i) s += col[i * N + n];
    db[n] = (T)s;
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

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static size_t pad256(size_t b) { return (b + 255) / 256 * 256; }

static bool linear_shape_ok(int32_t dtype, int64_t d_in, int64_t d_out, int64_t max_rows) {
    return dtype_valid(dtype) && d_in >= 1 && d_in <= LINEAR_MAX_WIDTH && d_out >= 1 &&
           d_out <= LINEAR_MAX_WIDTH && max_rows >= 1 && max_rows <= MLP_MAX_BATCH;
}

// Workspace: g, then the partial column sums.
static size_t linear_carve(LinearCtx *c, char *ws) {
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = ws + at;
        at += pad256(bytes);
        return p;
    };
    c->ldg = (c->d_out + 7) / 8 * 8;
    c->g = take((size_t)c->max_rows * c->ldg * dtype_bytes(c->dtype));
    c->col = (float *)take(sizeof(float) * COL_CHUNKS * (size_t)c->d_out);
    return at;
}

template <class T>
static hipError_t product(const LinearCtx &c, const ProductArgs &a) {
    const dim3 grid((unsigned)ceil_div(a.M, 64), (unsigned)ceil_div(a.N, 64));
    hipLaunchKernelGGL(k_product<T>, grid, dim3(256), 0, c.stream, a);
    return hipGetLastError();
}

template <class T>
static hipError_t linear_forward(const LinearCtx &c, const void *X, int64_t ldx, int64_t rows, const Epilogue &e) {
    ProductArgs a{X, c.W, ldx, 1, c.d_out, 1, rows, c.d_out, c.d_in, e};
    return product<T>(c, a);
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
    int64_t chunks = 0;
    if (M > 0) {
        GradArgs a;
        a.groups = 1;
        while (a.groups < 32 && a.groups * 8 < N) a.groups *= 2;
        const int64_t step = 256 / a.groups;
        a.chunk = ceil_div(ceil_div(M, COL_CHUNKS), step) * step;
        chunks = ceil_div(M, a.chunk);
        a.Z = b.Z;
        a.dY = b.dY;
        a.G = c.g;
        a.col = b.db ? c.col : nullptr;
        a.ldz = b.ldz;
        a.lddy = b.lddy;
        a.ldg = c.ldg;
        a.M = M;
        a.N = N;
        a.act = c.act;
        a.drop = b.drop;
        hipLaunchKernelGGL(k_linear_grad<T>, dim3((unsigned)chunks, (unsigned)ceil_div(N, 8 * a.groups)),
                           dim3(256), 0, c.stream, a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (b.db) {
        hipLaunchKernelGGL(k_column_sums<T>, dim3((unsigned)ceil_div(N, 256)), dim3(256), 0, c.stream, c.col,
                           chunks, N, (T *)b.db);
        if (hipError_t e = hipGetLastError()) return e;
    }
    Epilogue e{};
    if (b.dX && M > 0) {
        e.Y = b.dX;
        e.ldy = b.lddx;
        if (hipError_t s = product<T>(c, ProductArgs{c.g, c.W, c.ldg, 1, 1, N, M, K, N, e})) return s;
    }
    if (b.dW) {
        e.Y = b.dW;
        e.ldy = N;
        if (hipError_t s = product<T>(c, ProductArgs{b.X, c.g, 1, b.ldx, c.ldg, 1, K, N, M, e})) return s;
    }
    return hipSuccess;
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
    if (hipGetDevice(&c->device) != hipSuccess) {
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
    if (!X || !Y || X == Y || Z == Y || Z == X || Y == c->W || Z == c->W || (Z && Z == residual) ||
        (residual == Y && ldr != ldy))
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
    if (rows > 0) {
        if (!dY || (dW && !X) || (c->act != MLP_ACT_NONE && !Z)) return MLP_ERR_INVALID_ARG;
        for (const void *o : {(const void *)dX, (const void *)dW, (const void *)dbias})
            if (o && (o == X || o == Z || o == dY || o == c->W || o == c->bias)) return MLP_ERR_INVALID_ARG;
        if ((dX && (dX == dW || dX == dbias)) || (dW && dW == dbias)) return MLP_ERR_INVALID_ARG;
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
