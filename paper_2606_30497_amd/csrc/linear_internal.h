// linear_internal.h -- shared declarations of the dense layer: its epilogue and the
// matrix product on the matrix cores (linear.hip, linear_gemm.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "layer.h"

namespace mlp {

// What becomes of the fp32 sums of a matrix product: Y = R + dropout(a(scale sum + bias)),
// Z = scale sum + bias; everything but Y may be missing.
struct Epilogue {
    float scale = 1.0f;   // a power of two
    const void *bias, *R;
    void *Z, *Y;
    int64_t ldr, ldz, ldy;
    int act;
    Drop drop;
};

// The epilogue of columns [c, c + 8), c a multiple of 8, for a lane that takes them of
// several rows. Columns from n on are not touched.
template <class T>
struct Finish {
    float bias[8];
    DropState drop;
    __device__ __forceinline__ void init(const Epilogue &e, int64_t c, int64_t n) {
#pragma unroll
        for (int j = 0; j < 8; ++j) bias[j] = 0.0f;
        if (e.bias && c < n) load8((const T *)e.bias, c, n, bias);
        if (e.drop.rng) drop.init(e.drop, n);
    }
    // v: the sums of row r; res: the row's residual
    __device__ __forceinline__ void finish(const Epilogue &e, int64_t r, int64_t c, int64_t n, float (&v)[8],
                                           const Oct<T> &res) const {
        if (e.scale != 1.0f) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= e.scale;
        }
        if (e.bias) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += bias[j];
        }
        if (e.Z) store8((T *)e.Z + r * e.ldz, c, n, v);
        activate8(e.act, v);
        if (e.drop.rng) drop8(drop.bits(r, c), e.drop.threshold, e.drop.scale, v);
        if (e.R) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += up(res.e[j]);
        }
        store8((T *)e.Y + r * e.ldy, c, n, v);
    }
};

// An operand of a product on tiles: rows of `ld` elements. 16-bit: 16-byte aligned, ld and
// the length of a row multiples of 8 (what pads a row is zero). fp32: at any address, `len`
// elements of a row readable, four at least (what pads a row is zero).
struct Operand {
    const void *p;
    int64_t ld, len;
};

// C[m][n] = sum_k a(m, k) b(k, n) for m < M, n < N, k < K. The products there are:
// NN: a(m, k) = A[m][k], b(k, n) = B[k][n]; NT: b(k, n) = B[n][k]; TN: a(m, k) = A[k][m],
// b(k, n) = B[k][n].
enum { GEMM_NN = 0, GEMM_NT = 1, GEMM_TN = 2 };

struct GemmArgs {
    Operand A, B;
    int64_t M, N, K;
    int64_t kc;              // depth of a split (a multiple of the chunk)
    int tiles_m, tiles_n, splits;
    float *part;             // splits > 1: [splits][M][N] fp32 sums
    Epilogue e;
};

// C (through e) of type dtype; part: room for part_floats partial sums. One or two
// launches on `stream`.
hipError_t launch_gemm(int op, int32_t dtype, const Operand &A, const Operand &B, int64_t M, int64_t N,
                       int64_t K, const Epilogue &e, float *part, int64_t part_floats, hipStream_t stream);

// The 16-bit GEMM_TN of N < 8 outputs where B counts as the sum of two: its rows are of 16
// elements, the second values from the eighth on.
hipError_t launch_gemm_fold(int32_t dtype, const Operand &A, const Operand &B, int64_t M, int64_t N, int64_t K,
                            const Epilogue &e, float *part, int64_t part_floats, hipStream_t stream);

hipError_t launch_gemm_f32(int op, const GemmArgs &g, int64_t part_floats, hipStream_t stream);
// the splits' sums through the epilogue, where there are splits
template <class T>
hipError_t join_splits(const GemmArgs &g, hipStream_t stream);

// The products of few rows, or small ones (linear_skinny.hip), on operands as the caller
// has them, of any alignment. GEMM_NN: Y = X W with W [K x N]; GEMM_NT: W [N x K].
// low (GEMM_NT of 16-bit types): 0, or X + low holds what the rounding of X's elements
// left, and X counts as the sum of both.
// part: room for part_floats partial sums; arrived: arrived_words words, zero before the
// call and after it. The grid is ceil(M / 16 or 32) workgroups high (below 65,536). N and
// K are at least SKINNY_WIDTH.
constexpr int64_t SKINNY_WIDTH = 8;
hipError_t launch_skinny(int op, int32_t dtype, const void *X, int64_t ldx, int64_t low, const void *W,
                         int64_t ldw, int64_t M, int64_t N, int64_t K, const Epilogue &e, float *part,
                         int64_t part_floats, uint32_t *arrived, int64_t arrived_words, hipStream_t stream);
// Y = X W of N < SKINNY_WIDTH outputs
hipError_t launch_narrow(int32_t dtype, const void *X, int64_t ldx, const void *W, int64_t M, int64_t N, int64_t K,
                         const Epilogue &e, hipStream_t stream);
// dW [K x N] = scale X^T G of M rows, N >= SKINNY_WIDTH; low as above, of G
hipError_t launch_outer(int32_t dtype, const void *X, int64_t ldx, const void *G, int64_t ldg, int64_t low,
                        int64_t M, int64_t K, int64_t N, float scale, void *dW, hipStream_t stream);

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace mlp
