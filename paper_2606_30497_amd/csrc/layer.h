// layer.h -- what the layer operators (linear.hip, dropout.hip) share: element types,
// activations and their derivatives, and dropout from the Philox4x32-10 counter-based
// generator (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy
// as 1, 2, 3", SC'11).
#pragma once

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "bf16x3.h"
#include "mlp.h"

namespace mlp {

typedef __bf16 bf16;
typedef _Float16 f16;

// Eight consecutive elements of a row, as a lane holds them between memory and fp32
// registers. Rows are aligned to their element only: the packed words let the compiler
// use the widest load there is at any address.
template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Oct {
    T e[8];
};

__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ float up(bf16 v) { return (float)v; }
__device__ __forceinline__ float up(f16 v) { return (float)v; }

// columns [c, c + 8) of the row at p; columns from n on read nothing and give 0
template <class T>
__device__ __forceinline__ Oct<T> fetch8(const T *p, int64_t c, int64_t n) {
    Oct<T> o;
    if (c + 8 <= n) {
        o = *reinterpret_cast<const Oct<T> *>(p + c);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) o.e[j] = c + j < n ? p[c + j] : (T)0.0f;
    }
    return o;
}

template <class T>
__device__ __forceinline__ void load8(const T *p, int64_t c, int64_t n, float (&v)[8]) {
    const Oct<T> o = fetch8(p, c, n);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = up(o.e[j]);
}

// v, rounded once, to columns [c, c + 8) of the row at p, as far as they are below n
template <class T>
__device__ __forceinline__ void store8(T *p, int64_t c, int64_t n, const float (&v)[8]) {
    Oct<T> o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o.e[j] = (T)v[j];
    if (c + 8 <= n) {
        *reinterpret_cast<Oct<T> *>(p + c) = o;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < n) p[c + j] = o.e[j];
    }
}

// ---- dropout --------------------------------------------------------------------------

// One block of Philox4x32-10: ten rounds of two 32 x 32 -> 64 bit products, the key
// raised by two odd constants in between.
__device__ __forceinline__ u4v philox(uint64_t key, uint64_t counter) {
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = 0, c3 = 0;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u4v{c0, c1, c2, c3};
}

// Dropout of one call: 16 bits an element, so that a block serves the eight elements a
// lane holds and the generator's ten rounds stay below the time of their memory traffic.
struct Drop {
    const uint64_t *rng = nullptr;   // device (seed, offset); null: no dropout
    uint32_t threshold = 0;          // T: kept where the 16 bits are >= T (65536: nothing is)
    float scale = 1.0f;              // 1 / (1 - T 2^-16)
};

// false: p is no probability, or rng is missing
inline bool make_drop(float p, const uint64_t *rng, Drop *d) {
    *d = Drop();
    if (!(p >= 0.0f && p <= 1.0f)) return false;
    d->threshold = (uint32_t)floor((double)p * 65536.0 + 0.5);
    if (d->threshold == 0) return true;
    if (!rng) return false;
    d->rng = rng;
    d->scale = d->threshold < 65536u ? (float)(65536.0 / (65536.0 - d->threshold)) : 0.0f;
    return true;
}

// The seed and offset, read once by each thread.
struct DropState {
    uint64_t seed = 0, offset = 0, blocks_per_row = 0;
    __device__ __forceinline__ void init(const Drop &d, int64_t cols) {
        seed = d.rng[0];
        offset = d.rng[1];
        blocks_per_row = (uint64_t)((cols + 7) >> 3);
    }
    // the 128 bits of columns [c, c + 8) of row r, c a multiple of 8
    __device__ __forceinline__ u4v bits(int64_t r, int64_t c) const {
        return philox(seed, offset + (uint64_t)r * blocks_per_row + (uint64_t)(c >> 3));
    }
};

// v of the eight columns of a block: what is dropped becomes 0 whatever it was
__device__ __forceinline__ void drop8(u4v bits, uint32_t threshold, float scale, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t u = j & 1 ? bits[j >> 1] >> 16 : bits[j >> 1] & 0xFFFFu;
        v[j] = u >= threshold ? v[j] * scale : 0.0f;
    }
}

// ---- activations ------------------------------------------------------------------------

// 1 / (1 + exp(-t)), by the hardware's exponential and reciprocal (a few 2^-24 of its
// value, and |t| 2^-24 from the rounding of the exponent)
__device__ __forceinline__ float sigmoid(float t) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t * -1.44269504f));
}

constexpr float GELU_C = 1.5957691216057308f;   // 2 sqrt(2 / pi): z / (1 + exp(-C (z + 0.044715 z^3)))
constexpr float GELU_A = 0.044715f;

// The normal distribution function: Phi(-x) = e^(-x^2 / 2) F(x) for x >= 0, where F, with
// t = 1 / (1 + 0.31 x), is t times a polynomial in t (degree 7, fitted to F = erfcx(x /
// sqrt 2) / 2 for the least largest relative error, 1.6e-7; in fp32 Phi is within 2.2e-7
// of exact). A third of the instructions of 1 + erf, and e^(-z^2 / 2) (in `bell`) is the
// derivative's. For GELU of a 256 x 256 tile that is the larger part of its epilogue.
__device__ __forceinline__ float normal_cdf(float z, float &bell) {
    const float x = fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(0.31f, x, 1.0f));
    float p = 0.035841804f;
    p = fmaf(p, t, -0.14160487f);
    p = fmaf(p, t, 0.15506828f);
    p = fmaf(p, t, -0.014903724f);
    p = fmaf(p, t, 0.11011028f);
    p = fmaf(p, t, 0.10777105f);
    p = fmaf(p, t, 0.12406035f);
    p = fmaf(p, t, 0.12365691f);
    bell = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
    const float q = p * t * bell;
    return z < 0.0f ? q : 1.0f - q;
}

// v <- a(v)
__device__ __forceinline__ void activate8(int act, float (&v)[8]) {
    switch (act) {
    case MLP_ACT_RELU:
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = v[j] < 0.0f ? 0.0f : v[j];   // a NaN passes
        break;
    case MLP_ACT_GELU:
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float bell;
            v[j] *= normal_cdf(v[j], bell);
        }
        break;
    case MLP_ACT_GELU_TANH:
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= sigmoid(GELU_C * (v[j] + GELU_A * v[j] * v[j] * v[j]));
        break;
    case MLP_ACT_SILU:
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= sigmoid(v[j]);
        break;
    }
}

// v <- v a'(z); where ReLU masks, 0 whatever v is
__device__ __forceinline__ void activate_back8(int act, const float (&z)[8], float (&v)[8]) {
    switch (act) {
    case MLP_ACT_RELU:
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = z[j] > 0.0f ? v[j] : 0.0f;
        break;
    case MLP_ACT_GELU:   // Phi(z) + z phi(z)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float bell;
            const float cdf = normal_cdf(z[j], bell);
            v[j] *= cdf + z[j] * 0.39894228f * bell;
        }
        break;
    case MLP_ACT_GELU_TANH:
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // (s is 0 or 1 long before z^2 = 10^4; past it z^2 would become infinite)
            const float zz = GELU_A * fminf(z[j] * z[j], 1e4f), s = sigmoid(GELU_C * fmaf(z[j], zz, z[j]));
            v[j] *= s + z[j] * s * (1.0f - s) * GELU_C * fmaf(3.0f, zz, 1.0f);
        }
        break;
    case MLP_ACT_SILU:
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float s = sigmoid(z[j]);
            v[j] *= s * (1.0f + z[j] * (1.0f - s));
        }
        break;
    }
}

inline bool dtype_valid(int32_t t) { return t == MLP_F32 || t == MLP_BF16 || t == MLP_F16; }
inline size_t dtype_bytes(int32_t t) { return t == MLP_F32 ? 4 : 2; }

}  // namespace mlp
