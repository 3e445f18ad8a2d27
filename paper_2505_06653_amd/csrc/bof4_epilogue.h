// bof4_epilogue.h - where the products' kernels leave their sums: as they are (binary32 rows, or partial results that
// another kernel adds), or as the layer around the product has them:
//
//   y = act(z + bias) * mul + residual,   z = x W^T;   pre = z + bias is kept for the backward pass where it is wanted.
//
// Everything is binary32 up to the one rounding of each tensor that is written.  The choice of the kernels' Out type leaves
// the plain products as they were without it.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "bof4_device.h"

namespace bof4 {

// ------------------------------------------------------------------------------------------------ activations
// (the numbers of the C interface)
constexpr uint32_t ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4, ACT_COUNT = 5;
constexpr float GELU_TANH_A = 0.79788456080286536f, GELU_TANH_B = 0.044715f;  // sqrt(2 / pi)

// exp with the error of the argument's product with log2 e, 1.5 |q| 2^-24 of itself: what that leaves in a sigmoid times its
// argument is below 2^-24.
__device__ __forceinline__ float short_exp(float q) { return __builtin_amdgcn_exp2f(q * 1.44269504088896341f); }
__device__ __forceinline__ float sigmoid(float q) { return __builtin_amdgcn_rcpf(1.0f + short_exp(-q)); }
// (1 + tanh t) / 2 is the sigmoid of 2 t: silu and the tanh form of gelu share it.
__device__ __forceinline__ float activation(uint32_t act, float z) {
    if (act == ACT_NONE) return z;
    if (act == ACT_RELU) return z > 0.0f ? z : z != z ? z : 0.0f;
    if (act == ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    return z * sigmoid(act == ACT_SILU ? z : 2.0f * GELU_TANH_A * z * fmaf(GELU_TANH_B * z, z, 1.0f));
}
// The activation and its derivative.
__device__ __forceinline__ void activation_slope(uint32_t act, float z, float& value, float& slope) {
    if (act == ACT_NONE) {
        value = z;
        slope = 1.0f;
    } else if (act == ACT_RELU) {
        value = activation(act, z);
        slope = z > 0.0f ? 1.0f : z != z ? z : 0.0f;
    } else if (act == ACT_GELU) {
        const float cdf = 0.5f * (1.0f + erff(z * 0.70710678118654752f));
        value = z * cdf;
        slope = fmaf(z, 0.39894228040143268f * short_exp(-0.5f * z * z), cdf);
    } else {
        // (beyond 30 the tanh form's sigmoid is 0 or 1 in binary32; farther out its polynomial's slope would overflow)
        const bool silu = act == ACT_SILU;
        const float y = silu ? z : z > 30.0f ? 30.0f : z < -30.0f ? -30.0f : z;
        const float s = sigmoid(silu ? y : 2.0f * GELU_TANH_A * y * fmaf(GELU_TANH_B * y, y, 1.0f));
        const float inner = silu ? 1.0f : 2.0f * GELU_TANH_A * fmaf(3.0f * GELU_TANH_B * y, y, 1.0f);
        value = z * s;
        slope = s * fmaf(y * (1.0f - s), inner, 1.0f);
    }
}

// ------------------------------------------------------------------------------------------------ rows of either type
// N neighbouring elements (1, 2, 4 or 8) of a bfloat16 or binary32 row, of which the first n are there; in one or two accesses
// where all of them are, at any alignment (odd row strides element by element: 11009 x 4096, 2000 tokens, gradients 330 us
// instead of 248).
template <int N>
__device__ __forceinline__ void load_row(const void* p, uint64_t i, bool bf16, uint32_t n, float* v) {
    uint32_t w[N];
    if (bf16) {
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p) + i;
        if (N > 1 && n >= (uint32_t)N) {
            if constexpr (N == 2) w[0] = *reinterpret_cast<const u32_any*>(q);
            if constexpr (N == 4) {
                const u32x2_any t = *reinterpret_cast<const u32x2_any*>(q);
                w[0] = t.x;
                w[1] = t.y;
            }
            if constexpr (N == 8) {
                const u32x4_any t = *reinterpret_cast<const u32x4_any*>(q);
                w[0] = t.x;
                w[1] = t.y;
                w[2] = t.z;
                w[3] = t.w;
            }
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = k % 2 ? __uint_as_float(w[k / 2] & 0xffff0000u) : __uint_as_float(w[k / 2] << 16);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = (uint32_t)k < n ? bf16_bits_to_f32(q[k]) : 0.0f;
        }
    } else {
        const float* q = reinterpret_cast<const float*>(p) + i;
        if (N > 1 && n >= (uint32_t)N) {
            if constexpr (N == 2) {
                const u32x2_any t = *reinterpret_cast<const u32x2_any*>(q);
                w[0] = t.x;
                w[1] = t.y;
            } else {
#pragma unroll
                for (int k = 0; k + 4 <= N; k += 4) {
                    const u32x4_any t = *reinterpret_cast<const u32x4_any*>(q + k);
                    w[k] = t.x;
                    w[k + 1] = t.y;
                    w[k + 2] = t.z;
                    w[k + 3] = t.w;
                }
            }
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = __uint_as_float(w[k]);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = (uint32_t)k < n ? q[k] : 0.0f;
        }
    }
}
template <int N>
__device__ __forceinline__ void store_row(void* p, uint64_t i, bool bf16, uint32_t n, const float* v) {
    if (bf16) {
        uint16_t* q = reinterpret_cast<uint16_t*>(p) + i;
        if (N > 1 && n >= (uint32_t)N) {
            uint32_t w[N / 2 + 1];
#pragma unroll
            for (int k = 0; k < N / 2; ++k) w[k] = gemm_pack_bf16(v[2 * k], v[2 * k + 1]);
            if constexpr (N == 2) *reinterpret_cast<u32_any*>(q) = w[0];
            if constexpr (N == 4) *reinterpret_cast<u32x2_any*>(q) = u32x2_any{w[0], w[1]};
            if constexpr (N == 8) *reinterpret_cast<u32x4_any*>(q) = u32x4_any{w[0], w[1], w[2], w[3]};
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if ((uint32_t)k < n) q[k] = (uint16_t)f32_to_bf16_rne(v[k]);
        }
    } else {
        float* q = reinterpret_cast<float*>(p) + i;
        if (N > 1 && n >= (uint32_t)N) {
            uint32_t w[N];
#pragma unroll
            for (int k = 0; k < N; ++k) w[k] = __float_as_uint(v[k]);
            if constexpr (N == 2) {
                *reinterpret_cast<u32x2_any*>(q) = u32x2_any{w[0], w[1]};
            } else {
#pragma unroll
                for (int k = 0; k + 4 <= N; k += 4) *reinterpret_cast<u32x4_any*>(q + k) = u32x4_any{w[k], w[k + 1], w[k + 2], w[k + 3]};
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if ((uint32_t)k < n) q[k] = v[k];
        }
    }
}

// ------------------------------------------------------------------------------------------------ where sums go
// As they are: the first part of a row's columns to `first`, the others behind each other to `more`.
struct PlainOut {
    static constexpr bool LAYER = false;
    template <int T>
    struct Ahead {};
    float *first, *more;
    __device__ __forceinline__ float* part(uint32_t p, uint64_t n_tokens, uint32_t rows) const {
        return p == 0 ? first : more + (uint64_t)(p - 1) * n_tokens * rows;
    }
};

// The layer's result.  `parts`: not yet - every part of a row's columns goes there, for a kernel that adds them.
struct LayerOut {
    static constexpr bool LAYER = true;
    const void *bias, *mul, *residual;  // null: not there
    void *y, *pre;                      // (pre null: not wanted)
    uint64_t ld_mul, ld_residual, ld_y, ld_pre;
    uint32_t act;
    bool bias_bf16, mul_bf16, residual_bf16, y_bf16, pre_bf16;
    uint32_t token0;
    float* parts;
    __device__ __forceinline__ float* part(uint32_t p, uint64_t n_tokens, uint32_t rows) const {
        return parts + (uint64_t)p * n_tokens * rows;
    }
    // What one row's results of T tokens take besides the sums, asked for ahead of them.
    template <int T>
    struct Ahead {
        float bias, f[T], r[T];
    };
    template <int T>
    __device__ __forceinline__ Ahead<T> ask(uint32_t row) const {
        Ahead<T> a = {};
        if (bias) load_row<1>(bias, row, bias_bf16, 1, &a.bias);
#pragma unroll
        for (int t = 0; t < T; ++t) {
            if (mul) load_row<1>(mul, (uint64_t)(token0 + t) * ld_mul + row, mul_bf16, 1, &a.f[t]);
            if (residual) load_row<1>(residual, (uint64_t)(token0 + t) * ld_residual + row, residual_bf16, 1, &a.r[t]);
        }
        return a;
    }
    template <int T>
    __device__ __forceinline__ void store_one(uint32_t t, uint32_t row, const Ahead<T>& a, float z) const {
        if (bias) z += a.bias;
        if (pre) store_row<1>(pre, (uint64_t)(token0 + t) * ld_pre + row, pre_bf16, 1, &z);
        float v = activation(act, z);
        if (mul) v *= a.f[t];
        if (residual) v += a.r[t];
        store_row<1>(y, (uint64_t)(token0 + t) * ld_y + row, y_bf16, 1, &v);
    }
    // The sums of N neighbouring rows (a multiple of N first) of one token: read first, then written, so that y may be
    // the residual or the factor itself.
    template <int N>
    __device__ __forceinline__ void store(uint32_t token, uint32_t row, uint32_t rows, const float* sums) const {
        const uint32_t n = rows - row;  // (row < rows)
        const uint64_t t = token0 + token;
        float z[N], v[N], f[N], r[N];
#pragma unroll
        for (int k = 0; k < N; ++k) z[k] = sums[k];
        if (mul) load_row<N>(mul, t * ld_mul + row, mul_bf16, n, f);
        if (residual) load_row<N>(residual, t * ld_residual + row, residual_bf16, n, r);
        if (bias) {
            load_row<N>(bias, row, bias_bf16, n, v);
#pragma unroll
            for (int k = 0; k < N; ++k) z[k] += v[k];
        }
        if (pre) store_row<N>(pre, t * ld_pre + row, pre_bf16, n, z);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = activation(act, z[k]);
            if (mul) v[k] *= f[k];
            if (residual) v[k] += r[k];
        }
        store_row<N>(y, t * ld_y + row, y_bf16, n, v);
    }
};

}  // namespace bof4
