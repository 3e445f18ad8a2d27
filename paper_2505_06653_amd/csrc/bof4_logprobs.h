// bof4_logprobs.h - log probabilities of given tokens from a model's logits, with entropy and the largest alternatives,
// and the gradient by the logits.  What a quantised model is judged by (the perplexity of section 5 is the exponential of
// the mean negative log probability) and trained by.
//
//   p_j = exp(x_j - m) / S,  m = max_j x_j,  S = sum_j exp(x_j - m);   log p_j = (x_j - m) - log S
//   entropy H = -sum_j p_j log p_j = log S - T / S,  T = sum_j exp(x_j - m) (x_j - m)   (two sums of one sign each:
//   nothing cancels)
//
// A logit of -inf has no probability: it adds nothing to S and T and is no alternative.  A row of nothing else is told by
// m = -inf; a NaN or +inf makes S, and with it every result of the row, NaN.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "bof4_device.h"

namespace bof4 {

constexpr uint32_t LOGPROBS_MAX_TOP = 64;

template <bool BF16>
__device__ __forceinline__ float load_logit(const void* p, uint64_t i) {
    if constexpr (BF16) return bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p)[i]);
    else return reinterpret_cast<const float*>(p)[i];
}

// m, S and T of a part of a row.  u = x - m is kept above -1e30 where it is a factor only, so that a logit without
// probability (e = 0, u = -inf) adds 0 and not NaN to T.
struct RowSums {
    float m, s, t;
};
constexpr float LOG2_E = 1.44269504088896340736f;
__device__ __forceinline__ float logprobs_exp(float u) { return __builtin_amdgcn_exp2f(u * LOG2_E); }
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }  // a maximum to subtract
__device__ __forceinline__ RowSums merge_sums(RowSums a, RowSums b) {
    const float m = fmaxf(a.m, b.m), ms = finite_max(m);
    const float ua = a.m - ms, ub = b.m - ms, fa = logprobs_exp(ua), fb = logprobs_exp(ub);
    return {m, a.s * fa + b.s * fb,
            fa * fmaf(a.s, fmaxf(ua, -1e30f), a.t) + fb * fmaf(b.s, fmaxf(ub, -1e30f), b.t)};
}

// A logit and its id as one number: larger is the larger logit, then the lower id.  0 is less than any.
__device__ __forceinline__ uint64_t logit_key(float x, uint32_t id) {
    const uint32_t b = __float_as_uint(x + 0.0f);  // (-0 and +0 are equal)
    const uint32_t ordered = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    return ((uint64_t)ordered << 32) | (0xffffffffu - id);
}
__device__ __forceinline__ float key_logit(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ uint32_t key_id(uint64_t key) { return 0xffffffffu - (uint32_t)key; }
// an alternative: neither NaN nor without probability
__device__ __forceinline__ bool is_alternative(float x) { return x > -INFINITY; }

struct LogprobsArgs {
    const void* logits;
    uint64_t ld;
    uint32_t n_rows, vocab, top;
    const int64_t* target;
    float *logprob, *entropy, *top_logprob, *stats;
    int64_t* top_idx;
};

// What one row answers, from its sums (every thread of the workgroup's first wave calls it; tops: its sorted keys, one a lane).
template <bool BF16>
__device__ __forceinline__ void finish_row(const LogprobsArgs& a, uint32_t row, RowSums r, uint64_t key, uint32_t lane) {
    const bool nothing = r.m == -INFINITY && r.s == 0.0f;
    const float log_s = nothing ? 0.0f : logf(r.s);
    if (lane == 0) {
        if (a.logprob) {
            const int64_t t = a.target[row];
            float lp = 0.0f;
            if (t >= 0 && t < (int64_t)a.vocab) {
                const float x = load_logit<BF16>(a.logits, (uint64_t)row * a.ld + (uint64_t)t);
                lp = nothing ? -INFINITY : (x - r.m) - log_s;
            }
            a.logprob[row] = lp;
        }
        if (a.entropy) a.entropy[row] = nothing ? 0.0f : log_s - r.t / r.s;
        if (a.stats) {
            a.stats[2 * (uint64_t)row] = r.m;
            a.stats[2 * (uint64_t)row + 1] = log_s;
        }
    }
    if (lane < a.top) {
        const uint64_t at = (uint64_t)row * a.top + lane;
        const bool is_nan = r.s != r.s;
        a.top_idx[at] = key == 0 || is_nan ? -1 : (int64_t)key_id(key);
        a.top_logprob[at] = is_nan ? r.s : key == 0 ? -INFINITY : (key_logit(key) - r.m) - log_s;
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void logprobs_kernel(LogprobsArgs a) {
    __shared__ RowSums sums[256];
    __shared__ uint64_t best[256];
    const uint32_t tid = threadIdx.x, row = blockIdx.x;
    const uint64_t base = (uint64_t)row * a.ld;
    RowSums r = {-INFINITY, 0.0f, 0.0f};
    for (uint32_t j = tid; j < a.vocab; j += 256) r = merge_sums(r, {load_logit<BF16>(a.logits, base + j), 1.0f, 0.0f});
    sums[tid] = r;
    for (uint32_t half = 128; half > 0; half >>= 1) {
        __syncthreads();
        if (tid < half) sums[tid] = merge_sums(sums[tid], sums[tid + half]);
    }
    uint64_t mine = 0, last = ~0ull;
    for (uint32_t k = 0; k < a.top; ++k) {
        uint64_t b = 0;
        for (uint32_t j = tid; j < a.vocab; j += 256) {
            const float x = load_logit<BF16>(a.logits, base + j);
            const uint64_t key = is_alternative(x) ? logit_key(x, j) : 0;
            if (key < last && key > b) b = key;
        }
        __syncthreads();
        best[tid] = b;
        for (uint32_t half = 128; half > 0; half >>= 1) {
            __syncthreads();
            if (tid < half && best[tid + half] > best[tid]) best[tid] = best[tid + half];
        }
        __syncthreads();
        last = best[0];
        if (tid == k) mine = last;
    }
    __syncthreads();
    if (tid < 64) finish_row<BF16>(a, row, sums[0], mine, tid);
}

// d x_j = g (delta_jt - p_j) - h p_j (log p_j + H), g and h the gradients of the row's log probability and entropy.  One
// thread per four logits of a row.
struct LogprobsGradArgs {
    const void* logits;
    void* out;
    uint64_t ld, ld_out;
    uint32_t n_rows, vocab;
    const int64_t* target;
    const float *stats, *d_logprob, *entropy, *d_entropy;
};
template <bool BF16, bool OUT_BF16>
__global__ __launch_bounds__(256) void logprobs_grad_kernel(LogprobsGradArgs a) {
    const uint32_t row = blockIdx.x;
    const float m = a.stats[2 * (uint64_t)row], log_s = a.stats[2 * (uint64_t)row + 1];
    const int64_t t = a.target ? a.target[row] : -1;
    const bool asked = t >= 0 && t < (int64_t)a.vocab;
    const float g = asked && a.d_logprob ? a.d_logprob[row] : 0.0f;
    const float h = a.d_entropy ? a.d_entropy[row] : 0.0f, H = a.d_entropy ? a.entropy[row] : 0.0f;
    const bool nothing = m == -INFINITY && log_s == 0.0f;
    for (uint32_t j = blockIdx.y * 256 + threadIdx.x; j < a.vocab; j += gridDim.y * 256) {
        const float lp = (load_logit<BF16>(a.logits, (uint64_t)row * a.ld + j) - finite_max(m)) - log_s;
        const float p = logprobs_exp(lp);
        float d = -p * fmaf(h, fmaxf(lp, -1e30f) + H, g);
        if (asked && j == (uint32_t)t) d += g;
        if (nothing) d = 0.0f;
        if constexpr (OUT_BF16) reinterpret_cast<uint16_t*>(a.out)[(uint64_t)row * a.ld_out + j] = (uint16_t)f32_to_bf16_rne(d);
        else reinterpret_cast<float*>(a.out)[(uint64_t)row * a.ld_out + j] = d;
    }
}

}  // namespace bof4
