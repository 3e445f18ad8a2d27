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
#include "bof4_logprobs_plan.h"

namespace bof4 {

constexpr uint32_t LOGPROBS_MAX_TOP = 64;

template <bool BF16>
__device__ __forceinline__ float load_logit(const void* p, uint64_t i) {
    if constexpr (BF16) return bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p)[i]);
    else return reinterpret_cast<const float*>(p)[i];
}

// m, S and T of a part of a row.  Where u = x - m is a factor next to its exponential (0 below -104) it is kept above -1e4, so that
// a logit without probability (u = -inf) or far below the others adds 0 and neither NaN nor an overflow.
constexpr float LOGPROBS_FAR = -1e4f;
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
            fa * fmaf(a.s, fmaxf(ua, LOGPROBS_FAR), a.t) + fb * fmaf(b.s, fmaxf(ub, LOGPROBS_FAR), b.t)};
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
            a.stats[2 * (uint64_t)row] = r.s != r.s ? r.s : r.m;  // (the maximum passes NaN over)
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

// ------------------------------------------------------------------------------------------------ the largest keys
// The 64 lanes' values exchanged between lanes whose numbers differ in bit D.
template <int D>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
    const int x = (int)v;
    if constexpr (D == 1) return (uint32_t)__builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, true);   // quad_perm 1 0 3 2
    if constexpr (D == 2) return (uint32_t)__builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, true);   // quad_perm 2 3 0 1
    if constexpr (D == 4)  // mirrored in eights, then in fours
        return (uint32_t)__builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true);
    if constexpr (D == 8) return (uint32_t)__builtin_amdgcn_mov_dpp(x, 0x128, 0xf, 0xf, true);  // rotated by 8 of 16
    if constexpr (D == 16) {  // one copy's odd rows of 16 lanes against the other's even ones: rows 0 0 2 2 and 1 1 3 3
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return (__lane_id() & 16u) ? r[0] : r[1];
    }
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);  // the lower half twice and the upper half twice
    return (__lane_id() & 32u) ? r[0] : r[1];
}
template <int D>
__device__ __forceinline__ uint64_t lane_xor64(uint64_t v) {
    return ((uint64_t)lane_xor<D>((uint32_t)(v >> 32)) << 32) | lane_xor<D>((uint32_t)v);
}
// One step of a bitonic network: the larger of a pair goes to the lower lane where `down`.
template <int D>
__device__ __forceinline__ uint64_t exchange(uint64_t v, uint32_t lane, bool down) {
    const uint64_t o = lane_xor64<D>(v);
    return ((lane & D) == 0u) == down ? (v > o ? v : o) : (v > o ? o : v);
}
// Descending order over the lanes of what is already a bitonic sequence of SIZE lanes each.
template <int SIZE>
__device__ __forceinline__ uint64_t bitonic_merge(uint64_t v, uint32_t lane, bool down) {
    if constexpr (SIZE >= 64) v = exchange<32>(v, lane, down);
    if constexpr (SIZE >= 32) v = exchange<16>(v, lane, down);
    if constexpr (SIZE >= 16) v = exchange<8>(v, lane, down);
    if constexpr (SIZE >= 8) v = exchange<4>(v, lane, down);
    if constexpr (SIZE >= 4) v = exchange<2>(v, lane, down);
    return exchange<1>(v, lane, down);
}
__device__ __forceinline__ uint64_t sort_ascending(uint64_t v, uint32_t lane) {
    v = bitonic_merge<2>(v, lane, (lane & 2u) == 0u);
    v = bitonic_merge<4>(v, lane, (lane & 4u) == 0u);
    v = bitonic_merge<8>(v, lane, (lane & 8u) == 0u);
    v = bitonic_merge<16>(v, lane, (lane & 16u) == 0u);
    v = bitonic_merge<32>(v, lane, (lane & 32u) == 0u);
    return bitonic_merge<64>(v, lane, false);
}
// The 64 largest of a descending and an ascending sequence, descending.
__device__ __forceinline__ uint64_t merge_ascending(uint64_t list, uint64_t ascending, uint32_t lane) {
    return bitonic_merge<64>(list > ascending ? list : ascending, lane, true);
}
template <int D>
__device__ __forceinline__ uint64_t larger_of_pair(uint64_t v) {
    const uint64_t o = lane_xor64<D>(v);
    return v > o ? v : o;
}
__device__ __forceinline__ uint64_t largest_lane(uint64_t v) {  // in every lane
    return larger_of_pair<32>(larger_of_pair<16>(larger_of_pair<8>(larger_of_pair<4>(larger_of_pair<2>(larger_of_pair<1>(v))))));
}
__device__ __forceinline__ uint64_t readlane64(uint64_t v, uint32_t lane) {
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), (int)lane) << 32) |
           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, (int)lane);
}

// ------------------------------------------------------------------------------------------------ a row's pass
// One pass over the logits.  A wave takes tiles of 256 16-byte words, four to a lane (the next tile's on their way
// meanwhile), and keeps m, S and T per lane: the maximum moves at most once per tile, and per logit there are a
// subtraction, an exponential and three more operations.  The lanes and waves join at the end of the row.
//   The alternatives ride along: a wave knows a bound that its `top` best so far all reach, and only a tile in which some
// lane's maximum reaches it is looked at again.  Then the tile is parked in LDS, what reaches the bound is collected (as
// keys that no two logits share) and, 64 at a time, sorted and merged into the wave's sorted list, one key to a lane.
// Before a tile with many such lanes is collected the bound is raised to what at least `top` lanes' maxima reach (their
// highest 16 bits, by bisection), so that the first tile does not bring a thousand candidates.  Every element that is
// left out is smaller than `top` others, so the result does not depend on how the row was cut.
//   With few rows a row is cut into n_splits parts, one per workgroup, whose records logprobs_join_kernel joins.
struct LogprobsPart {  // what a part of a row leaves: its sums, then `top` keys
    RowSums r;
    uint32_t unused;
};
__device__ __forceinline__ LogprobsPart* logprobs_part(char* ws, uint64_t at, uint32_t top) {
    return reinterpret_cast<LogprobsPart*>(ws + at * (sizeof(LogprobsPart) + 8ull * top));
}

template <int D>
__device__ __forceinline__ RowSums join_step(RowSums r) {
    const RowSums o = {__uint_as_float(lane_xor<D>(__float_as_uint(r.m))), __uint_as_float(lane_xor<D>(__float_as_uint(r.s))),
                       __uint_as_float(lane_xor<D>(__float_as_uint(r.t)))};
    return merge_sums(r, o);
}
// All lanes' sums joined, as the first lane has them, in every lane.
__device__ __forceinline__ RowSums join_lanes(RowSums r) {
    r = join_step<32>(join_step<16>(join_step<8>(join_step<4>(join_step<2>(join_step<1>(r))))));
    return {__uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(r.m))),
            __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(r.s))),
            __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(r.t)))};
}

template <bool BF16, uint32_t WAVES>
__global__ __launch_bounds__(64 * WAVES) void logprobs_kernel(LogprobsArgs a, uint32_t n_splits,
                                                                       uint32_t tiles_per_split, char* ws) {
    constexpr uint32_t PER_WORD = logprobs_word_elements(BF16), SIZE = BF16 ? 2 : 4;
    struct Shared {
        uint4 tile[WAVES][LOGPROBS_TILE];
        uint64_t found[WAVES][128];
        uint64_t list[WAVES][64];
        RowSums sums[WAVES];
        uint32_t n_found[WAVES], has_list[WAVES];
    };
    __shared__ __attribute__((aligned(16))) Shared sh;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t row = blockIdx.x / n_splits, split = blockIdx.x - row * n_splits;
    // The row in 16-byte words of memory: the first and the last may hold logits of other rows or none, and only
    // the row's own are read of those two.
    const char* row_ptr = static_cast<const char*>(a.logits) + (uint64_t)row * a.ld * SIZE;
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(row_ptr) & 15u) / SIZE;  // logits in front of the row's first
    const char* words = row_ptr - off * SIZE;
    const uint32_t end = off + a.vocab, n_words = (end + PER_WORD - 1) / PER_WORD;
    const uint32_t n_tiles = (n_words + LOGPROBS_TILE - 1) / LOGPROBS_TILE;
    const uint32_t tile0 = split * tiles_per_split, tile1 = min(n_tiles, tile0 + tiles_per_split);

    struct Tile {
        uint4 q[LOGPROBS_WORDS];
    };
    auto fetch = [&](uint32_t tile) __attribute__((always_inline)) {
        Tile t;
        const uint32_t w0 = tile * LOGPROBS_TILE + lane;
        if (tile > 0 && (tile + 1) * LOGPROBS_TILE * PER_WORD <= end) {  // whole words only
#pragma unroll
            for (uint32_t k = 0; k < LOGPROBS_WORDS; ++k) t.q[k] = load_stream(reinterpret_cast<const uint4*>(words) + w0 + 64 * k);
            return t;
        }
        constexpr uint32_t NONE = BF16 ? 0xff80ff80u : 0xff800000u;  // -inf
#pragma unroll
        for (uint32_t k = 0; k < LOGPROBS_WORDS; ++k) {
            const uint32_t w = w0 + 64 * k, first = w * PER_WORD;
            if (first >= off && first + PER_WORD <= end) {
                t.q[k] = reinterpret_cast<const uint4*>(words)[w];
                continue;
            }
            uint32_t v[4] = {NONE, NONE, NONE, NONE};
#pragma unroll
            for (uint32_t i = 0; i < PER_WORD; ++i) {
                if (first + i < off || first + i >= end) continue;
                if constexpr (BF16) {
                    const uint32_t x = reinterpret_cast<const uint16_t*>(words)[first + i];
                    v[i / 2] = i % 2 ? (v[i / 2] & 0xffffu) | (x << 16) : (v[i / 2] & 0xffff0000u) | x;
                } else {
                    v[i] = reinterpret_cast<const uint32_t*>(words)[first + i];
                }
            }
            t.q[k] = make_uint4(v[0], v[1], v[2], v[3]);
        }
        return t;
    };

    float m = -INFINITY, s0 = 0.0f, s1 = 0.0f, t0 = 0.0f, t1 = 0.0f;
    uint64_t list = 0;                     // the wave's best, descending over the lanes
    // What a logit has to reach to be an alternative: at first the lowest number, which -inf and NaN do not.
    float bound = -3.4028234663852886e38f;
    float last_of_list = bound;             // the `top`-th best so far
    uint32_t n_found = 0;
    uint64_t* found = sh.found[wave];
    auto drain = [&]() {  // the first 64 of what was collected go into the list
        wave_lds_fence();
        const uint64_t v = lane < n_found ? found[lane] : 0;
        const uint64_t rest = 64 + lane < n_found ? found[64 + lane] : 0;
        wave_lds_fence();
        if (64 + lane < n_found) found[lane] = rest;
        n_found = n_found > 64 ? n_found - 64 : 0;
        if (a.top == 1) {
            const uint64_t best = largest_lane(list > v ? list : v);
            list = lane == 0 ? best : 0;
        } else {
            list = merge_ascending(list, sort_ascending(v, lane), lane);
        }
        const uint64_t last = readlane64(list, a.top - 1);
        if (last != 0) {
            last_of_list = key_logit(last);
            bound = fmaxf(bound, key_logit(last + (1ull << 32)));  // more than that: what comes later has a higher id
        }
    };
    auto collect = [&](const Tile& t, const float* x, uint32_t tile, float lane_max, uint64_t reach) {
        if (__popcll(reach) > a.top) {  // what `top` lanes' maxima reach, in their highest 16 bits
            const uint32_t key = lane_max >= bound ? (uint32_t)(logit_key(lane_max, 0) >> 48) : 0u;
            uint32_t b = 0;
            for (uint32_t bit = 0x8000u; bit != 0; bit >>= 1)
                if ((uint32_t)__popcll(__builtin_amdgcn_ballot_w64(key >= (b | bit))) >= a.top) b |= bit;
            bound = fmaxf(bound, key_logit((uint64_t)b << 48));
        }
        uint32_t bits = 0;  // which of the lane's logits reach it
#pragma unroll
        for (uint32_t i = 0; i < LOGPROBS_WORDS * PER_WORD; ++i) bits |= x[i] >= bound ? 1u << i : 0u;
        float least = bound;
        uint4* parked = sh.tile[wave];
#pragma unroll
        for (uint32_t k = 0; k < LOGPROBS_WORDS; ++k) parked[64 * k + lane] = t.q[k];
        wave_lds_fence();
        for (uint64_t mask = __builtin_amdgcn_ballot_w64(bits != 0u); mask != 0; mask = __builtin_amdgcn_ballot_w64(bits != 0u)) {
            const uint32_t i = logprobs_lowest(bits, PER_WORD), at_word = logprobs_tile_word(i, lane, PER_WORD);
            const float v = load_logit<BF16>(parked, at_word * PER_WORD + i % PER_WORD);
            const uint32_t place = n_found + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
            if (bits != 0u) found[place] = logit_key(v, (tile * LOGPROBS_TILE + at_word) * PER_WORD + i % PER_WORD - off);
            bits &= bits - 1u;
            n_found += (uint32_t)__popcll(mask);
            if (n_found >= 64) {
                drain();
                if (last_of_list > least) {  // (an equal one with a lower id may follow within the tile)
                    least = last_of_list;
                    uint32_t still = 0;
#pragma unroll
                    for (uint32_t j = 0; j < LOGPROBS_WORDS * PER_WORD; ++j) still |= x[j] >= least ? 1u << j : 0u;
                    bits &= still;
                }
            }
        }
        wave_lds_fence();
    };
    auto add = [&](const Tile& t, uint32_t tile) __attribute__((always_inline)) {
        float x[LOGPROBS_WORDS * PER_WORD];
#pragma unroll
        for (uint32_t k = 0; k < LOGPROBS_WORDS; ++k) {
            const uint32_t w[4] = {t.q[k].x, t.q[k].y, t.q[k].z, t.q[k].w};
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                if constexpr (BF16) {
                    x[8 * k + 2 * i] = __uint_as_float(w[i] << 16);
                    x[8 * k + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                } else {
                    x[4 * k + i] = __uint_as_float(w[i]);
                }
            }
        }
        float lane_max = x[0];
#pragma unroll
        for (uint32_t i = 1; i < LOGPROBS_WORDS * PER_WORD; ++i) lane_max = fmaxf(lane_max, x[i]);
        const float m_new = fmaxf(m, lane_max), ms = finite_max(m_new);
        const float moved = m - ms, f = logprobs_exp(moved), moved_f = fmaxf(moved, LOGPROBS_FAR);
        t0 = f * fmaf(s0, moved_f, t0);
        t1 = f * fmaf(s1, moved_f, t1);
        s0 *= f;
        s1 *= f;
        m = m_new;
#pragma unroll
        for (uint32_t i = 0; i < LOGPROBS_WORDS * PER_WORD; i += 2) {
            const float u0 = x[i] - ms, u1 = x[i + 1] - ms, e0 = logprobs_exp(u0), e1 = logprobs_exp(u1);
            s0 += e0;
            s1 += e1;
            t0 = fmaf(e0, fmaxf(u0, LOGPROBS_FAR), t0);
            t1 = fmaf(e1, fmaxf(u1, LOGPROBS_FAR), t1);
        }
        if (a.top > 0) {
            const uint64_t reach = __builtin_amdgcn_ballot_w64(lane_max >= bound);
            if (reach != 0) collect(t, x, tile, lane_max, reach);
        }
    };
    uint32_t tile = tile0 + wave;
    if (tile < tile1) {
        Tile now = fetch(tile);
        for (; tile < tile1; tile += WAVES) {
            Tile next = now;
            if (tile + WAVES < tile1) next = fetch(tile + WAVES);
            __builtin_amdgcn_sched_barrier(0);
            add(now, tile);
            now = next;
        }
    }
    // lanes, then waves, in a fixed order; what the waves collected and did not sort yet is sorted together
    RowSums r = join_lanes({m, s0 + s1, t0 + t1});
    if (lane == 0) sh.sums[wave] = r;
    if (a.top > 0) {
        const bool has_list = readlane64(list, 0) != 0;
        if (a.top == 1) {
            wave_lds_fence();
            const uint64_t v = lane < n_found ? found[lane] : 0;
            list = largest_lane(list > v ? list : v);
            if (lane == 0) sh.list[wave][0] = list;
        } else {
            if (has_list) sh.list[wave][lane] = list;
            if (lane == 0) {
                sh.n_found[wave] = n_found;
                sh.has_list[wave] = has_list ? 1u : 0u;
            }
        }
    }
    if (WAVES > 1) __syncthreads();
    if (wave != 0) return;
    for (uint32_t w = 1; w < WAVES; ++w) r = merge_sums(r, sh.sums[w]);
    if (a.top == 1) {
        for (uint32_t w = 1; w < WAVES; ++w) list = list > sh.list[w][0] ? list : sh.list[w][0];
    } else if (a.top > 0) {
        uint32_t total = 0, before[WAVES];
#pragma unroll
        for (uint32_t w = 0; w < WAVES; ++w) {
            if (w > 0 && sh.has_list[w]) list = merge_ascending(list, sh.list[w][63 - lane], lane);
            before[w] = total;
            total += sh.n_found[w];
        }
        for (uint32_t i0 = 0; i0 < total; i0 += 64) {
            const uint32_t i = i0 + lane;
            uint64_t v = 0;
#pragma unroll
            for (uint32_t w = 0; w < WAVES; ++w)
                if (i >= before[w] && i < (w + 1 < WAVES ? before[w + 1] : total)) v = sh.found[w][i - before[w]];
            list = merge_ascending(list, sort_ascending(v, lane), lane);
        }
    }
    if (n_splits == 1) {
        finish_row<BF16>(a, row, r, list, lane);
        return;
    }
    LogprobsPart* part = logprobs_part(ws, blockIdx.x, a.top);
    if (lane == 0) part->r = r;
    if (lane < a.top) reinterpret_cast<uint64_t*>(part + 1)[lane] = list;
}

// A row from the records of its parts, in their order: one workgroup per row, whose waves take up to four parts each and
// then merge their lists in pairs.
template <bool BF16>
__global__ __launch_bounds__(64 * LOGPROBS_JOIN_WAVES) void logprobs_join_kernel(LogprobsArgs a, uint32_t n_splits, char* ws) {
    static_assert(LOGPROBS_MAX_SPLITS <= 4 * LOGPROBS_JOIN_WAVES && LOGPROBS_MAX_SPLITS <= 64, "one part's sums per lane");
    __shared__ uint64_t lists[LOGPROBS_JOIN_WAVES][64];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n_waves = blockDim.x >> 6;
    const uint32_t row = blockIdx.x;
    const uint64_t first = (uint64_t)row * n_splits;
    RowSums r = {-INFINITY, 0.0f, 0.0f};
    if (wave == 0 && lane < n_splits) r = logprobs_part(ws, first + lane, a.top)->r;
    uint64_t list = 0;
    if (a.top == 1) {  // (one wave)
        list = largest_lane(lane < n_splits ? *reinterpret_cast<const uint64_t*>(logprobs_part(ws, first + lane, 1) + 1) : 0);
    } else if (a.top > 0) {
        uint64_t keys[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t p = wave + i * n_waves, at = i == 0 ? lane : 63 - lane;
            keys[i] = p < n_splits && at < a.top ? reinterpret_cast<const uint64_t*>(logprobs_part(ws, first + p, a.top) + 1)[at] : 0;
        }
        list = keys[0];
#pragma unroll
        for (uint32_t i = 1; i < 4; ++i)
            if (wave + i * n_waves < n_splits) list = merge_ascending(list, keys[i], lane);
        for (uint32_t half = n_waves / 2; half > 0; half /= 2) {
            if (wave >= half && wave < 2 * half) lists[wave][lane] = list;
            __syncthreads();
            if (wave < half) list = merge_ascending(list, lists[wave + half][63 - lane], lane);
        }
    }
    if (wave != 0) return;
    finish_row<BF16>(a, row, join_lanes(r), list, lane);
}

// d x_j = g (delta_jt - p_j) - h p_j (log p_j + H), g and h the gradients of the row's log probability and entropy: read
// once, written once.  A workgroup takes a stretch of a row, in 16-byte words of the logits as they lie in memory.
struct LogprobsGradArgs {
    const void* logits;
    void* out;
    uint64_t ld, ld_out;
    uint32_t n_rows, vocab;
    const int64_t* target;
    const float *stats, *d_logprob, *entropy, *d_entropy;
};
// Eight logits per thread: one word of bfloat16, two of binary32 (2000 x 32000, one / two / four words: bfloat16 42 / 45 / 49 us,
// binary32 to bfloat16 67 / 65 / 66).
constexpr uint32_t logprobs_grad_words(bool bf16) { return bf16 ? 1 : 2; }
constexpr uint32_t LOGPROBS_GRAD_STRETCH = 256 * 8;  // logits per workgroup
template <bool BF16, bool OUT_BF16, bool ENTROPY>
__global__ __launch_bounds__(256) void logprobs_grad_kernel(LogprobsGradArgs a, uint32_t stretches) {
    constexpr uint32_t PER_WORD = logprobs_word_elements(BF16), SIZE = BF16 ? 2 : 4, OUT_SIZE = OUT_BF16 ? 2 : 4;
    constexpr uint32_t WORDS = logprobs_grad_words(BF16);
    const uint32_t row = blockIdx.x / stretches, stretch = blockIdx.x - row * stretches;
    const char* row_ptr = static_cast<const char*>(a.logits) + (uint64_t)row * a.ld * SIZE;
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(row_ptr) & 15u) / SIZE;
    const char* words = row_ptr - off * SIZE;
    const uint32_t end = off + a.vocab, n_words = (end + PER_WORD - 1) / PER_WORD;
    const uint32_t w0 = stretch * 256 * WORDS + threadIdx.x;
    char* out = static_cast<char*>(a.out) + (uint64_t)row * a.ld_out * OUT_SIZE - (uint64_t)off * OUT_SIZE;
    const float m = a.stats[2 * (uint64_t)row], log_s = a.stats[2 * (uint64_t)row + 1];
    const int64_t t = a.target ? a.target[row] : -1;
    const bool asked = t >= 0 && t < (int64_t)a.vocab;
    const float g = asked ? a.d_logprob[row] : 0.0f;
    const uint32_t target = asked ? off + (uint32_t)t : 0xffffffffu;
    const float h = ENTROPY ? a.d_entropy[row] : 0.0f, H = ENTROPY ? a.entropy[row] : 0.0f;
    const bool nothing = m == -INFINITY && log_s == 0.0f;
    const float ms = finite_max(m);
    auto slope = [&](float x) __attribute__((always_inline)) {
        const float lp = (x - ms) - log_s, p = logprobs_exp(lp);
        // (p times log p first: with a large h their product is what is finite)
        return ENTROPY ? -fmaf(p * (fmaxf(lp, LOGPROBS_FAR) + H), h, p * g) : -p * g;
    };
    auto one = [&](uint32_t j) {  // j counted from the first word, as `target`
        const float x = load_logit<BF16>(words, j);
        float d = slope(x);
        if (j == target) d += g;
        if (nothing) d = 0.0f;
        if constexpr (OUT_BF16) reinterpret_cast<uint16_t*>(out)[j] = (uint16_t)f32_to_bf16_rne(d);
        else reinterpret_cast<float*>(out)[j] = d;
    };
    uint4 q[WORDS];
    bool whole[WORDS];
#pragma unroll
    for (uint32_t k = 0; k < WORDS; ++k) {
        const uint32_t w = w0 + 256 * k, first = w * PER_WORD;
        whole[k] = w < n_words && first >= off && first + PER_WORD <= end;
        if (whole[k]) q[k] = load_stream(reinterpret_cast<const uint4*>(words) + w);
    }
#pragma unroll
    for (uint32_t k = 0; k < WORDS; ++k) {
        const uint32_t w = w0 + 256 * k, first = w * PER_WORD;
        if (!whole[k]) {
            if (w < n_words)
                for (uint32_t j = first < off ? off : first; j < end && j < first + PER_WORD; ++j) one(j);
            continue;
        }
        const uint32_t v[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
        float d[PER_WORD];
#pragma unroll
        for (uint32_t i = 0; i < PER_WORD; ++i) {
            float x;
            if constexpr (BF16) x = i % 2 ? __uint_as_float(v[i / 2] & 0xffff0000u) : __uint_as_float(v[i / 2] << 16);
            else x = __uint_as_float(v[i]);
            d[i] = nothing ? 0.0f : slope(x);
        }
        if (target - first < PER_WORD) {
#pragma unroll
            for (uint32_t i = 0; i < PER_WORD; ++i)
                if (first + i == target && !nothing) d[i] += g;
        }
        char* to = out + (uint64_t)first * OUT_SIZE;
        if constexpr (OUT_BF16) {
            uint32_t o[PER_WORD / 2];
#pragma unroll
            for (uint32_t i = 0; i < PER_WORD / 2; ++i) o[i] = gemm_pack_bf16(d[2 * i], d[2 * i + 1]);
            if constexpr (PER_WORD == 8) __builtin_nontemporal_store(u32x4_any{o[0], o[1], o[2], o[3]}, reinterpret_cast<u32x4_any*>(to));
            else *reinterpret_cast<u32x2_any*>(to) = u32x2_any{o[0], o[1]};
        } else {
#pragma unroll
            for (uint32_t i = 0; i < PER_WORD; i += 4)
                __builtin_nontemporal_store(u32x4_any{__float_as_uint(d[i]), __float_as_uint(d[i + 1]), __float_as_uint(d[i + 2]),
                                                      __float_as_uint(d[i + 3])}, reinterpret_cast<u32x4_any*>(to) + i / 4);
        }
    }
}

}  // namespace bof4
