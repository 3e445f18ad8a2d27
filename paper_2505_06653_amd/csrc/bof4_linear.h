// bof4_linear.h - the gradients of a linear layer with a quantised matrix (bof4_epilogue.h has the layer's forward side):
//
//   dz = dy * mul * act'(z),   dx = dz W^,   dmul = dy * act(z),   dbias = sum over the tokens of dz.
//
// dx contracts over the rows of W^, so the matrix cores want it turned.  A call works in two steps, as the product for many
// tokens does whose matrix is decoded first: linear_turn_kernel decodes the packed matrix into the operands of W^^T, in
// slabs that stay in the cache behind the L2s, and gemm_decoded_kernel multiplies them with dz.  linear_dz makes dz from dy in the
// order of the operands, and dmul and dbias on the way.
//   The matrix cores take bfloat16, so dz is the sum of one to three bfloat16 terms, each multiplied with the same decoded
// chunk (linear_dz_terms).  dy and dx in bfloat16: one, off by 2^-8 of dz at most, as far as dx's own rounding.
// (dx is then off by 0.0024 of its size where the rounding of the result alone makes 0.0017; a second term would leave just that,
// at 49 us instead of 38 for 4096 x 4096 with 333 tokens and 398 instead of 230 for 11008 x 4096 with 2000.)  dx in bfloat16 from
// binary32 dy: two, off by 2^-16.  dx in binary32: three, which hold all 24 bits (59 and 555 us), or as few as hold dz.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "bof4_epilogue.h"
#include "bof4_gemm.h"

namespace bof4 {

struct LinearGradArgs {
    const void *dy, *pre, *mul;  // pre, mul null: not there (pre is there where act or dmul asks for it)
    void* dmul;                  // null: not wanted
    float* dbias_parts;          // null: not wanted
    uint64_t ld_dy, ld_pre, ld_mul, ld_dmul;
    uint32_t act, terms;
    bool dy_bf16, pre_bf16, mul_bf16, dmul_bf16;
};
constexpr uint32_t LINEAR_MOST_TERMS = 3;
inline uint32_t linear_dz_terms(uint32_t act, bool dy_bf16, bool mul, bool mul_bf16, bool dx_bf16) {
    const uint32_t wanted = !dx_bf16 ? 3 : dy_bf16 ? 1 : 2;
    // without a curved activation dz is dy (or 0), or its product with the factor: eight bits times eight are sixteen
    const uint32_t exact = act > ACT_RELU || !dy_bf16 || (mul && !mul_bf16) ? 3 : mul ? 2 : 1;
    return wanted < exact ? wanted : exact;
}

// dz in the products' order (gemm_pack_x_kernel's, rows in the place of columns, a chunk's terms behind each other): a workgroup
// takes a chunk of 64 rows and `tiles_per_range` tiles of 32 tokens, eight threads per token, which read 128 consecutive bytes and write 16-byte words of
// which eight neighbouring tokens make up 128.  Bound by memory: 2000 tokens x 11008 rows with factor, activation and dmul, 220
// MB, 44 us (5.0 TB/s; with 8-byte accesses 55).
constexpr uint32_t LINEAR_MOST_RANGES = 64;  // parts of dbias at most
typedef float LinearDzSums[32][65];
__device__ __forceinline__ void linear_dz(uint32_t chunk, uint32_t range, LinearDzSums& sums, const LinearGradArgs& a,
                                          uint32_t n_tokens, uint32_t rows, uint32_t n_chunks, uint32_t tok_tiles,
                                          uint32_t tiles_per_range, uint4* __restrict__ xp) {
    const uint32_t tid = threadIdx.x, word = tid & 7, token_in_tile = tid >> 3;
    const uint32_t row = chunk * GEMM_CHUNK + 8 * word;
    float bias[8] = {};
    const uint32_t tile1 = min(tok_tiles, (range + 1) * tiles_per_range);
    for (uint32_t tile = range * tiles_per_range; tile < tile1; ++tile) {
        const uint64_t t = tile * GEMM_TOKENS + token_in_tile;
        float dy[8] = {};
        if (t < n_tokens && row < rows) {
            const uint32_t n = rows - row;
            float z[8] = {}, f[8], value, slope;
            load_row<8>(a.dy, t * a.ld_dy + row, a.dy_bf16, n, dy);
            if (a.pre) load_row<8>(a.pre, t * a.ld_pre + row, a.pre_bf16, n, z);
            if (a.mul) load_row<8>(a.mul, t * a.ld_mul + row, a.mul_bf16, n, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                activation_slope(a.act, z[i], value, slope);
                z[i] = value * dy[i];
                if (a.mul) dy[i] *= f[i];
                if (a.act != ACT_NONE) dy[i] *= slope;
                if ((uint32_t)i >= n) dy[i] = 0.0f;
                bias[i] += dy[i];
            }
            if (a.dmul) store_row<8>(a.dmul, t * a.ld_dmul + row, a.dmul_bf16, n, z);
        }
        uint4* to = xp + ((uint64_t)tile * n_chunks + chunk) * a.terms * GEMM_TILE_WORDS + (word & 3) * 64 + (word >> 2) * 32 + token_in_tile;
        for (uint32_t term = 0;;) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = gemm_pack_bf16(dy[2 * i], dy[2 * i + 1]);
            to[term * GEMM_TILE_WORDS] = make_uint4(w[0], w[1], w[2], w[3]);
            if (++term == a.terms) break;
#pragma unroll
            for (int i = 0; i < 8; ++i) {  // what the term leaves; nothing where it is not finite
                const float rounded = __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
                dy[i] = fabsf(rounded) < INFINITY ? dy[i] - rounded : 0.0f;
            }
        }
    }
    if (!a.dbias_parts) return;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) sums[token_in_tile][8 * word + i] = bias[i];
    __syncthreads();
    if (tid < GEMM_CHUNK && chunk * GEMM_CHUNK + tid < rows) {
        float s = 0.0f;
        for (uint32_t k = 0; k < 32; ++k) s += sums[k][tid];
        a.dbias_parts[(uint64_t)range * rows + chunk * GEMM_CHUNK + tid] = s;
    }
}
__device__ __forceinline__ void linear_dbias(uint32_t group, const float* __restrict__ parts, uint32_t n_parts, uint32_t rows,
                                             float* __restrict__ dbias) {
    const uint32_t row = group * 256 + threadIdx.x;
    if (row >= rows) return;
    double s = 0.0;
#pragma unroll 8
    for (uint32_t k = 0; k < n_parts; ++k) s += parts[(uint64_t)k * rows + row];
    dbias[row] = (float)s;
}
__global__ __launch_bounds__(256) void linear_dbias_kernel(const float* __restrict__ parts, uint32_t n_parts, uint32_t rows,
                                                           float* __restrict__ dbias) {
    linear_dbias(blockIdx.x, parts, n_parts, rows, dbias);
}

__global__ __launch_bounds__(256) void linear_dz_kernel(LinearGradArgs a, uint32_t n_tokens, uint32_t rows, uint32_t n_chunks,
                                                        uint32_t tok_tiles, uint32_t tiles_per_range, uint4* __restrict__ xp) {
    __shared__ LinearDzSums sums;
    linear_dz(blockIdx.x, blockIdx.y, sums, a, n_tokens, rows, n_chunks, tok_tiles, tiles_per_range, xp);
}

// W^^T in the order of the operands: 4096-byte tiles of 32 columns x 64 rows, from the packed tiles of 32 rows x 64 columns.
// A wave turns 64 rows x 64 columns: it decodes as gemm_decode_kernel does (lane = row, 32 columns), puts neighbouring rows
// of a column together with its neighbour lane (one lane exchange and one byte permutation per two weights), parks the
// pairs in LDS by column, writes the tiles' list entries over their placeholders there and reads eight rows of a column at
// a time.  A column takes LINEAR_TURN_LD bytes, so that sixteen lanes' 16-byte reads fall into different banks.  Bound by the
// look-ups and LDS traffic next to memory: 45 M weights in 24 us with a list, 16 M in 8 us without (gemm_decode_kernel, which turns
// nothing, 19.5 and 7).
constexpr uint32_t LINEAR_TURN_WAVES = 4, LINEAR_TURN_LD = 144;
//   For small dz the first launch of a call makes it as well: dz_groups workgroups, dealt out among the others, so that the one's memory
// accesses and the other's look-ups and LDS traffic overlap.
struct LinearDzCall {
    LinearGradArgs a;
    uint32_t dz_groups, n_tokens, rows, tok_tiles, tiles_per_range;
    uint4* xp;
};
template <bool OUTLIERS>
__global__ __launch_bounds__(64 * LINEAR_TURN_WAVES) void linear_turn_kernel(
    const char* __restrict__ packed, uint32_t first_ct, uint32_t n_ct, uint32_t n_chunks, uint32_t row_chunks, CodebookArgs cb,
    const uint32_t* __restrict__ list_ptr, const uint32_t* __restrict__ entries, uint32_t n_out, GemmListGeometry lg,
    uint32_t row_tiles, uint4* __restrict__ decoded, LinearDzCall dz) {
    struct Turn {
        float tab[16];
        uint4 turned[LINEAR_TURN_WAVES][64 * LINEAR_TURN_LD / 16];
    };
    __shared__ __attribute__((aligned(16))) union {
        Turn turn;
        LinearDzSums sums;
    } shared;
    uint32_t group = blockIdx.x;
    if (gemm_deal(group, dz.dz_groups, gridDim.x)) {
        linear_dz(group % row_chunks, group / row_chunks, shared.sums, dz.a, dz.n_tokens, dz.rows, row_chunks, dz.tok_tiles,
                  dz.tiles_per_range, dz.xp);
        return;
    }
    Turn& sh = shared.turn;
    const uint32_t tid = threadIdx.x, lane = tid & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (tid < 16) sh.tab[tid] = cb.lv32[tid];
    __syncthreads();
    const char* tab = reinterpret_cast<const char*>(sh.tab);
    const uint64_t job = (uint64_t)group * LINEAR_TURN_WAVES + wave;
    if (job >= (uint64_t)((n_ct + 1) / 2) * row_chunks) return;
    const uint32_t ct_local = 2 * (uint32_t)(job / row_chunks), rc = (uint32_t)(job % row_chunks);
    const uint32_t ch = (first_ct + ct_local) / 2;  // (first_ct is even)
    uint4 q[2];
    uint16_t m[2];
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
        const char* tile = packed + ((uint64_t)(2 * rc + k) * n_chunks + ch) * GEMM_TILE_BYTES;
        q[k] = load_stream(reinterpret_cast<const uint4*>(tile) + lane);
        m[k] = __builtin_nontemporal_load(reinterpret_cast<const uint16_t*>(tile + 1024) + lane);
    }
    uint32_t lo[2] = {}, n_en[2] = {};
    if (OUTLIERS) {
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {
            if (2 * rc + k >= row_tiles) continue;  // wave-uniform
            uint32_t hi;
            gemm_list_range(list_ptr + (uint64_t)(2 * rc + k) * lg.n_groups + (ch >> lg.log2_group), n_out, lg.log2_group, lo[k], hi);
            n_en[k] = hi - lo[k];
        }
    }
    char* turned = reinterpret_cast<char*>(sh.turned[wave]);
    const uint32_t odd = lane & 1u, pick = odd ? 0x03020706u : 0x05040100u;
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
        const float msc = f16_bits_to_f32(m[k]);
        const uint32_t w[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
        // the lane's pair of rows; even lanes keep the even columns, odd lanes the odd ones
        char* at = turned + (32 * (lane >> 5) + odd) * LINEAR_TURN_LD + (16 * k + ((lane & 31u) >> 1)) * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t even = (w[j] << 2) & 0x3c3c3c3cu, odds = (w[j] >> 2) & 0x3c3c3c3cu;
            const uint32_t oe[4] = {byte_of<0>(even), byte_of<1>(even), byte_of<2>(even), byte_of<3>(even)};
            const uint32_t oo[4] = {byte_of<0>(odds), byte_of<1>(odds), byte_of<2>(odds), byte_of<3>(odds)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float le = *reinterpret_cast<const float*>(tab + oe[i]);
                const float lv = *reinterpret_cast<const float*>(tab + oo[i]);
                const uint32_t mine = gemm_pack_bf16(msc * le, msc * lv);  // the decoder's product and rounding
                const uint32_t other = (uint32_t)__builtin_amdgcn_mov_dpp((int)mine, 0xb1, 0xf, 0xf, true);  // lane ^ 1
                *reinterpret_cast<uint32_t*>(at + (8 * j + 2 * i) * LINEAR_TURN_LD) = __builtin_amdgcn_perm(other, mine, pick);
            }
        }
    }
    wave_lds_fence();
    if (OUTLIERS) {
        const uint32_t place = ch & ((1u << lg.log2_group) - 1u);
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k)
            for (uint32_t i = lane; i < n_en[k]; i += 64u) {
                const uint32_t e = entries[lo[k] + i], at = (e >> 16) & 2047u;
                if ((e >> 27) != place) continue;
                const uint32_t col = 32 * ((at >> 8) & 1u) + 8 * (at >> 9) + (at & 7u), row = 32 * k + ((at >> 3) & 31u);
                *reinterpret_cast<uint16_t*>(turned + col * LINEAR_TURN_LD + 2 * row) = (uint16_t)e;
            }
        wave_lds_fence();
    }
#pragma unroll
    for (uint32_t t = 0; t < 2; ++t) {
        if (ct_local + t >= n_ct) break;  // wave-uniform
        uint4* out = decoded + ((uint64_t)(ct_local + t) * row_chunks + rc) * GEMM_TILE_WORDS + lane;
        const char* from = turned + (32 * t + (lane & 31u)) * LINEAR_TURN_LD + 64 * (lane >> 5);
#pragma unroll
        for (int j = 0; j < 4; ++j) out[64 * j] = *reinterpret_cast<const uint4*>(from + 16 * j);
    }
}

// gemm_sum_layer_kernel for dx (dx_groups workgroups to a token, `step` tokens side by side), and the sums of dbias in
// workgroups of their own behind it.
__global__ __launch_bounds__(256) void linear_sum_kernel(uint32_t n_parts, uint32_t n_tokens, uint32_t cols, LayerOut dst,
                                                         uint32_t dx_groups, uint32_t step, const float* __restrict__ dbias_parts,
                                                         uint32_t n_dbias_parts, uint32_t rows, float* __restrict__ dbias) {
    if (blockIdx.x < dx_groups * step) gemm_sum_layer(blockIdx.x % dx_groups, blockIdx.x / dx_groups, step, n_parts, n_tokens, cols, dst);
    else linear_dbias(blockIdx.x - dx_groups * step, dbias_parts, n_dbias_parts, rows, dbias);
}

}  // namespace bof4
