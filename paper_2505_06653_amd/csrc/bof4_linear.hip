// bof4_linear.hip - C entries of the linear layer around a product with a quantised matrix and of its gradients
// (include/bof4.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "bof4.h"
#include "bof4_host.h"
#include "bof4_linear.h"
#include "bof4_products.h"

static_assert(BOF4_ACT_NONE == bof4::ACT_NONE && BOF4_ACT_RELU == bof4::ACT_RELU && BOF4_ACT_GELU == bof4::ACT_GELU &&
              BOF4_ACT_GELU_TANH == bof4::ACT_GELU_TANH && BOF4_ACT_SILU == bof4::ACT_SILU, "one numbering");

namespace {
using namespace bof4;

constexpr uint64_t LINEAR_MAX_ROWS = 1ull << 30, LINEAR_BACKWARD_MAX_ROWS = 1ull << 18;

// A tensor of tokens x rows as a call names it.
struct Rows {
    const void* p;
    uint32_t type;
    uint64_t ld;
    bool ok(uint64_t rows) const { return !p || (valid_type(type) && aligned(p, type_bytes(type)) && ld >= rows); }
    // the other tensor of the same elements, or another place altogether
    bool same_or_apart(const Rows& o) const { return !p || p != o.p || (type == o.type && ld == o.ld); }
};

int layer_out(const bof4_layer* layer, uint64_t rows, const void* x_dev, LayerOut* out) {
    if (!layer) return fail(BOF4_ERR_ARG, "linear layer: null layer");
    const bof4_layer& l = *layer;
    if (!l.y_dev) return fail(BOF4_ERR_ARG, "linear layer: null pointer (y)");
    if (l.act >= ACT_COUNT) return fail(BOF4_ERR_ARG, "linear layer: unknown activation");
    const Rows bias = {l.bias_dev, l.bias_type, rows}, mul = {l.mul_dev, l.mul_type, l.ld_mul};
    const Rows residual = {l.residual_dev, l.residual_type, l.ld_residual}, y = {l.y_dev, l.y_type, l.ld_y};
    const Rows pre = {l.pre_dev, l.pre_type, l.ld_pre};
    if (!bias.ok(rows) || !mul.ok(rows) || !residual.ok(rows) || !y.ok(rows) || !pre.ok(rows))
        return fail(BOF4_ERR_ARG, "linear layer: bias, mul, residual, y and pre are BOF4_F32 or BOF4_BF16, aligned to their "
                                  "element, row strides not below rows");
    if (!y.same_or_apart(mul) || !y.same_or_apart(residual) || !pre.same_or_apart(mul) || !pre.same_or_apart(residual))
        return fail(BOF4_ERR_ARG, "linear layer: results go over mul or the residual only with their type and row stride");
    if (l.y_dev == x_dev || l.pre_dev == x_dev || l.pre_dev == l.y_dev || (l.bias_dev && (l.bias_dev == l.y_dev || l.bias_dev == l.pre_dev)))
        return fail(BOF4_ERR_ARG, "linear layer: y and pre need memory of their own");
    *out = LayerOut{l.bias_dev, l.mul_dev, l.residual_dev, l.y_dev, l.pre_dev, l.ld_mul, l.ld_residual, l.ld_y, l.ld_pre, l.act,
                    l.bias_type == BOF4_BF16, l.mul_type == BOF4_BF16, l.residual_type == BOF4_BF16, l.y_type == BOF4_BF16,
                    l.pre_type == BOF4_BF16, 0, nullptr};
    return BOF4_OK;
}

// How the gradient by x is taken: W^^T in slabs of column tiles (the rows of the turned matrix), its rows' chunks, once for each
// term of dz, over `split` workgroups, and where things lie in the workspace.
//   Several terms take the tokens in passes of as many groups of them as LINEAR_TERMS_BYTES hold, each with the matrix turned anew,
// so that a large call needs little more memory than with one term: of 2^18 rows that is 2688 tokens in three terms, for which
// turning 2^18 x 4096 weights costs a fifteenth of the products.
constexpr uint64_t LINEAR_TERMS_BYTES = 4ull << 30;
struct LinearBackwardPlan {
    GemmDecodedPlan turned;
    uint32_t passes, tokens;           // of a pass but the last, which takes the rest
    uint32_t ranges, tiles_per_range;  // of a pass's tokens, for dbias
    size_t dbias, parts, decoded, total;
};
LinearBackwardPlan backward_plan_one(uint64_t rows, uint64_t cols, uint64_t n_tokens, uint64_t terms) {
    constexpr uint64_t GROUP = GEMM_WIDE_TOK_TILES * GEMM_TOKENS;
    const uint64_t row_chunks = (rows + GEMM_CHUNK - 1) / GEMM_CHUNK, token_bytes = terms * row_chunks * GEMM_CHUNK * 2;
    LinearBackwardPlan P;
    const uint64_t most = terms == 1 ? n_tokens : LINEAR_TERMS_BYTES / token_bytes / GROUP * GROUP;
    P.tokens = (uint32_t)(n_tokens < most ? n_tokens : most);
    P.passes = (uint32_t)((n_tokens + P.tokens - 1) / P.tokens);
    const uint64_t tok_tiles = (P.tokens + GEMM_TOKENS - 1) / GEMM_TOKENS;
    P.turned = gemm_decoded_plan(cols, rows, tok_tiles, terms);
    const uint64_t per = (tok_tiles + LINEAR_MOST_RANGES - 1) / LINEAR_MOST_RANGES;
    P.tiles_per_range = (uint32_t)per;
    P.ranges = (uint32_t)((tok_tiles + per - 1) / per);
    P.dbias = align_up(tok_tiles * GEMM_TOKENS * token_bytes, 256);
    P.parts = align_up(P.dbias + (uint64_t)P.passes * P.ranges * rows * 4, 256);
    P.decoded = align_up(P.parts + (P.turned.split > 1 ? P.turned.split * (uint64_t)P.tokens * cols * 4 : 0), 256);
    P.total = P.decoded + P.turned.slab_bytes;
    return P;
}
// Enough for every number of terms and of tokens up to this (the split falls as they rise, so the largest need is not that of the most).
size_t backward_ws_bytes(uint64_t rows, uint64_t cols, uint64_t n_tokens) {
    constexpr uint64_t GROUP = GEMM_WIDE_TOK_TILES * GEMM_TOKENS;
    size_t need = 0;
    for (uint64_t below = 0; below < n_tokens; below += GROUP) {  // (one plan for all token tiles of a group)
        for (uint64_t terms = 1; terms <= LINEAR_MOST_TERMS; ++terms) {
            const size_t bytes = backward_plan_one(rows, cols, below + GROUP < n_tokens ? below + GROUP : n_tokens, terms).total;
            if (bytes > need) need = bytes;
        }
    }
    return need;
}
}  // namespace

extern "C" {

int bof4_gemv_linear(const uint8_t* codes_dev, const uint16_t* scales_dev, uint64_t rows, uint64_t cols, uint32_t block,
                     const double* cb_host, const void* table_dev, uint64_t n_outliers, const void* x_dev, uint32_t n_tokens,
                     const bof4_layer* layer, void* stream) {
    if (!codes_dev || !scales_dev || !x_dev) return fail(BOF4_ERR_ARG, "bof4_gemv_linear: null pointer");
    if (!valid_block(block) || rows == 0 || cols == 0 || cols % block != 0 || n_tokens == 0)
        return fail(BOF4_ERR_ARG, "bof4_gemv_linear: bad rows, cols (a positive multiple of block), block or n_tokens");
    if (rows > LINEAR_MAX_ROWS || cols > GEMM_MAX_COLS)
        return fail(BOF4_ERR_ARG, "bof4_gemv_linear: at most 2^30 rows and 32768 columns");
    if (!valid_codebook(cb_host)) return fail(BOF4_ERR_ARG, "bof4_gemv_linear: codebook must be 16 finite ascending levels");
    if (n_outliers > 0 && !table_dev) return fail(BOF4_ERR_ARG, "bof4_gemv_linear: outliers without their table");
    if (n_outliers > 0xffffffffull) return fail(BOF4_ERR_ARG, "bof4_gemv_linear: more than 2^32 - 1 outliers");
    if (!aligned(codes_dev, 16) || !aligned(x_dev, 16) || !aligned(scales_dev, 2) || !aligned(table_dev, 8))
        return fail(BOF4_ERR_ARG, "bof4_gemv_linear: misaligned pointer (codes and x need 16 bytes, the table 8)");
    LayerOut out;
    const int rc = layer_out(layer, rows, x_dev, &out);
    if (rc != BOF4_OK) return rc;
    return gemv_run({codes_dev, scales_dev, rows, cols, block, cb_host, table_dev, n_outliers, x_dev, n_tokens, (hipStream_t)stream}, out);
}

size_t bof4_gemm_linear_workspace_bytes(uint64_t rows, uint64_t cols, uint32_t n_tokens) {
    if (rows == 0 || cols == 0 || n_tokens == 0) return 0;
    return gemm_ws_bytes(rows, cols, n_tokens, true);
}

int bof4_gemm_linear(const void* packed_dev, uint64_t rows, uint64_t cols, const double* cb_host, const void* table_dev,
                     uint64_t n_outliers, const void* x_dev, uint32_t n_tokens, const bof4_layer* layer, void* ws_dev,
                     size_t ws_bytes, void* stream) {
    if (!packed_dev || !x_dev || !ws_dev) return fail(BOF4_ERR_ARG, "bof4_gemm_linear: null pointer");
    if (rows == 0 || cols == 0 || cols % 32 != 0 || n_tokens == 0)
        return fail(BOF4_ERR_ARG, "bof4_gemm_linear: bad rows, cols (a positive multiple of 32) or n_tokens");
    if (rows > LINEAR_MAX_ROWS || cols > GEMM_MAX_COLS || n_tokens > GEMM_MAX_TOKENS)
        return fail(BOF4_ERR_ARG, "bof4_gemm_linear: at most 2^30 rows, 32768 columns and 65536 tokens");
    if (!valid_codebook(cb_host)) return fail(BOF4_ERR_ARG, "bof4_gemm_linear: codebook must be 16 finite ascending levels");
    if (n_outliers > 0 && !table_dev) return fail(BOF4_ERR_ARG, "bof4_gemm_linear: outliers without their table");
    if (n_outliers > 0xffffffffull) return fail(BOF4_ERR_ARG, "bof4_gemm_linear: more than 2^32 - 1 outliers");
    if (!aligned(packed_dev, 16) || !aligned(x_dev, 16) || !aligned(table_dev, 8) || !aligned(ws_dev, 256))
        return fail(BOF4_ERR_ARG, "bof4_gemm_linear: misaligned pointer (packed matrix and x need 16 bytes, the table 8, the workspace 256)");
    LayerOut out;
    const int rc = layer_out(layer, rows, x_dev, &out);
    if (rc != BOF4_OK) return rc;
    const GemmPlan P = gemm_plan(rows, cols, n_tokens, n_outliers > 0, ws_bytes,
                                 out.y_bf16 && (!out.pre || out.pre_bf16) ? GEMM_LAYER_BF16 : GEMM_LAYER);
    if (ws_bytes < P.ws.total) return fail(BOF4_ERR_WORKSPACE, "bof4_gemm_linear: workspace too small");
    return gemm_run({packed_dev, rows, cols, cb_host, table_dev, n_outliers, x_dev, n_tokens, ws_dev, (hipStream_t)stream}, P, out);
}

size_t bof4_gemm_linear_backward_workspace_bytes(uint64_t rows, uint64_t cols, uint32_t n_tokens) {
    if (rows == 0 || cols == 0 || n_tokens == 0 || rows > LINEAR_BACKWARD_MAX_ROWS || cols > GEMM_MAX_COLS || n_tokens > GEMM_MAX_TOKENS)
        return 0;
    return backward_ws_bytes(rows, cols, n_tokens);
}

int bof4_gemm_linear_backward(const void* packed_dev, uint64_t rows, uint64_t cols, const double* cb_host, const void* table_dev,
                              uint64_t n_outliers, uint32_t n_tokens, const bof4_layer_gradient* gradient, void* ws_dev,
                              size_t ws_bytes, void* stream) {
    if (!packed_dev || !gradient || !ws_dev) return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: null pointer");
    const bof4_layer_gradient& l = *gradient;
    if (!l.dy_dev || !l.dx_dev) return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: null pointer (dy, dx)");
    if (rows == 0 || cols == 0 || cols % 32 != 0 || n_tokens == 0)
        return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: bad rows, cols (a positive multiple of 32) or n_tokens");
    if (rows > LINEAR_BACKWARD_MAX_ROWS || cols > GEMM_MAX_COLS || n_tokens > GEMM_MAX_TOKENS)
        return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: at most 2^18 rows, 32768 columns and 65536 tokens");
    if (!valid_codebook(cb_host)) return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: codebook must be 16 finite ascending levels");
    if (n_outliers > 0 && !table_dev) return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: outliers without their table");
    if (n_outliers > 0xffffffffull) return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: more than 2^32 - 1 outliers");
    if (l.act >= ACT_COUNT) return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: unknown activation");
    if (l.act != ACT_NONE && !l.pre_dev) return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: an activation needs pre");
    if (l.dmul_dev && (!l.mul_dev || !l.pre_dev)) return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: dmul needs mul and pre");
    const Rows dy = {l.dy_dev, l.dy_type, l.ld_dy}, mul = {l.mul_dev, l.mul_type, l.ld_mul}, pre = {l.pre_dev, l.pre_type, l.ld_pre};
    const Rows dmul = {l.dmul_dev, l.dmul_type, l.ld_dmul}, dx = {l.dx_dev, l.dx_type, l.ld_dx};
    if (!dy.ok(rows) || !mul.ok(rows) || !pre.ok(rows) || !dmul.ok(rows) || !dx.ok(cols) || !aligned(l.dbias_dev, 4))
        return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: dy, pre, mul, dmul and dx are BOF4_F32 or BOF4_BF16, aligned to their "
                                  "element, row strides not below their width");
    if (!dmul.same_or_apart(dy) || !dmul.same_or_apart(mul) || !dmul.same_or_apart(pre))
        return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: dmul goes over dy, mul or pre only with their type and row stride");
    if (l.dx_dev == l.dmul_dev || (const void*)l.dx_dev == l.dbias_dev || (l.dbias_dev && (void*)l.dbias_dev == l.dmul_dev))
        return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: dx, dmul and dbias need memory of their own");
    if (!aligned(packed_dev, 16) || !aligned(table_dev, 8) || !aligned(ws_dev, 256))
        return fail(BOF4_ERR_ARG, "bof4_gemm_linear_backward: misaligned pointer (the packed matrix needs 16 bytes, the table 8, the workspace 256)");
    const uint32_t terms = linear_dz_terms(l.act, l.dy_type == BOF4_BF16, l.mul_dev != nullptr, l.mul_type == BOF4_BF16, l.dx_type == BOF4_BF16);
    const LinearBackwardPlan P = backward_plan_one(rows, cols, n_tokens, terms);
    if (ws_bytes < P.total) return fail(BOF4_ERR_WORKSPACE, "bof4_gemm_linear_backward: workspace too small");
    const GemmTableLayout T = gemm_table_layout(rows, cols);
    const uint32_t* offsets_dev = (const uint32_t*)table_dev;
    const uint32_t* entries_dev = table_dev ? (const uint32_t*)((const char*)table_dev + T.entries) : nullptr;
    hipStream_t s = (hipStream_t)stream;
    const CodebookArgs cb = make_codebook_args(cb_host);
    char* ws = (char*)ws_dev;
    uint4* xp = (uint4*)ws;
    float* dbias_parts = (float*)(ws + P.dbias);
    uint4* decoded = (uint4*)(ws + P.decoded);
    const uint32_t row_chunks = (uint32_t)((rows + GEMM_CHUNK - 1) / GEMM_CHUNK), chunks = (uint32_t)((cols + GEMM_CHUNK - 1) / GEMM_CHUNK);
    LinearGradArgs a = {l.dy_dev, l.act != ACT_NONE || l.dmul_dev ? l.pre_dev : nullptr, l.mul_dev, l.dmul_dev,
                        l.dbias_dev ? dbias_parts : nullptr, l.ld_dy, l.ld_pre, l.ld_mul, l.ld_dmul, l.act, terms,
                        l.dy_type == BOF4_BF16, l.pre_type == BOF4_BF16, l.mul_type == BOF4_BF16, l.dmul_type == BOF4_BF16};
    LayerOut out = {};
    out.y = l.dx_dev;
    out.ld_y = l.ld_dx;
    out.y_bf16 = l.dx_type == BOF4_BF16;
    out.parts = (float*)(ws + P.parts);
    const GemmDecodedPlan& D = P.turned;
    const uint32_t col_tiles = (uint32_t)(cols / GEMM_ROWS);
    // Chunks in one chain of the matrix cores' additions (32 products of 16 terms): the sums of the chains are added in
    // binary32 as well, so a sum over 11008 rows takes 22 of them.
    constexpr uint32_t FLUSH = 8;
    timing_begin(s);
    // dz in the launch that turns the matrix or in one of its own, where it is not held to the few workgroups per compute unit
    // that the other's LDS leaves (calls with all gradients, own launch / joint, us: 1024 x 1024 with 64 tokens 21.9 / 19.1, 4096 x
    // 4096 with 333 / 1000 / 2000 39.9 / 38.5, 64.2 / 63.0, 100.2 / 101.2, 11008 x 4096 with 256 / 512 / 1000 / 2000 67.0 / 61.6, 89.5 /
    // 87.4, 137.0 / 138.0, 230 / 244).
    const bool dz_apart = (uint64_t)n_tokens * rows > (6ull << 20);
    const uint32_t dbias_groups = l.dbias_dev ? (uint32_t)((rows + 255) / 256) : 0;
    uint32_t n_parts = 0;  // of dbias
    for (uint32_t pass = 0; pass < P.passes; ++pass) {
        const bool last = pass + 1 == P.passes;
        const uint32_t n = last ? n_tokens - pass * P.tokens : P.tokens, tok_tiles = (n + GEMM_TOKENS - 1) / GEMM_TOKENS;
        const uint32_t ranges = (tok_tiles + P.tiles_per_range - 1) / P.tiles_per_range;
        n_parts += ranges;
        if (dz_apart)
            hipLaunchKernelGGL(linear_dz_kernel, dim3(row_chunks, ranges), dim3(256), 0, s, a, n, (uint32_t)rows, row_chunks,
                               tok_tiles, P.tiles_per_range, xp);
        for (uint32_t ct0 = 0; ct0 < col_tiles; ct0 += D.slab_tiles) {
            const uint32_t n_ct = col_tiles - ct0 < D.slab_tiles ? col_tiles - ct0 : D.slab_tiles;
            const uint64_t jobs = (uint64_t)((n_ct + 1) / 2) * row_chunks;
            const LinearDzCall dz = {a, ct0 == 0 && !dz_apart ? row_chunks * ranges : 0, n, (uint32_t)rows, tok_tiles, P.tiles_per_range, xp};
#define BOF4_LAUNCH_TURN(OUT_)                                                                                          \
    hipLaunchKernelGGL((linear_turn_kernel<OUT_>),                                                                      \
                       dim3(dz.dz_groups + (uint32_t)((jobs + LINEAR_TURN_WAVES - 1) / LINEAR_TURN_WAVES)),             \
                       dim3(64 * LINEAR_TURN_WAVES), 0, s, (const char*)packed_dev, ct0, n_ct, chunks, row_chunks, cb,  \
                       offsets_dev, entries_dev, (uint32_t)n_outliers, T.lg, T.row_tiles, decoded, dz);
            if (n_outliers > 0) { BOF4_LAUNCH_TURN(true) } else { BOF4_LAUNCH_TURN(false) }
#undef BOF4_LAUNCH_TURN
#define BOF4_MULTIPLY(TERMS_) \
    gemm_multiply_decoded<TERMS_>(D, FLUSH, false, decoded, ct0 * GEMM_ROWS, n_ct, cols, TERMS_ * row_chunks, xp, n, out, s);
            if (terms == 1) { BOF4_MULTIPLY(1) } else if (terms == 2) { BOF4_MULTIPLY(2) } else { BOF4_MULTIPLY(3) }
#undef BOF4_MULTIPLY
        }
        if (D.split > 1) {
            const uint32_t dx_groups = (uint32_t)((cols + 1023) / 1024), most = n < 65535 ? n : 65535;
            hipLaunchKernelGGL(linear_sum_kernel, dim3(dx_groups * most + (last ? dbias_groups : 0)), dim3(256), 0, s, D.split, n,
                               (uint32_t)cols, out, dx_groups, most, dbias_parts, n_parts, (uint32_t)rows, l.dbias_dev);
        } else if (last && l.dbias_dev) {
            hipLaunchKernelGGL(linear_dbias_kernel, dim3(dbias_groups), dim3(256), 0, s, dbias_parts, n_parts, (uint32_t)rows, l.dbias_dev);
        }
        // the next pass's tokens
        a.dy = (const char*)a.dy + (uint64_t)n * a.ld_dy * type_bytes(l.dy_type);
        if (a.pre) a.pre = (const char*)a.pre + (uint64_t)n * a.ld_pre * type_bytes(l.pre_type);
        if (a.mul) a.mul = (const char*)a.mul + (uint64_t)n * a.ld_mul * type_bytes(l.mul_type);
        if (a.dmul) a.dmul = (char*)a.dmul + (uint64_t)n * a.ld_dmul * type_bytes(l.dmul_type);
        if (a.dbias_parts) a.dbias_parts += (uint64_t)ranges * rows;
        out.token0 += n;
    }
    timing_end(s);
    HIP_TRY(hipGetLastError());
    return BOF4_OK;
}

}  // extern "C"
