// The plans of linear layers for tests on the CPU: compiled and called by tests/test_host_layer_plan.py.
#include "bof4_gemm_plan.h"

using namespace bof4;

struct LayerPlan {
    uint32_t way, decoded_split, decoded_slab_tiles, flush, carry;
    uint64_t need, slab_bytes;  // `need`: workspace without which the call takes another way
};

extern "C" void layer_plan(uint64_t rows, uint64_t cols, uint32_t n_tokens, int list, int bf16, uint64_t ws_bytes, LayerPlan* out) {
    const GemmPlan P = gemm_plan(rows, cols, n_tokens, list != 0, (size_t)ws_bytes, bf16 ? GEMM_LAYER_BF16 : GEMM_LAYER);
    *out = {(uint32_t)P.way, P.decoded.split, P.decoded.slab_tiles, P.chains.wide_flush, P.chains.wide_carry ? 1u : 0u, P.ws.total,
            P.decoded.slab_bytes};
    if (P.way == GEMM_WIDE) out->need = P.ws.wide(P.wide.split, n_tokens, rows, true);
    if (P.way == GEMM_DECODED) out->need = P.ws.decoded(P.decoded.split, n_tokens, rows, true) + P.decoded.slab_bytes;
}
extern "C" uint64_t layer_workspace_bytes(uint64_t rows, uint64_t cols, uint32_t n_tokens) {
    return gemm_ws_bytes(rows, cols, n_tokens, true);
}
