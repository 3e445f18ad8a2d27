// bof4_logprobs.hip - C entries of the token log probabilities and their gradient (include/bof4.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "bof4.h"
#include "bof4_gemm_plan.h"
#include "bof4_host.h"
#include "bof4_logprobs.h"
#include "bof4_logprobs_plan.h"

namespace {
using namespace bof4;

constexpr uint64_t LOGPROBS_MAX_ROWS = 1ull << 23, LOGPROBS_MAX_VOCAB = 1ull << 30;  // (a launch holds fewer than 2^32 lanes)
}  // namespace

extern "C" {

size_t bof4_token_logprobs_workspace_bytes(uint64_t n_rows, uint64_t vocab, uint32_t top) {
    if (n_rows == 0 || vocab == 0 || top > LOGPROBS_MAX_TOP || n_rows > LOGPROBS_MAX_ROWS || vocab > LOGPROBS_MAX_VOCAB) return 0;
    const uint32_t f32 = logprobs_cut(n_rows, vocab, false).splits, bf16 = logprobs_cut(n_rows, vocab, true).splits;
    const uint64_t most = f32 > bf16 ? f32 : bf16;
    return most > 1 ? align_up(n_rows * most * (sizeof(LogprobsPart) + 8 * top), 256) : 256;
}

int bof4_token_logprobs(const void* logits_dev, uint32_t logits_type, uint64_t n_rows, uint64_t vocab, uint64_t ld_logits,
                        const int64_t* target_dev, uint32_t top, float* logprob_dev, float* entropy_dev,
                        int64_t* top_idx_dev, float* top_logprob_dev, float* stats_dev, void* ws_dev, size_t ws_bytes,
                        void* stream) {
    if (!logits_dev || !ws_dev) return fail(BOF4_ERR_ARG, "bof4_token_logprobs: null pointer");
    if (!valid_type(logits_type)) return fail(BOF4_ERR_ARG, "bof4_token_logprobs: logits are BOF4_F32 or BOF4_BF16");
    if (n_rows == 0 || vocab == 0 || n_rows > LOGPROBS_MAX_ROWS || vocab > LOGPROBS_MAX_VOCAB)
        return fail(BOF4_ERR_ARG, "bof4_token_logprobs: 1 to 2^23 rows and 1 to 2^30 tokens in the vocabulary");
    if (ld_logits < vocab) return fail(BOF4_ERR_ARG, "bof4_token_logprobs: row stride below the vocabulary");
    if (!target_dev != !logprob_dev)
        return fail(BOF4_ERR_ARG, "bof4_token_logprobs: targets and their log probabilities come together");
    if (top > LOGPROBS_MAX_TOP || (top > 0 && (!top_idx_dev || !top_logprob_dev)))
        return fail(BOF4_ERR_ARG, "bof4_token_logprobs: at most 64 alternatives, with both their buffers");
    if (!aligned(logits_dev, type_bytes(logits_type)) || !aligned(target_dev, 8) || !aligned(logprob_dev, 4) ||
        !aligned(entropy_dev, 4) || !aligned(top_idx_dev, 8) || !aligned(top_logprob_dev, 4) || !aligned(stats_dev, 4) ||
        !aligned(ws_dev, 256))
        return fail(BOF4_ERR_ARG, "bof4_token_logprobs: misaligned pointer (its element's size; the workspace 256)");
    if (ws_bytes < bof4_token_logprobs_workspace_bytes(n_rows, vocab, top))
        return fail(BOF4_ERR_WORKSPACE, "bof4_token_logprobs: workspace too small");
    hipStream_t s = (hipStream_t)stream;
    const LogprobsArgs a = {logits_dev, ld_logits, (uint32_t)n_rows, (uint32_t)vocab, top, target_dev,
                            logprob_dev, entropy_dev, top_logprob_dev, stats_dev, top_idx_dev};
    const bool bf16 = logits_type == BOF4_BF16;
    const LogprobsCut cut = logprobs_cut(n_rows, vocab, bf16);
    timing_begin(s);
#define BOF4_LAUNCH_LOGPROBS(BF16_, WAVES_)                                                                                   \
    hipLaunchKernelGGL((logprobs_kernel<BF16_, WAVES_>), dim3(a.n_rows * cut.splits), dim3(64 * WAVES_), 0, s, a, cut.splits, \
                       cut.tiles_per_split, (char*)ws_dev);
    if (bf16) {
        if (cut.waves == 2) { BOF4_LAUNCH_LOGPROBS(true, 2) } else { BOF4_LAUNCH_LOGPROBS(true, 4) }
    } else {
        if (cut.waves == 2) { BOF4_LAUNCH_LOGPROBS(false, 2) } else { BOF4_LAUNCH_LOGPROBS(false, 4) }
    }
#undef BOF4_LAUNCH_LOGPROBS
    timing_end(s);
    if (cut.splits > 1) {
        uint32_t waves = 1;  // one of two to four parts' lists each; one where there are no lists of more than one
        while (top > 1 && waves < LOGPROBS_JOIN_WAVES && 2 * waves < cut.splits) waves *= 2;
        if (bf16) {
            hipLaunchKernelGGL((logprobs_join_kernel<true>), dim3(a.n_rows), dim3(64 * waves), 0, s, a, cut.splits, (char*)ws_dev);
        } else {
            hipLaunchKernelGGL((logprobs_join_kernel<false>), dim3(a.n_rows), dim3(64 * waves), 0, s, a, cut.splits, (char*)ws_dev);
        }
    }
    HIP_TRY(hipGetLastError());
    return BOF4_OK;
}

int bof4_token_logprobs_backward(const void* logits_dev, uint32_t logits_type, uint64_t n_rows, uint64_t vocab,
                                 uint64_t ld_logits, const float* stats_dev, const int64_t* target_dev,
                                 const float* d_logprob_dev, const float* entropy_dev, const float* d_entropy_dev,
                                 void* d_logits_dev, uint32_t d_logits_type, uint64_t ld_d_logits, void* stream) {
    if (!logits_dev || !stats_dev || !d_logits_dev) return fail(BOF4_ERR_ARG, "bof4_token_logprobs_backward: null pointer");
    if (!valid_type(logits_type) || !valid_type(d_logits_type))
        return fail(BOF4_ERR_ARG, "bof4_token_logprobs_backward: logits and gradients are BOF4_F32 or BOF4_BF16");
    if (n_rows == 0 || vocab == 0 || n_rows > LOGPROBS_MAX_ROWS || vocab > LOGPROBS_MAX_VOCAB)
        return fail(BOF4_ERR_ARG, "bof4_token_logprobs_backward: 1 to 2^23 rows and 1 to 2^30 tokens in the vocabulary");
    if (ld_logits < vocab || ld_d_logits < vocab)
        return fail(BOF4_ERR_ARG, "bof4_token_logprobs_backward: row stride below the vocabulary");
    if (!target_dev != !d_logprob_dev || !entropy_dev != !d_entropy_dev)
        return fail(BOF4_ERR_ARG, "bof4_token_logprobs_backward: targets come with d_logprob, the entropy with d_entropy");
    if (d_logits_dev == logits_dev && (logits_type != d_logits_type || ld_logits != ld_d_logits))
        return fail(BOF4_ERR_ARG, "bof4_token_logprobs_backward: in place only with one type and row stride");
    if (!aligned(logits_dev, type_bytes(logits_type)) || !aligned(d_logits_dev, type_bytes(d_logits_type)) ||
        !aligned(target_dev, 8) || !aligned(stats_dev, 4) || !aligned(d_logprob_dev, 4) || !aligned(entropy_dev, 4) ||
        !aligned(d_entropy_dev, 4))
        return fail(BOF4_ERR_ARG, "bof4_token_logprobs_backward: misaligned pointer (its element's size)");
    hipStream_t s = (hipStream_t)stream;
    const LogprobsGradArgs a = {logits_dev, d_logits_dev, ld_logits, ld_d_logits, (uint32_t)n_rows, (uint32_t)vocab,
                                target_dev, stats_dev, d_logprob_dev, entropy_dev, d_entropy_dev};
    const bool bf16 = logits_type == BOF4_BF16;
    const uint64_t per_word = logprobs_word_elements(bf16), words = (vocab + 2 * per_word - 2) / per_word;  // wherever a row begins
    const uint64_t stretches = (words * per_word + LOGPROBS_GRAD_STRETCH - 1) / LOGPROBS_GRAD_STRETCH;
    if (n_rows * stretches >= 1ull << 24)
        return fail(BOF4_ERR_ARG, "bof4_token_logprobs_backward: 2^24 and more stretches of 2048 logits");
    const dim3 grid((uint32_t)(n_rows * stretches));
    timing_begin(s);
#define BOF4_LAUNCH_GRAD(IN_, OUT_)                                                                                     \
    if (d_entropy_dev) {                                                                                               \
        hipLaunchKernelGGL((logprobs_grad_kernel<IN_, OUT_, true>), grid, dim3(256), 0, s, a, (uint32_t)stretches);     \
    } else {                                                                                                           \
        hipLaunchKernelGGL((logprobs_grad_kernel<IN_, OUT_, false>), grid, dim3(256), 0, s, a, (uint32_t)stretches);    \
    }
    if (bf16) {
        if (d_logits_type == BOF4_BF16) { BOF4_LAUNCH_GRAD(true, true) } else { BOF4_LAUNCH_GRAD(true, false) }
    } else {
        if (d_logits_type == BOF4_BF16) { BOF4_LAUNCH_GRAD(false, true) } else { BOF4_LAUNCH_GRAD(false, false) }
    }
#undef BOF4_LAUNCH_GRAD
    timing_end(s);
    HIP_TRY(hipGetLastError());
    return BOF4_OK;
}

}  // extern "C"
