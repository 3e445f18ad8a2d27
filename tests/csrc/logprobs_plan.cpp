// The cuts of the token log probabilities for tests on the CPU: compiled and called by tests/test_host_logprobs_plan.py.
#include "bof4_logprobs_plan.h"

using namespace bof4;

extern "C" uint32_t lowest(uint32_t bits, uint32_t per_word) { return logprobs_lowest(bits, per_word); }
extern "C" uint32_t tile_word(uint32_t bits, uint32_t lane, uint32_t per_word) {
    return logprobs_tile_word(logprobs_lowest(bits, per_word), lane, per_word);
}
extern "C" uint32_t tile_words() { return LOGPROBS_TILE; }
extern "C" void cut(uint64_t n_rows, uint64_t vocab, int bf16, uint32_t* out) {
    const LogprobsCut c = logprobs_cut(n_rows, vocab, bf16 != 0);
    out[0] = c.waves;
    out[1] = c.splits;
    out[2] = c.tiles_per_split;
}
