// bof4_logprobs_plan.h - how bof4_token_logprobs cuts its rows: tiles, waves and parts.  Without the GPU's headers.
#pragma once
#include <cstddef>
#include <cstdint>

namespace bof4 {

constexpr uint32_t LOGPROBS_WORDS = 4, LOGPROBS_JOIN_WAVES = 16;  // 16-byte words per lane and tile; waves per row that joins
constexpr uint32_t LOGPROBS_TILE = 64 * LOGPROBS_WORDS;           // words
constexpr uint32_t LOGPROBS_MAX_SPLITS = 64;
constexpr uint32_t logprobs_word_elements(bool bf16) { return bf16 ? 8 : 4; }

// The lowest of a lane's logits of a tile that `bits` names, or its last one where none is named: always one of the tile.
constexpr uint32_t logprobs_lowest(uint32_t bits, uint32_t per_word) {
    return (uint32_t)__builtin_ctz(bits | 1u << (LOGPROBS_WORDS * per_word - 1));
}
// Where a lane's i-th logit lies in a tile: its word.
constexpr uint32_t logprobs_tile_word(uint32_t i, uint32_t lane, uint32_t per_word) { return 64 * (i / per_word) + lane; }

// Waves and parts per row.  About 2048 waves keep the chip busy; more of them cost more than they bring, since what a wave does
// at its row's end is worth a tile or two.  So two waves share a row from 1024 rows on (four where a row of bfloat16 is long: a
// compute unit holds fewer of those waves, and two leave the last round of workgroups too empty), four from 512 on, and fewer rows
// are cut into parts of at least a tile per wave for two waves each.  us, one alternative, this / four waves and twice the workgroups:
// bfloat16 256 x 32000 11.6 / 12.9, 600 x 32000 15.6 / 19.6, 256 x 128000 20.5 / 23.1, binary32 600 x 32000 17.7 / 21.3; 2000 x 128000
// with two / four waves bfloat16 123 / 103, binary32 187 / 193.
struct LogprobsCut {
    uint32_t waves, splits, tiles_per_split;
};
inline LogprobsCut logprobs_cut(uint64_t n_rows, uint64_t vocab, bool bf16) {
    const uint64_t per_word = logprobs_word_elements(bf16), words = (vocab + 2 * per_word - 2) / per_word;  // wherever it begins
    const uint64_t tiles = (words + LOGPROBS_TILE - 1) / LOGPROBS_TILE;
    if (n_rows >= 512) return {n_rows >= 1024 && !(bf16 && tiles >= 48) ? 2u : 4u, 1u, (uint32_t)tiles};
    uint64_t splits = (1024 + n_rows - 1) / n_rows;
    if (splits > LOGPROBS_MAX_SPLITS) splits = LOGPROBS_MAX_SPLITS;
    uint64_t per = (tiles + splits - 1) / splits;
    if (per < 2) per = 2;
    return {2, (uint32_t)((tiles + per - 1) / per), (uint32_t)per};
}

}  // namespace bof4
