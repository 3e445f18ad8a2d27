// bof4_products.h - the host side of the products with a quantised matrix, from checked arguments to launches, for the plain
// products (bof4.hip) and for the layers around them (bof4_linear.hip): Out says where the sums go.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "bof4_gemm.h"
#include "bof4_gemv.h"
#include "bof4_host.h"

namespace bof4 {

// Workgroups of a gemv_kernel that the current device holds at once (cached per kernel, workgroup size and dynamic LDS; 0
// on failure).
template <class Out>
uint64_t gemv_resident_workgroups(int variant, uint32_t threads, size_t lds) {
    struct Key {
        int device, variant;
        uint32_t threads;
        size_t lds;
        uint64_t slots;
    };
    static thread_local Key cache[16] = {};
    static thread_local int next = 0;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return 0;
    for (const Key& k : cache)
        if (k.slots && k.device == dev && k.variant == variant && k.threads == threads && k.lds == lds) return k.slots;
    int per_cu = 0, cus = 0;
    hipError_t e;
#define BOF4_OCCUPANCY(T_, OUT_) \
    e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, gemv_kernel<T_, OUT_, Out>, (int)threads, lds); break;
    switch (variant) {
        case 0: BOF4_OCCUPANCY(1, false)
        case 1: BOF4_OCCUPANCY(1, true)
        case 2: BOF4_OCCUPANCY(2, false)
        case 3: BOF4_OCCUPANCY(2, true)
        case 4: BOF4_OCCUPANCY(3, false)
        case 5: BOF4_OCCUPANCY(3, true)
        case 6: BOF4_OCCUPANCY(4, false)
        default: BOF4_OCCUPANCY(4, true)
    }
#undef BOF4_OCCUPANCY
    if (e != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess)
        return 0;
    if (per_cu < 1) per_cu = 1;
    Key& slot = cache[next];
    next = (next + 1) % 16;
    slot = Key{dev, variant, threads, lds, (uint64_t)per_cu * (uint64_t)cus};
    return slot.slots;
}

// The largest matrix (in weights) that three or four tokens pass through in one launch of bof4_gemv instead of two: a weight is looked
// up once instead of twice and a launch saved, at three and two waves per SIMD instead of four.  What fits a compute unit
// then depends on a workgroup's waves, one per strip of 2048 columns up to eight, and decides on large matrices.  Two
// launches / one over 18 widths at 4 M to 600 M weights (us; three or four tokens, `l` with a list):
//   three  1001 x 1536 10.5 / 6.6, 22016 x 4096 30.7 / 23.7, l 40.7 / 31.9; four strips 28672 x 8192 65.5 / 53.2, l 81.6 / 82.7, l
//          40000 x 8192 113 / 119; six strips 1500 x 11008 1.12 - 1.15, 3600 x 11008 and more 0.98 - 0.85; more than eight
//          (two per wave) 80 M weights 1.04 - 1.27, 260 M 0.89 - 1.11
//   four   4096 x 4096 14.6 / 10.0; 28672 x 4096 41.9 / 41.1, l 55.9 / 61.2, l 16384 x 4096 38.1 / 37.6; three strips 6500 x 6144
//          1.07, l 1.11, 20000 x 6144 46.7 / 54.8, l 57.8 / 64.8; five strips 1.1 - 1.5; 28672 x 8192 76.7 / 77.6, l 95.3 / 91.9;
//          l six strips 120 M 1.03, 260 M 0.96
inline uint64_t gemv_most_weights(uint64_t strips, uint32_t n_tokens, bool list) {
    if (n_tokens == 3) {
        if (strips == 6) return 1ull << 25;
        if (strips > 8) return 1ull << 26;
        return strips == 4 && list ? 3ull << 26 : strips < 6 ? ~0ull : 1ull << 28;
    }
    if (strips == 5 || (strips == 1 && list)) return ~0ull;
    if (strips == 3 || (strips == 2 && list)) return list ? 1ull << 26 : 1ull << 25;
    if (list) return strips == 6 || (strips > 8 && strips < 13) ? 1ull << 27 : 1ull << 28;
    return strips > 8 && strips < 13 ? 1ull << 26 : 1ull << 27;
}

// Outlier table of bof4_gemv: offsets [rows * strips + 1] (padded to 8 bytes), then one {column, delta} pair per entry.
struct GemvTableLayout {
    size_t entries, total;
};
inline GemvTableLayout gemv_table_layout(uint64_t rows, uint64_t strips, uint64_t n_outliers) {
    GemvTableLayout L;
    L.entries = align_up((rows * strips + 1) * 4, 8);
    L.total = L.entries + n_outliers * 8;
    return L;
}

// The table of bof4_gemm: offsets per tile of 32 rows and group of chunks, one closing offset, then the entries (4 bytes
// each) - inside the bytes of the gemv table for the same matrix and list, and with the entries at the same place.  The
// groups are as fine as fits in front of them.  Nothing here depends on the length of the list: a product that is told
// another length than the table was made for still finds offsets and entries where they are.
struct GemmTableLayout {
    GemmListGeometry lg;
    uint32_t row_tiles;
    size_t entries;
};
inline GemmTableLayout gemm_table_layout(uint64_t rows, uint64_t cols) {
    GemmTableLayout T;
    T.entries = gemv_table_layout(rows, (cols + GEMV_STRIP - 1) / GEMV_STRIP, 0).entries;
    const uint64_t row_tiles = (rows + GEMM_ROWS - 1) / GEMM_ROWS, chunks = (cols + GEMM_CHUNK - 1) / GEMM_CHUNK;
    T.row_tiles = (uint32_t)row_tiles;
    for (T.lg.log2_group = 0;; ++T.lg.log2_group) {  // ends: with 2^5 chunks per group there is one group per strip
        T.lg.n_groups = (uint32_t)((chunks + (1u << T.lg.log2_group) - 1) >> T.lg.log2_group);
        if ((row_tiles * T.lg.n_groups + 1) * 4 <= T.entries || T.lg.log2_group == 5) return T;
    }
}

// The partial sums of n_tokens x rows, `split` of them, to where they belong.
template <class Out>
void gemm_add_parts(uint32_t split, uint32_t n_tokens, uint64_t rows, const Out& dst, hipStream_t s) {
    if constexpr (Out::LAYER) {
        const uint32_t groups = (uint32_t)((rows + 1023) / 1024), most = n_tokens < 65535 ? n_tokens : 65535;
        hipLaunchKernelGGL((gemm_sum_layer_kernel<Out>), dim3(groups, most), dim3(256), 0, s, split, n_tokens, (uint32_t)rows, dst);
    } else {
        const uint64_t count = (uint64_t)n_tokens * rows;
        hipLaunchKernelGGL(gemm_sum_kernel, dim3((uint32_t)((count + 255) / 256)), dim3(256), 0, s, dst.first, dst.more, split - 1,
                           count, dst.first);
    }
}

// A slab of the decoded matrix times x (in TERMS bfloat16 terms, each with a chunk of its own), with 256 or 192 rows to a workgroup.
template <uint32_t TERMS = 1, class Out>
void gemm_multiply_decoded(const GemmDecodedPlan& D, uint32_t flush, bool carry, const uint4* decoded, uint32_t first_row, uint32_t n_rt,
                           uint64_t rows, uint32_t chunks, const uint4* xp, uint32_t n_tokens, const Out& dst, hipStream_t s) {
    const uint32_t tok_tiles = (n_tokens + GEMM_TOKENS - 1) / GEMM_TOKENS;
    const uint32_t tok_groups = (tok_tiles + GEMM_WIDE_TOK_TILES - 1) / GEMM_WIDE_TOK_TILES;
    const uint32_t tiles = gemm_decoded_tile(n_rt, tok_groups * D.split, D.per_split).row_tiles, groups = (n_rt + tiles - 1) / tiles;
#define BOF4_LAUNCH_DECODED(CARRY_, TILES_)                                                                                  \
    hipLaunchKernelGGL((gemm_decoded_kernel<CARRY_, TILES_, TERMS, Out>), dim3(tok_groups * groups * D.split), dim3(64 * GEMM_WIDE_WAVES), \
                       0, s, decoded, first_row, n_rt, (uint32_t)rows, chunks, xp, tok_tiles, tok_groups, D.per_split, flush,  \
                       n_tokens, D.split, dst);
    if constexpr (TERMS > 1) {  // (of gradients, whose sums are not carried)
        if (tiles == 8) { BOF4_LAUNCH_DECODED(false, 8) } else { BOF4_LAUNCH_DECODED(false, 6) }
    } else if (tiles == 8) {
        if (carry) { BOF4_LAUNCH_DECODED(true, 8) } else { BOF4_LAUNCH_DECODED(false, 8) }
    } else {
        if (carry) { BOF4_LAUNCH_DECODED(true, 6) } else { BOF4_LAUNCH_DECODED(false, 6) }
    }
#undef BOF4_LAUNCH_DECODED
}

struct GemmCall {
    const void* packed_dev;
    uint64_t rows, cols;
    const double* cb_host;
    const void* table_dev;
    uint64_t n_outliers;
    const void* x_dev;
    uint32_t n_tokens;
    void* ws_dev;
    hipStream_t stream;
};
template <class Out>
int gemm_run(const GemmCall& call, const GemmPlan& P, Out dst) {
    const auto [packed_dev, rows, cols, cb_host, table_dev, n_outliers, x_dev, n_tokens, ws_dev, s] = call;
    const GemmWsLayout& L = P.ws;
    const GemmTableLayout T = gemm_table_layout(rows, cols);
    const uint32_t* offsets_dev = (const uint32_t*)table_dev;
    const uint32_t* entries_dev = table_dev ? (const uint32_t*)((const char*)table_dev + T.entries) : nullptr;
    const CodebookArgs cb = make_codebook_args(cb_host);
    const uint32_t split = gemm_split(rows, cols, n_tokens), chunks = (uint32_t)((cols + GEMM_CHUNK - 1) / GEMM_CHUNK);
    const GemmChains& C = P.chains;
    const uint32_t per_wg_tiles = gemm_row_tiles_per_wg(rows, cols, n_tokens);
    const uint32_t row_groups = (uint32_t)(gemm_row_tiles(rows) / per_wg_tiles);
    const uint32_t n_pad = (n_tokens + GEMM_TOKENS - 1) / GEMM_TOKENS * GEMM_TOKENS, tok_tiles = n_pad / GEMM_TOKENS;
    const uint4* xp = (const uint4*)((char*)ws_dev + L.xp);
    float* part = (float*)((char*)ws_dev + L.part);
    const uint64_t x_words = (uint64_t)tok_tiles * chunks * 256;
    const uint32_t pack_groups = (uint32_t)((x_words + 255) / 256);
    if (!P.x_in_place && P.way != GEMM_DECODED) {
        hipLaunchKernelGGL(gemm_pack_x_kernel, dim3(pack_groups), dim3(256), 0, s,
                           (const uint16_t*)x_dev, n_tokens, (uint32_t)cols, chunks, n_pad, (uint4*)xp);
    }
    timing_begin(s);
    const uint32_t tok_groups = (tok_tiles + GEMM_WIDE_TOK_TILES - 1) / GEMM_WIDE_TOK_TILES;
    float* wide_parts = (float*)((char*)ws_dev + L.wide_part);
    if constexpr (Out::LAYER) dst.parts = wide_parts;
    else dst.more = wide_parts;
    if (P.way == GEMM_DECODED) {
        const GemmDecodedPlan& D = P.decoded;
        uint4* decoded = (uint4*)((char*)ws_dev + L.decoded(D.split, n_tokens, rows, Out::LAYER));
        for (uint32_t rt0 = 0; rt0 < T.row_tiles; rt0 += D.slab_tiles) {
            const uint32_t n_rt = T.row_tiles - rt0 < D.slab_tiles ? T.row_tiles - rt0 : D.slab_tiles;
            const uint64_t jobs = (uint64_t)n_rt * ((chunks + GEMM_DECODE_TILES - 1) / GEMM_DECODE_TILES);
            const uint32_t packing = rt0 == 0 ? pack_groups : 0, decoding = (uint32_t)((jobs + GEMM_DECODE_WAVES - 1) / GEMM_DECODE_WAVES);
#define BOF4_LAUNCH_DECODE(OUT_)                                                                                       \
    hipLaunchKernelGGL((gemm_decode_kernel<OUT_>), dim3(packing + decoding), dim3(64 * GEMM_DECODE_WAVES), 0, s,       \
                       (const char*)packed_dev, rt0, n_rt, chunks, cb, offsets_dev, entries_dev, (uint32_t)n_outliers, T.lg, \
                       T.row_tiles, decoded, packing, (const uint16_t*)x_dev, n_tokens, (uint32_t)cols, n_pad, (uint4*)xp);
            if (n_outliers > 0) { BOF4_LAUNCH_DECODE(true) } else { BOF4_LAUNCH_DECODE(false) }
            gemm_multiply_decoded(D, D.flush, D.carry, decoded, rt0 * GEMM_ROWS, n_rt, rows, chunks, xp, n_tokens, dst, s);
#undef BOF4_LAUNCH_DECODE
        }
        if (D.split > 1) gemm_add_parts(D.split, n_tokens, rows, dst, s);
        timing_end(s);
        HIP_TRY(hipGetLastError());
        return BOF4_OK;
    }
    if (P.way == GEMM_WIDE) {
        const GemmWideSplit& W = P.wide;
        const uint32_t wide_groups = (T.row_tiles + GEMM_WIDE_WAVES - 1) / GEMM_WIDE_WAVES;
#define BOF4_LAUNCH_WIDE(OUT_, CARRY_)                                                                               \
    hipLaunchKernelGGL((gemm_wide_kernel<OUT_, CARRY_, Out>), dim3(tok_groups * wide_groups * W.split),                  \
                       dim3(64 * GEMM_WIDE_WAVES), 0, s, (const char*)packed_dev, (uint32_t)rows, (uint32_t)cols,   \
                       cb, offsets_dev, entries_dev, (uint32_t)n_outliers, T.lg, T.row_tiles,                       \
                       (uint32_t)gemm_row_tiles(rows), xp, tok_tiles, tok_groups, W.per_split, C.wide_flush, n_tokens,     \
                       W.split, dst);
        if (n_outliers > 0) {
            if constexpr (Out::LAYER) {
                if (C.wide_carry) { BOF4_LAUNCH_WIDE(true, true) } else { BOF4_LAUNCH_WIDE(true, false) }
            } else {
                BOF4_LAUNCH_WIDE(true, true)
            }
        }
        else if (C.wide_carry) { BOF4_LAUNCH_WIDE(false, true) }
        else { BOF4_LAUNCH_WIDE(false, false) }
#undef BOF4_LAUNCH_WIDE
        if (W.split > 1) gemm_add_parts(W.split, n_tokens, rows, dst, s);
        timing_end(s);
        HIP_TRY(hipGetLastError());
        return BOF4_OK;
    }
    for (uint32_t tile0 = 0; tile0 < tok_tiles;) {
        const uint32_t left = tok_tiles - tile0, nt_tiles = left >= 4 ? 4 : left;
        const uint32_t t0 = tile0 * GEMM_TOKENS;
        const uint32_t nt = n_tokens - t0 < nt_tiles * GEMM_TOKENS ? n_tokens - t0 : nt_tiles * GEMM_TOKENS;
        Out to = dst;
        if constexpr (Out::LAYER) {
            to.token0 = t0;
            to.parts = part;
        } else {
            to.first = split > 1 ? part : dst.first + (uint64_t)t0 * rows;
            to.more = part + (uint64_t)nt * rows;
        }
#define BOF4_LAUNCH_GEMM(R_, NT_, OUT_, IN_)                                                                      \
    hipLaunchKernelGGL((gemm_kernel<R_, NT_, OUT_, IN_, Out>), dim3(row_groups, split), dim3(64 * C.waves), 0, s,           \
                       (const char*)packed_dev, (uint32_t)rows, (uint32_t)cols, cb, offsets_dev, entries_dev,     \
                       (uint32_t)n_outliers, T.lg, T.row_tiles, xp, (const uint16_t*)x_dev, tile0, nt, C.list_flush, C.n_runs, to);
#define BOF4_LAUNCH_GEMM_NT(R_, OUT_)                                                                             \
    if (nt_tiles == 4) { BOF4_LAUNCH_GEMM(R_, 4, OUT_, false) }                                                     \
    else if (nt_tiles == 3) { BOF4_LAUNCH_GEMM(R_, 3, OUT_, false) }                                               \
    else if (nt_tiles == 2) { BOF4_LAUNCH_GEMM(R_, 2, OUT_, false) } else { BOF4_LAUNCH_GEMM(R_, 1, OUT_, false) }
        if (P.x_in_place && n_outliers > 0) {  // (with a list only on matrices that take one tile of rows per wave)
            BOF4_LAUNCH_GEMM(1, 1, true, true)
        } else if (P.x_in_place) {
            if (per_wg_tiles == 2) { BOF4_LAUNCH_GEMM(2, 1, false, true) } else { BOF4_LAUNCH_GEMM(1, 1, false, true) }
        } else if (n_outliers > 0) {
            if (per_wg_tiles == 2) { BOF4_LAUNCH_GEMM_NT(2, true) } else { BOF4_LAUNCH_GEMM_NT(1, true) }
        } else {
            if (per_wg_tiles == 2) { BOF4_LAUNCH_GEMM_NT(2, false) } else { BOF4_LAUNCH_GEMM_NT(1, false) }
        }
#undef BOF4_LAUNCH_GEMM_NT
#undef BOF4_LAUNCH_GEMM
        if (split > 1) {
            if constexpr (Out::LAYER) {
                gemm_add_parts(split, nt, rows, to, s);
            } else {
                const uint64_t count = (uint64_t)nt * rows;
                hipLaunchKernelGGL(gemm_sum_kernel, dim3((uint32_t)((count + 255) / 256)), dim3(256), 0, s, part,
                                   part + count, split - 1, count, dst.first + (uint64_t)t0 * rows);
            }
        }
        tile0 += nt_tiles;
    }
    timing_end(s);
    HIP_TRY(hipGetLastError());
    return BOF4_OK;
}

struct GemvCall {
    const uint8_t* codes_dev;
    const uint16_t* scales_dev;
    uint64_t rows, cols;
    uint32_t block;
    const double* cb_host;
    const void* table_dev;
    uint64_t n_outliers;
    const void* x_dev;
    uint32_t n_tokens;
    hipStream_t stream;
};
template <class Out>
int gemv_run(const GemvCall& call, const Out& dst) {
    const auto [codes_dev, scales_dev, rows, cols, block, cb_host, table_dev, n_outliers, x_dev, n_tokens, s] = call;
    const uint64_t strips = (cols + GEMV_STRIP - 1) / GEMV_STRIP;
    const uint32_t* offsets_dev = (const uint32_t*)table_dev;
    const uint2* entries_dev =
        table_dev ? (const uint2*)((const char*)table_dev + gemv_table_layout(rows, strips, n_outliers).entries) : nullptr;
    const CodebookArgs cb = make_codebook_args(cb_host);
    uint32_t log2_block = 5;
    while ((1u << log2_block) < block) ++log2_block;
    const uint4* codes = (const uint4*)codes_dev;
    const uint16_t* x = (const uint16_t*)x_dev;
    timing_begin(s);
    for (uint32_t t0 = 0, nt; t0 < n_tokens; t0 += nt) {
        nt = n_tokens - t0 < GEMV_MAX_TOKENS ? n_tokens - t0 : GEMV_MAX_TOKENS;
        if (nt > 2 && rows * cols > gemv_most_weights(strips, nt, n_outliers > 0)) nt = 2;
        const uint16_t* xt = x + (uint64_t)t0 * cols;
        Out to = dst;
        if constexpr (Out::LAYER) to.token0 = t0;
        else to.first = dst.first + (uint64_t)t0 * rows;
        // with a list every wave keeps its slice of x in LDS as well
        const uint32_t waves = (uint32_t)(strips < GEMV_MAX_WAVES ? strips : GEMV_MAX_WAVES);
        const size_t lds = n_outliers > 0 ? (size_t)waves * GEMV_STRIP * 2 * nt : 0;
        // Rows per workgroup: every workgroup pays for its slice of x, the level table and two barriers, so the
        // rows are dealt out evenly over as many workgroups as the chip holds at once - one round, no tail - or, with more
        // than GEMV_MAX_RC rows for each of them, over full rounds (40000 x 8192, three tokens with a list, which hold two
        // workgroups per compute unit: 113 more workgroups than fit 185 us, two rounds 119).
        const int variant = 2 * (int)(nt - 1) + (n_outliers > 0 ? 1 : 0);
        const uint64_t slots = gemv_resident_workgroups<Out>(variant, 64 * waves, lds);
        if (slots == 0) return fail(BOF4_ERR_HIP, "bof4_gemv: occupancy query failed");
        const uint64_t rounds = (rows + slots * GEMV_MAX_RC - 1) / (slots * GEMV_MAX_RC);
        const uint64_t rc64 = (rows + slots * rounds - 1) / (slots * rounds);
        const uint32_t rc = (uint32_t)(rc64 < 4 ? 4 : rc64);
        const uint32_t grid = (uint32_t)((rows + rc - 1) / rc);
#define BOF4_LAUNCH_GEMV(T_, OUT_)                                                                                \
    hipLaunchKernelGGL((gemv_kernel<T_, OUT_, Out>), dim3(grid), dim3(64 * waves), lds, s, codes, scales_dev,          \
                       (uint32_t)rows, (uint32_t)cols, log2_block, rc, (uint32_t)strips, cb, offsets_dev,         \
                       entries_dev, (uint32_t)n_outliers, xt, to);
#define BOF4_LAUNCH_GEMV_NT(OUT_)                                                                                 \
    if (nt == 1) { BOF4_LAUNCH_GEMV(1, OUT_) } else if (nt == 2) { BOF4_LAUNCH_GEMV(2, OUT_) }                     \
    else if (nt == 3) { BOF4_LAUNCH_GEMV(3, OUT_) } else { BOF4_LAUNCH_GEMV(4, OUT_) }
        if (n_outliers > 0) { BOF4_LAUNCH_GEMV_NT(true) } else { BOF4_LAUNCH_GEMV_NT(false) }
#undef BOF4_LAUNCH_GEMV_NT
#undef BOF4_LAUNCH_GEMV
    }
    timing_end(s);
    HIP_TRY(hipGetLastError());
    return BOF4_OK;
}

}  // namespace bof4
