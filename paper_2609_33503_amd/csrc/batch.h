// Internal declarations of the batched serving calls (row maps of a step, norm and
// rotation, attention of many requests over one context cache).
#pragma once

#include "internal.h"

namespace relaxkv {

// (token, head) rows of one request that a suffix workgroup takes: four 32-row MFMA
// blocks in bf16, one 16-row block of the float32 core.
constexpr int kBatchRowsBf16 = 128;
constexpr int kBatchRowsF32 = 16;
inline int batch_tile_rows(const relaxkv_problem& p) {
    return p.dtype == RELAXKV_DTYPE_BF16 ? kBatchRowsBf16 : kBatchRowsF32;
}

// A request has ceil(new * G / rows) tiles: at most a full one per `rows` rows of the step
// and one more for each request that has a row.
inline int64_t batch_tile_cap(int64_t rows, int64_t G, int64_t n_seq, int64_t tile_rows) {
    return rows * G / tile_rows + (n_seq < rows ? n_seq : rows);
}

// One row tile of a step (two 16-byte loads): its request, the request's first row and
// number of new rows, its tokens before the step, and the tile's first (token, head) row
// within the request.
struct alignas(16) BatchTile {
    int32_t seq, row_begin, n_new, past;
    int32_t row0, pad[3];
};

// How the bf16 attention of a step is split, computed by the plan (which knows the step) and
// kept behind the public counts.
constexpr int kBaRows = kBatchRowsBf16;
constexpr int kBaKeys = 32;            // keys per tile
constexpr int kBaWgs = 768;            // workgroups the splits aim for (three per CU)
constexpr int kBaItemWgs = 512;        // of them for context items that one worker has alone
constexpr int kBaMinTiles = 8;         // fewest tiles per split
constexpr int kBaXcds = 8;
constexpr int kBaLongSuffix = 1024;    // tokens from which the suffix items go first
// float32: workgroups of 8 waves, listed 4, so that two or four share a CU and one's start and end
// pass beside another's keys (33 requests of 4 rows, 3 heads, over 2097 keys: 15.4 us, 21.4 with 16
// waves, 14.8 and a longer merge with 4; 65 rows of 8 heads over 200 listed and suffix keys: 18.3,
// 20.5 with 8, 29.0 with 16).  A split's keys are at least one 16-key block for each wave.  Shared:
// up to kBaF32More splits more where as many as kBaF32Items items leave places of the last round
// idle (64 requests of 5 rows, 8 heads, over 32K: 526-543 us, 778 without).
constexpr int kBaF32Waves = 8, kBaF32ListWaves = 4;
constexpr int kBaF32Keys = 16 * kBaF32Waves, kBaF32ListKeys = 16 * kBaF32ListWaves;
constexpr int kBaF32Wgs = 256, kBaF32ListWgs = 512, kBaF32Items = 512, kBaF32More = 3;
// Workgroups of several splits: below kBaF32Wgs items at most kBaF32Wgs and kBaF32More per item.  Above,
// n splits of an item are taken only where their rounds r of kBaF32Wgs workgroups are fewer than
// 2 n, those of one split each (r (units / n + 1) < 2 (units + 1)), so they are at most 2 n - 1 rounds:
// seven with four splits.
constexpr int kBaF32Parts = kBaF32Wgs + kBaF32More * kBaF32Items;
static_assert(kBaF32Items == 2 * kBaF32Wgs && kBaF32Parts >= (2 * (kBaF32More + 1) - 1) * kBaF32Wgs &&
                  kBaF32Parts >= (1 + kBaF32More) * kBaF32Wgs,
              "the splits of every step fit");
constexpr int kBatchSplitAt = 16;      // first word of the split in relaxkv_batch::counts

// Shared context: item (g, chunk) = g * chunks + chunk holds `tiles` key tiles, worker w takes
// the tiles [w * quota, (w + 1) * quota) of the items laid one after another.  Where every item
// gets several workers, the items are padded to a whole number of quotas (len), so a worker
// has one item and the chunks of a key range run side by side on one XCD, whose L2 then
// serves all but the first (64 decoding requests over 32K: 32 workers per item).  With fewer
// workers per item the padding would idle a large part of them (20 ragged questions over 8K: 4
// per item), so there the workers cut the items anywhere, one worker's range covering
// parts of several.
struct BatchSplit {
    int32_t rows, row_tiles;           // of the step
    int32_t chunks, items, tiles, len, quota, workers;
    int32_t per_item;                  // workers of an item; 0: cut anywhere
    int32_t suffix_first;              // order of the items in the launch
    int32_t suf_n, suf_kps;            // suffix splits, keys each
    int32_t f32_n, f32_kps;            // float32: splits of the context, keys each
    int32_t f32_sn, f32_skps;          // and of a row tile's suffix
};

// Splits n of `tiles` key tiles, `quota` (at least `least`) tiles each, so that `items` of them
// are about `wgs` workgroups.
__host__ __device__ inline void batch_split_keys(int tiles, int items, int wgs, int least, int& n,
                                                 int& quota) {
    const int want = items >= wgs ? 1 : wgs / (items > 0 ? items : 1);
    quota = (tiles + want - 1) / want;
    quota = quota < least ? least : quota;
    n = tiles > 0 ? (tiles + quota - 1) / quota : 1;
}

__host__ __device__ inline BatchSplit batch_split(int rows, int row_tiles, int longest, int T, int G,
                                                  int Hkv) {
    BatchSplit s;
    s.rows = rows;
    s.row_tiles = row_tiles;
    s.chunks = (rows * G + kBaRows - 1) / kBaRows;
    s.items = s.chunks * Hkv;
    s.tiles = (T + kBaKeys - 1) / kBaKeys;
    const int most = (s.tiles + kBaMinTiles - 1) / kBaMinTiles;
    // One chunk of rows is bound by memory, and one workgroup per CU streams better than three
    // with a third of the keys (1-16 requests over 32K: 34-40 us, 38-44).  Several chunks take
    // two per CU and leave the third place to the suffix items, which then run beside them (with
    // suffixes of 300 tokens: 160 rows over 32K 52 us, 56 with three; 384 rows 80, 88; 640 rows 131,
    // 145; 320 rows over 8K 40, 46; without suffixes 320 rows over 32K 67, 68).
    const int wgs = s.chunks == 1 ? kBaWgs / 3 : kBaItemWgs;
    int n = s.items > 0 ? wgs / s.items : 0;
    n = n < most ? n : most;
    // (whole rounds of the XCDs)
    while (n > 0 && (n * Hkv + kBaXcds - 1) / kBaXcds * kBaXcds * s.chunks > wgs) --n;
    s.per_item = n >= 6 || n == most ? n : 0;
    if (s.per_item) {
        s.quota = (s.tiles + n - 1) / n;
        s.len = n * s.quota;
        s.workers = s.items * n;
    } else {
        const int64_t all = (int64_t)s.items * s.tiles;
        const int64_t q = (all + kBaWgs - 1) / kBaWgs;
        s.quota = q < kBaMinTiles ? kBaMinTiles : (int32_t)q;
        s.len = s.tiles;
        s.workers = (int32_t)((all + s.quota - 1) / s.quota);
    }
    // Long suffixes are bound by memory, several chunks of rows by computation: the suffix items
    // go first, so that the two overlap (64 requests of 5 rows with 3000 suffix tokens over 32K: 189
    // us, 210 with them last; 128 of 4 rows with 1500 over 8K: 155, 168); short ones go last,
    // behind the longer items (64 with up to 700 over 32K: 68, 72 first).
    s.suffix_first = s.chunks > 1 && longest >= kBaLongSuffix;
    int quota;
    batch_split_keys((longest + kBaKeys - 1) / kBaKeys, row_tiles * Hkv, kBaWgs, kBaMinTiles, s.suf_n,
                     quota);
    s.suf_kps = quota * kBaKeys;
    // A workgroup takes about as long as its units of kBaF32Keys keys and one more.
    auto f32_split = [&](int keys, int items, int& n, int& kps) {
        const int units = (keys + kBaF32Keys - 1) / kBaF32Keys;
        batch_split_keys(units, items, kBaF32Wgs, 1, n, kps);
        const int least = n, more = items <= kBaF32Items ? kBaF32More : 0;
        int best = (n * items + kBaF32Wgs - 1) / kBaF32Wgs * (kps + 1);
        for (int i = least + 1; i <= least + more && i <= units; ++i) {
            const int quota = (units + i - 1) / i, m = (units + quota - 1) / quota;
            const int cost = (m * items + kBaF32Wgs - 1) / kBaF32Wgs * (quota + 1);
            if (cost < best) {
                best = cost;
                n = m;
                kps = quota;
            }
        }
        kps *= kBaF32Keys;
    };
    f32_split(T, (rows * G + kBatchRowsF32 - 1) / kBatchRowsF32 * Hkv, s.f32_n, s.f32_kps);
    f32_split(longest, row_tiles * Hkv, s.f32_sn, s.f32_skps);
    return s;
}

// Scratch of the bf16 batched attention: partial rows of 16-bit outputs, and 16 bytes of
// statistics each; those of the suffix items follow the context's.
struct BatchAttnWorkspace {
    size_t part_s_off;  // the statistics; the outputs lie at 0
    size_t total;
    size_t suf_part;    // first partial row of the suffix items
    int ctx_wgs, suf_wgs;
};

// n_sel = 0: the whole context.
BatchAttnWorkspace batch_attn_layout(const relaxkv_problem& p, const relaxkv_batch& b, int block,
                                     int n_sel);
size_t block_select_bytes(const relaxkv_problem& p, const relaxkv_batch& b, int block);

inline int block_count(const relaxkv_problem& p, int block) { return (p.T_c + block - 1) / block; }

struct SuffixStrides {
    int64_t seq, head, token;
};
inline SuffixStrides suffix_strides(const relaxkv_problem& p, const relaxkv_batch& b,
                                    const relaxkv_suffix& s) {
    SuffixStrides r;
    r.token = s.stride_token ? s.stride_token : p.d;
    r.head = s.stride_head ? s.stride_head : (int64_t)b.max_suffix * r.token;
    r.seq = s.stride_seq ? s.stride_seq : (int64_t)p.H_kv * r.head;
    return r;
}

hipError_t launch_batch_plan(const relaxkv_problem& p, const relaxkv_batch& b,
                             const int32_t* past_len, const int32_t* new_len, hipStream_t st);
// Dense outputs at explicit positions (batch null), or a batch's rows (positions null).
hipError_t launch_norm_rope(const relaxkv_problem& p, const relaxkv_rope& r,
                            const relaxkv_rows& in, const int32_t* positions,
                            const relaxkv_batch* b, void* q_out, void* k_out, void* v_out,
                            SuffixStrides ss, hipStream_t st);
hipError_t launch_block_means(const relaxkv_problem& p, int layer, int n_layers,
                              const void* k_cache, int block, void* means, hipStream_t st);
hipError_t launch_block_select(const relaxkv_problem& p, const relaxkv_batch& b, int block,
                               const void* means, const void* q, int n_sel, int32_t* blocks,
                               float* scores, hipStream_t st);
// n_sel = 0: the whole context (blocks null).
hipError_t launch_batch_attn(const relaxkv_problem& p, const relaxkv_batch& b, int layer,
                             const void* k_cache, const void* v_cache, const void* q,
                             const relaxkv_suffix& suf, int block, const int32_t* blocks, int n_sel,
                             void* out, float* lse_out, char* ws, hipStream_t st);

}  // namespace relaxkv
