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

// Scratch of the bf16 batched attention: per key split, KV head and (token, head) row the
// unnormalised output (float32) and (running max, sum of the rounded probabilities, sum of
// the exact ones, -).
struct BatchAttnWorkspace {
    size_t part_s_off;  // float4 [n_ctx + n_suf][H_kv][n_rows * G]; the outputs lie at 0
    size_t total;
    int n_ctx, kps;     // splits of the context keys (listed keys for the blocks), keys each
    int n_suf, kss;     // splits of the suffix keys, keys each
    int n_chunks;       // row chunks of kBatchRowsBf16 (of all rows; of one token's group)
};

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
