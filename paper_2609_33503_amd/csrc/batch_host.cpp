// Host side of the batched serving calls: validation, buffer sizing and carving, launches.

#include <math.h>
#include <stdint.h>

#include "batch.h"

using namespace relaxkv;

namespace {

constexpr size_t kAlign = 256;

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void* p) { return (uintptr_t)p % 16 == 0; }
int64_t elems16(const relaxkv_problem* p) { return p->dtype == RELAXKV_DTYPE_BF16 ? 8 : 4; }
relaxkv_status from_hip(hipError_t e) { return e == hipSuccess ? RELAXKV_OK : RELAXKV_EDEVICE; }

bool sizes_ok(const relaxkv_problem* p, int32_t n_seq, int32_t n_rows, int32_t max_suffix) {
    return n_seq >= 1 && n_seq <= RELAXKV_MAX_SEQS && n_rows >= 0 &&
           n_rows <= RELAXKV_MAX_BATCH_ROWS &&
           (int64_t)n_rows * p->H <= RELAXKV_MAX_BATCH_ROW_HEADS && max_suffix >= 1 &&
           max_suffix <= RELAXKV_MAX_TC;
}

struct BatchLayout {
    size_t row_off, rows, tiles, counts, total;
    int32_t tile_cap;
};

BatchLayout batch_layout(const relaxkv_problem* p, int32_t n_seq, int32_t n_rows) {
    BatchLayout l;
    l.tile_cap = (int32_t)batch_tile_cap(n_rows, p->H / p->H_kv, n_seq, batch_tile_rows(*p));
    l.row_off = align_up(((size_t)n_seq + 1) * 4);
    l.rows = align_up((size_t)n_rows * 4);
    l.tiles = align_up((size_t)l.tile_cap * sizeof(BatchTile));
    l.counts = align_up(kBatchSplitAt * 4 + sizeof(BatchSplit));
    l.total = l.row_off + 2 * l.rows + l.tiles + l.counts;
    return l;
}

// The problem is valid and b is a batch bound for its shape.
relaxkv_status batch_status(const relaxkv_problem* p, const relaxkv_batch* b) {
    const relaxkv_status st = relaxkv_validate(p);
    if (st != RELAXKV_OK) return st;
    if (!b || b->T_c != p->T_c || b->H != p->H || b->H_kv != p->H_kv || b->d != p->d ||
        b->dtype != p->dtype || !sizes_ok(p, b->n_seq, b->n_rows, b->max_suffix))
        return RELAXKV_EINVAL;
    if (!b->row_off || !b->row_seq || !b->row_pos || !b->tiles || !b->counts ||
        (uintptr_t)b->tiles % 16 || b->tile_cap != batch_layout(p, b->n_seq, b->n_rows).tile_cap)
        return RELAXKV_EINVAL;
    return RELAXKV_OK;
}

relaxkv_status suffix_status(const relaxkv_problem* p, const relaxkv_batch* b,
                             const relaxkv_suffix* s) {
    if (!s || !s->k || !s->v) return RELAXKV_EINVAL;
    if (s->stride_seq < 0 || s->stride_head < 0 || s->stride_token < 0) return RELAXKV_EINVAL;
    int64_t sT = s->stride_token ? s->stride_token : p->d, sH, sS;
    if (s->stride_head) sH = s->stride_head;
    else if (__builtin_mul_overflow((int64_t)b->max_suffix, sT, &sH)) return RELAXKV_EUNSUPPORTED;
    if (s->stride_seq) sS = s->stride_seq;
    else if (__builtin_mul_overflow((int64_t)p->H_kv, sH, &sS)) return RELAXKV_EUNSUPPORTED;
    StrideDim dims[3] = {{sT, b->max_suffix}, {sH, p->H_kv}, {sS, b->n_seq}};
    const relaxkv_status st = strides_nest(dims, p->d, elems16(p));
    if (st != RELAXKV_OK) return st;
    if (b->max_suffix > 1 && sT >= ((int64_t)1 << 24)) return RELAXKV_EUNSUPPORTED;
    if (!aligned(s->k) || !aligned(s->v)) return RELAXKV_EUNSUPPORTED;
    return RELAXKV_OK;
}

relaxkv_status rope_status(const relaxkv_problem* p, const relaxkv_rope* r,
                           const relaxkv_rows* in) {
    if (!r || !in || in->n_rows < 0) return RELAXKV_EINVAL;
    if (!(r->eps >= 0.f) || isinf(r->eps) || r->rot < 0 || r->rot > p->d ||
        (r->interleaved != 0 && r->interleaved != 1) || (r->rot > 0 && !r->inv_freq))
        return RELAXKV_EINVAL;
    if (r->rot % 16) return RELAXKV_EUNSUPPORTED;
    const struct { const void* x; int64_t stride, width; } rows[3] = {
        {in->q, in->q_stride, (int64_t)p->H * p->d},
        {in->k, in->k_stride, (int64_t)p->H_kv * p->d},
        {in->v, in->v_stride, (int64_t)p->H_kv * p->d}};
    for (const auto& x : rows) {
        if (!x.x) continue;
        if (x.stride != 0 && x.stride < x.width) return RELAXKV_EINVAL;
        if (x.stride % elems16(p) || !aligned(x.x)) return RELAXKV_EUNSUPPORTED;
        if (x.stride >= ((int64_t)1 << 40)) return RELAXKV_EUNSUPPORTED;
    }
    return RELAXKV_OK;
}

bool block_ok(int32_t block) { return block == 16 || block == 32 || block == 64 || block == 128; }

// A list length that the calls take.
relaxkv_status sel_status(const relaxkv_problem* p, int32_t block, int32_t n_sel) {
    if (!block_ok(block) || n_sel < 1 || n_sel > block_count(*p, block)) return RELAXKV_EINVAL;
    return n_sel > RELAXKV_MAX_SELECTED_BLOCKS ? RELAXKV_EUNSUPPORTED : RELAXKV_OK;
}

relaxkv_status attn(const relaxkv_problem* p, const relaxkv_batch* b, int32_t layer,
                    const void* k_cache, const void* v_cache, const void* q,
                    const relaxkv_suffix* suffix, int32_t block, const int32_t* blocks,
                    int32_t n_sel, void* out, float* lse_out, void* ws, size_t ws_bytes,
                    void* stream) {
    if (layer < 0 || layer >= p->L) return RELAXKV_EINVAL;
    relaxkv_status st = suffix_status(p, b, suffix);
    if (st != RELAXKV_OK) return st;
    if (!k_cache || !v_cache) return RELAXKV_EINVAL;
    if (b->n_rows > 0 && (!q || !out || (n_sel && !blocks))) return RELAXKV_EINVAL;
    if (!aligned(k_cache) || !aligned(v_cache) || !aligned(q) || !aligned(out))
        return RELAXKV_EUNSUPPORTED;
    const BatchAttnWorkspace w = batch_attn_layout(*p, *b, block, n_sel);
    if (w.total && !ws) return RELAXKV_EINVAL;
    if (ws_bytes < w.total) return RELAXKV_ENOSPACE;
    if ((uintptr_t)ws % 16) return RELAXKV_EUNSUPPORTED;
    if (b->n_rows == 0) return RELAXKV_OK;
    return from_hip(launch_batch_attn(*p, *b, layer, k_cache, v_cache, q, *suffix, block, blocks,
                                      n_sel, out, lse_out, (char*)ws, (hipStream_t)stream));
}

}  // namespace

extern "C" {

size_t relaxkv_batch_bytes(const relaxkv_problem* p, int32_t n_seq, int32_t n_rows,
                           int32_t max_suffix) {
    if (relaxkv_validate(p) != RELAXKV_OK || !sizes_ok(p, n_seq, n_rows, max_suffix)) return 0;
    return batch_layout(p, n_seq, n_rows).total;
}

relaxkv_status relaxkv_batch_bind(const relaxkv_problem* p, int32_t n_seq, int32_t n_rows,
                                  int32_t max_suffix, void* dev_buf, size_t bytes,
                                  relaxkv_batch* out) {
    const relaxkv_status st = relaxkv_validate(p);
    if (st != RELAXKV_OK) return st;
    if (!sizes_ok(p, n_seq, n_rows, max_suffix) || !dev_buf || !out) return RELAXKV_EINVAL;
    if ((uintptr_t)dev_buf % kAlign) return RELAXKV_EINVAL;
    const BatchLayout l = batch_layout(p, n_seq, n_rows);
    if (bytes < l.total) return RELAXKV_ENOSPACE;
    char* c = (char*)dev_buf;
    relaxkv_batch b;
    b.n_seq = n_seq;
    b.n_rows = n_rows;
    b.max_suffix = max_suffix;
    b.tile_cap = l.tile_cap;
    b.T_c = p->T_c;
    b.H = p->H;
    b.H_kv = p->H_kv;
    b.d = p->d;
    b.dtype = p->dtype;
    b.counts = (int32_t*)c; c += l.counts;
    b.row_off = (int32_t*)c; c += l.row_off;
    b.row_seq = (int32_t*)c; c += l.rows;
    b.row_pos = (int32_t*)c; c += l.rows;
    b.tiles = (int32_t*)c;
    *out = b;
    return RELAXKV_OK;
}

relaxkv_status relaxkv_batch_plan(const relaxkv_problem* p, const relaxkv_batch* b,
                                  const int32_t* past_len, const int32_t* new_len, void* stream) {
    const relaxkv_status st = batch_status(p, b);
    if (st != RELAXKV_OK) return st;
    if (!past_len || !new_len) return RELAXKV_EINVAL;
    return from_hip(launch_batch_plan(*p, *b, past_len, new_len, (hipStream_t)stream));
}

relaxkv_status relaxkv_batch_to_host(const relaxkv_batch* b, int32_t* host_counts, void* stream) {
    if (!b || !b->counts || !host_counts) return RELAXKV_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    hipError_t e = hipMemcpyAsync(host_counts, b->counts, 4 * sizeof(int32_t),
                                  hipMemcpyDeviceToHost, st);
    if (e == hipSuccess) e = hipStreamSynchronize(st);
    if (e != hipSuccess) return RELAXKV_EDEVICE;
    return host_counts[3] != 0 ? RELAXKV_EINVAL : RELAXKV_OK;
}

relaxkv_status relaxkv_fresh_rows(const relaxkv_problem* p, const relaxkv_rope* r,
                                  const relaxkv_rows* in, const int32_t* positions, void* q_out,
                                  void* k_out, void* v_out, void* stream) {
    relaxkv_status st = relaxkv_validate(p);
    if (st == RELAXKV_OK) st = rope_status(p, r, in);
    if (st != RELAXKV_OK) return st;
    if (!in->q != !q_out || !in->k != !k_out || !in->v != !v_out) return RELAXKV_EINVAL;
    if (in->n_rows > RELAXKV_MAX_FRESH_ROWS) return RELAXKV_EUNSUPPORTED;
    if (!aligned(q_out) || !aligned(k_out) || !aligned(v_out)) return RELAXKV_EUNSUPPORTED;
    if (in->n_rows == 0 || (!in->q && !in->k && !in->v)) return RELAXKV_OK;
    if (!positions) return RELAXKV_EINVAL;
    return from_hip(launch_norm_rope(*p, *r, *in, positions, nullptr, q_out, k_out, v_out,
                                     SuffixStrides{}, (hipStream_t)stream));
}

relaxkv_status relaxkv_batch_rows(const relaxkv_problem* p, const relaxkv_rope* r,
                                  const relaxkv_batch* b, const relaxkv_rows* in, void* q_out,
                                  const relaxkv_suffix* suffix, void* stream) {
    relaxkv_status st = batch_status(p, b);
    if (st == RELAXKV_OK) st = rope_status(p, r, in);
    if (st != RELAXKV_OK) return st;
    if (in->n_rows != b->n_rows || !in->q != !q_out) return RELAXKV_EINVAL;
    if (!aligned(q_out)) return RELAXKV_EUNSUPPORTED;
    st = suffix_status(p, b, suffix);
    if (st != RELAXKV_OK) return st;
    if (in->n_rows == 0 || (!in->q && !in->k && !in->v)) return RELAXKV_OK;
    return from_hip(launch_norm_rope(*p, *r, *in, nullptr, b, q_out, suffix->k, suffix->v,
                                     suffix_strides(*p, *b, *suffix), (hipStream_t)stream));
}

size_t relaxkv_shared_attn_workspace_bytes(const relaxkv_problem* p, const relaxkv_batch* b) {
    if (batch_status(p, b) != RELAXKV_OK) return 0;
    return batch_attn_layout(*p, *b, 0, 0).total;
}

relaxkv_status relaxkv_shared_attn(const relaxkv_problem* p, const relaxkv_batch* b, int32_t layer,
                                   const void* k_cache, const void* v_cache, const void* q,
                                   const relaxkv_suffix* suffix, void* out, float* lse_out,
                                   void* ws, size_t ws_bytes, void* stream) {
    const relaxkv_status st = batch_status(p, b);
    if (st != RELAXKV_OK) return st;
    return attn(p, b, layer, k_cache, v_cache, q, suffix, 0, nullptr, 0, out, lse_out, ws, ws_bytes,
                stream);
}

relaxkv_status relaxkv_block_means(const relaxkv_problem* p, int32_t layer, const void* k_cache,
                                   int32_t block, void* means, void* stream) {
    const relaxkv_status st = relaxkv_validate(p);
    if (st != RELAXKV_OK) return st;
    if (layer < -1 || layer >= p->L || !block_ok(block) || !k_cache || !means) return RELAXKV_EINVAL;
    if (!aligned(k_cache) || !aligned(means)) return RELAXKV_EUNSUPPORTED;
    return from_hip(launch_block_means(*p, layer < 0 ? 0 : layer, layer < 0 ? p->L : 1, k_cache,
                                       block, means, (hipStream_t)stream));
}

size_t relaxkv_block_select_workspace_bytes(const relaxkv_problem* p, const relaxkv_batch* b,
                                            int32_t block) {
    if (batch_status(p, b) != RELAXKV_OK || !block_ok(block)) return 0;
    return block_select_bytes(*p, *b, block);
}

relaxkv_status relaxkv_block_select(const relaxkv_problem* p, const relaxkv_batch* b, int32_t block,
                                    const void* means, const void* q, int32_t n_sel,
                                    int32_t* blocks, void* ws, size_t ws_bytes, void* stream) {
    relaxkv_status st = batch_status(p, b);
    if (st == RELAXKV_OK) st = sel_status(p, block, n_sel);
    if (st != RELAXKV_OK) return st;
    if (!means || (b->n_rows > 0 && (!q || !blocks || !ws))) return RELAXKV_EINVAL;
    if (!aligned(means) || !aligned(q) || (uintptr_t)ws % 16) return RELAXKV_EUNSUPPORTED;
    if (ws_bytes < block_select_bytes(*p, *b, block)) return RELAXKV_ENOSPACE;
    if (b->n_rows == 0) return RELAXKV_OK;
    return from_hip(launch_block_select(*p, *b, block, means, q, n_sel, blocks, (float*)ws,
                                        (hipStream_t)stream));
}

size_t relaxkv_block_attn_workspace_bytes(const relaxkv_problem* p, const relaxkv_batch* b,
                                          int32_t block, int32_t n_sel) {
    if (batch_status(p, b) != RELAXKV_OK || sel_status(p, block, n_sel) != RELAXKV_OK) return 0;
    return batch_attn_layout(*p, *b, block, n_sel).total;
}

relaxkv_status relaxkv_block_attn(const relaxkv_problem* p, const relaxkv_batch* b, int32_t layer,
                                  const void* k_cache, const void* v_cache, int32_t block,
                                  const int32_t* blocks, int32_t n_sel, const void* q,
                                  const relaxkv_suffix* suffix, void* out, float* lse_out,
                                  void* ws, size_t ws_bytes, void* stream) {
    relaxkv_status st = batch_status(p, b);
    if (st == RELAXKV_OK) st = sel_status(p, block, n_sel);
    if (st != RELAXKV_OK) return st;
    return attn(p, b, layer, k_cache, v_cache, q, suffix, block, blocks, n_sel, out, lse_out, ws,
                ws_bytes, stream);
}

}  // extern "C"
