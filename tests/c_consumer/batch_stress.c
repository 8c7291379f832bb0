/*
 * Host-side stress of the batched serving calls for the sanitizer build (test
 * infrastructure): over problem shapes and batch sizes, up to the limits the
 * header states, it calls the size queries and the binding, checks the carved
 * pointers, and calls every compute entry point with an argument that must be
 * rejected before anything is enqueued.  No call reaches a device.  Prints
 * "ok <checks>" and exits 0 when every check holds.
 */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "relaxkv.h"

static long n_checks = 0;

#define EXPECT(cond)                                                           \
    do {                                                                       \
        ++n_checks;                                                            \
        if (!(cond)) {                                                         \
            fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #cond); \
            exit(1);                                                           \
        }                                                                      \
    } while (0)

static void* at(uintptr_t a) { return (void*)a; }

static relaxkv_problem make(int T, int H, int Hkv, int d, int dtype) {
    relaxkv_problem p;
    memset(&p, 0, sizeof p);
    p.L = 2;
    p.T_c = T;
    p.n_query = 1;
    p.H = H;
    p.H_kv = Hkv;
    p.d = d;
    p.dtype = dtype;
    p.anchor_ratio = 0.15;
    p.q = at(0x1000);
    p.k_cache = at(0x2000);
    p.v_cache = at(0x3000);
    return p;
}

static void check_inside(const void* ptr, size_t n, uintptr_t base, size_t bytes) {
    const uintptr_t a = (uintptr_t)ptr;
    EXPECT(a % 256 == 0);
    EXPECT(a >= base && a - base <= bytes && n <= bytes - (a - base));
}

static void one(const relaxkv_problem* p, int n_seq, int n_rows, int room) {
    const int ok = n_seq >= 1 && n_seq <= RELAXKV_MAX_SEQS && n_rows >= 0 && n_rows <= RELAXKV_MAX_BATCH_ROWS &&
                   (int64_t)n_rows * p->H <= RELAXKV_MAX_BATCH_ROW_HEADS && room >= 1 && room <= RELAXKV_MAX_TC;
    const size_t bytes = relaxkv_batch_bytes(p, n_seq, n_rows, room);
    EXPECT((bytes > 0) == (ok && relaxkv_validate(p) == RELAXKV_OK));
    relaxkv_batch b;
    memset(&b, 0x5a, sizeof b);
    if (!bytes) {
        EXPECT(relaxkv_batch_bind(p, n_seq, n_rows, room, at(0x100000), 1u << 30, &b) < 0);
        return;
    }
    const uintptr_t base = 0x100000;
    EXPECT(relaxkv_batch_bind(p, n_seq, n_rows, room, at(base), bytes - 1, &b) == RELAXKV_ENOSPACE);
    EXPECT(relaxkv_batch_bind(p, n_seq, n_rows, room, at(base + 4), bytes, &b) == RELAXKV_EINVAL);
    EXPECT(relaxkv_batch_bind(p, n_seq, n_rows, room, NULL, bytes, &b) == RELAXKV_EINVAL);
    EXPECT(relaxkv_batch_bind(p, n_seq, n_rows, room, at(base), bytes, NULL) == RELAXKV_EINVAL);
    EXPECT(relaxkv_batch_bind(p, n_seq, n_rows, room, at(base), bytes, &b) == RELAXKV_OK);
    check_inside(b.counts, 64 * 4, base, bytes);
    check_inside(b.row_off, ((size_t)n_seq + 1) * 4, base, bytes);
    check_inside(b.row_seq, (size_t)n_rows * 4, base, bytes);
    check_inside(b.row_pos, (size_t)n_rows * 4, base, bytes);
    EXPECT(b.tile_cap >= 0);
    check_inside(b.tiles, (size_t)b.tile_cap * 32, base, bytes);

    relaxkv_suffix s;
    memset(&s, 0, sizeof s);
    s.k = at(0x5000);
    s.v = at(0x6000);
    relaxkv_rope r;
    memset(&r, 0, sizeof r);
    r.eps = 1e-6f;
    relaxkv_rows in;
    memset(&in, 0, sizeof in);
    in.q = at(0x7000);
    in.n_rows = n_rows;
    void *q = at(0x8000), *out = at(0x9000), *ws = at(0xa000);

    /* (suffix caches of more than 2^48 elements are refused before the rest) */
    const int fits = (double)n_seq * p->H_kv * room * p->d <= 281474976710656.0;

    const size_t sw = relaxkv_shared_attn_workspace_bytes(p, &b);
    EXPECT((sw > 0) == (n_rows > 0));
    /* (at least the partial rows of one split) */
    if (p->dtype == RELAXKV_DTYPE_BF16 && n_rows) EXPECT(sw >= 2 * (size_t)n_rows * p->H * (p->d * 2 + 16));
    if (sw) EXPECT(relaxkv_shared_attn(p, &b, 0, q, q, q, &s, out, NULL, ws, sw - 1, NULL) ==
                   (fits ? RELAXKV_ENOSPACE : RELAXKV_EUNSUPPORTED));
    EXPECT(relaxkv_shared_attn(p, &b, 2, q, q, q, &s, out, NULL, ws, sw, NULL) == RELAXKV_EINVAL);
    EXPECT(relaxkv_shared_attn(p, &b, 0, NULL, q, q, &s, out, NULL, ws, sw, NULL) ==
           (fits ? RELAXKV_EINVAL : RELAXKV_EUNSUPPORTED));
    EXPECT(relaxkv_shared_attn(p, &b, 0, at(0x2004), q, q, &s, out, NULL, ws, sw, NULL) == RELAXKV_EUNSUPPORTED);
    EXPECT(relaxkv_batch_plan(p, &b, NULL, at(0x4000), NULL) == RELAXKV_EINVAL);
    EXPECT(relaxkv_batch_rows(p, &r, &b, &in, NULL, &s, NULL) == RELAXKV_EINVAL);
    if (n_rows) EXPECT(relaxkv_fresh_rows(p, &r, &in, NULL, out, NULL, NULL, NULL) == RELAXKV_EINVAL);
    s.stride_seq = INT64_MAX;
    EXPECT(n_seq == 1 || relaxkv_shared_attn(p, &b, 0, q, q, q, &s, out, NULL, ws, sw, NULL) < 0);
    s.stride_seq = 0;
    s.stride_head = INT64_MAX / 2;
    EXPECT(p->H_kv == 1 || relaxkv_shared_attn(p, &b, 0, q, q, q, &s, out, NULL, ws, sw, NULL) < 0);
    s.stride_head = 0;
    s.stride_token = INT64_MAX / 4 * 4;
    EXPECT(room == 1 || relaxkv_shared_attn(p, &b, 0, q, q, q, &s, out, NULL, ws, sw, NULL) < 0);
    s.stride_token = 0;

    const int blocks[] = {16, 32, 64, 128};
    for (int i = 0; i < 4; ++i) {
        const int nb = (p->T_c + blocks[i] - 1) / blocks[i];
        const size_t need = relaxkv_block_select_workspace_bytes(p, &b, blocks[i]);
        EXPECT(need >= (size_t)n_rows * p->H_kv * nb * 4);
        if (n_rows)
            EXPECT(relaxkv_block_select(p, &b, blocks[i], q, q, 1, at(0xb000), ws, need - 1, NULL) == RELAXKV_ENOSPACE);
        const int sels[] = {0, 1, nb, nb + 1, RELAXKV_MAX_SELECTED_BLOCKS, RELAXKV_MAX_SELECTED_BLOCKS + 1, INT32_MAX};
        for (int j = 0; j < 7; ++j) {
            const int good = sels[j] >= 1 && sels[j] <= nb && sels[j] <= RELAXKV_MAX_SELECTED_BLOCKS;
            const size_t w = relaxkv_block_attn_workspace_bytes(p, &b, blocks[i], sels[j]);
            EXPECT((w > 0) == (good && n_rows > 0));
            const relaxkv_status st = relaxkv_block_attn(p, &b, 0, q, q, blocks[i], at(0xb000), sels[j], q, &s,
                                                         out, NULL, NULL, 0, NULL);
            EXPECT(good && !fits ? st == RELAXKV_EUNSUPPORTED
                   : good ? (n_rows ? st == RELAXKV_EINVAL : st == RELAXKV_OK)
                        : st == RELAXKV_EINVAL || st == RELAXKV_EUNSUPPORTED);
        }
        EXPECT(relaxkv_block_means(p, -2, q, blocks[i], out, NULL) == RELAXKV_EINVAL);
        EXPECT(relaxkv_block_means(p, 2, q, blocks[i], out, NULL) == RELAXKV_EINVAL);
    }
    EXPECT(relaxkv_block_means(p, 0, q, 48, out, NULL) == RELAXKV_EINVAL);
    EXPECT(relaxkv_block_select_workspace_bytes(p, &b, 0) == 0);
    b.tile_cap += 1;
    EXPECT(relaxkv_shared_attn_workspace_bytes(p, &b) == 0);
}

int main(void) {
    const int Ts[] = {1, 15, 64, 1000, 32768, 1 << 20, RELAXKV_MAX_TC};
    const int heads[][2] = {{1, 1}, {8, 2}, {40, 8}, {64, 64}, {200, 1}};
    const int seqs[] = {-1, 0, 1, 3, 64, 4096, RELAXKV_MAX_SEQS, RELAXKV_MAX_SEQS + 1, INT32_MAX};
    const int rows[] = {-1, 0, 1, 5, 320, 20000, RELAXKV_MAX_BATCH_ROWS, RELAXKV_MAX_BATCH_ROWS + 1, INT32_MAX};
    const int rooms[] = {0, 1, 700, RELAXKV_MAX_TC, RELAXKV_MAX_TC + 1};
    for (size_t t = 0; t < sizeof Ts / sizeof *Ts; ++t)
        for (size_t h = 0; h < sizeof heads / sizeof *heads; ++h)
            for (int d = 64; d <= 128; d += 64)
                for (int dt = 0; dt < 2; ++dt) {
                    const relaxkv_problem p = make(Ts[t], heads[h][0], heads[h][1], d,
                                                   dt ? RELAXKV_DTYPE_BF16 : RELAXKV_DTYPE_F32);
                    for (size_t i = 0; i < sizeof seqs / sizeof *seqs; ++i)
                        for (size_t j = 0; j < sizeof rows / sizeof *rows; ++j)
                            for (size_t k = 0; k < sizeof rooms / sizeof *rooms; ++k)
                                one(&p, seqs[i], rows[j], rooms[k]);
                }
    printf("ok %ld\n", n_checks);
    return 0;
}
