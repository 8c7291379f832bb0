// Launch sizes of the batched serving calls, on the host (test infrastructure).  The program's own
// launch functions take the place of the runtime's: they record each launch's grid and start
// nothing, so the entry points run here as a caller runs them, with addresses that are never read.
//
//   batch_launches steps N   N random steps: every workgroup and partial row that the split of the
//                            step's plan needs is launched and has room in the workspace.
//   batch_launches fresh     fresh_rows up to the header's largest number of rows: the grid is one that
//                            the hardware takes (fewer than 2^32 threads in a dimension).
//   batch_launches batch     the same of the batched calls at the header's most rows, heads and requests.
//   batch_launches select    block_select takes one launch where that is the faster form.
//
// Prints "ok <checks>" and exits 0 when every check holds.

#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <vector>

#include "batch.h"

using namespace relaxkv;

namespace {

struct Launch {
    dim3 grid, block;
};
std::vector<Launch> launches;
long n_checks = 0, n_bad = 0;

void expect(bool ok, const char* what) {
    ++n_checks;
    if (ok) return;
    if (++n_bad <= 20) fprintf(stderr, "check failed: %s\n", what);
}

void* at(uintptr_t a) { return (void*)a; }

uint64_t state = 88172645463325252ull;
uint64_t next() {
    state ^= state << 13;
    state ^= state >> 7;
    state ^= state << 17;
    return state;
}
// An integer of [lo, hi], spread over its logarithm.
int spread(int lo, int hi) {
    const double u = (double)(next() >> 11) / 9007199254740992.0;
    return std::min(hi, (int)(lo * pow((double)(hi + 1) / lo, u)));
}

relaxkv_problem make(int T, int H, int Hkv, int d, int dtype) {
    relaxkv_problem p;
    memset(&p, 0, sizeof p);
    p.L = 1;
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

relaxkv_batch bind(const relaxkv_problem& p, int n_seq, int n_rows, int room) {
    relaxkv_batch b;
    memset(&b, 0, sizeof b);
    const size_t bytes = relaxkv_batch_bytes(&p, n_seq, n_rows, room);
    expect(bytes > 0 && relaxkv_batch_bind(&p, n_seq, n_rows, room, at(1ull << 40), bytes, &b) == RELAXKV_OK,
           "bind");
    return b;
}

constexpr size_t kAll = (size_t)1 << 60;               // workspace bytes that hold everything
const relaxkv_suffix kSuffix = {(void*)0x5000, (void*)0x6000, 0, 0, 0};

long first_wgs() {
    if (launches.empty()) return 0;
    const dim3 g = launches[0].grid;
    return (long)g.x * g.y * g.z;
}

// One step of `news` new tokens behind `past` ones, in a batch with `more` rows and `room` suffix
// tokens beyond its own.
void step(const relaxkv_problem& p, const std::vector<int>& past, const std::vector<int>& news, int more,
          int room, int block, int n_sel) {
    const int G = p.H / p.H_kv, tile = batch_tile_rows(p);
    long rows = 0, tiles = 0;
    int longest = 0;
    for (size_t i = 0; i < news.size(); ++i) {
        rows += news[i];
        tiles += ((long)news[i] * G + tile - 1) / tile;
        if (news[i]) longest = std::max(longest, past[i] + news[i]);
    }
    const relaxkv_batch b = bind(p, (int)news.size(), (int)rows + more, longest + room);
    const BatchSplit s = batch_split((int)rows, (int)tiles, longest, p.T_c, G, p.H_kv);
    const bool f32 = p.dtype == RELAXKV_DTYPE_F32;
    char what[400];
    auto check = [&](const char* kind, long need, long have) {
        snprintf(what, sizeof what,
                 "%s: needs %ld, has %ld (dtype %d, T %d, H %d, H_kv %d, %zu requests, %ld + %d rows, "
                 "longest %d + %d, block %d, n_sel %d)",
                 kind, need, have, p.dtype, p.T_c, p.H, p.H_kv, news.size(), rows, more, longest, room,
                 block, n_sel);
        expect(need <= have, what);
    };
    const long chunk = f32 ? kBatchRowsF32 : kBaRows, per_row = f32 ? p.d * 4 + 4 : 0;
    for (int list = 0; list < 2; ++list) {
        const BatchAttnWorkspace w = batch_attn_layout(p, b, list ? block : 0, list ? n_sel : 0);
        launches.clear();
        const relaxkv_status st =
            list ? relaxkv_block_attn(&p, &b, 0, at(0x2000), at(0x3000), block, (int32_t*)at(0x7000), n_sel,
                                      at(0x4000), &kSuffix, at(0x8000), nullptr, at(1 << 20), w.total, nullptr)
                 : relaxkv_shared_attn(&p, &b, 0, at(0x2000), at(0x3000), at(0x4000), &kSuffix, at(0x8000),
                                       nullptr, at(1 << 20), w.total, nullptr);
        expect(st == RELAXKV_OK, "status");
        const long have = first_wgs(), list_items = rows * p.H_kv * ((G + chunk - 1) / chunk);
        if (f32 && !list) {
            check("float32 workgroups", (rows * G + chunk - 1) / chunk * p.H_kv * s.f32_n + tiles * p.H_kv * s.f32_sn,
                  have);
            check("float32 partial rows", (long)(s.f32_n + s.f32_sn) * rows * p.H, w.total / per_row);
        } else if (f32) {
            int n, kps;
            batch_split_keys((n_sel * block + kBaF32ListKeys - 1) / kBaF32ListKeys +
                                 (longest + kBaF32ListKeys - 1) / kBaF32ListKeys,
                             (int)list_items, kBaF32ListWgs, 1, n, kps);
            check("listed float32 workgroups", list_items * n, have);
            if (n > 1) check("listed float32 partial rows", n * rows * p.H, w.total / per_row);
        } else {
            check("workgroups", w.ctx_wgs + w.suf_wgs, have);
            check("suffix workgroups", tiles * p.H_kv * s.suf_n, w.suf_wgs);
            long ctx_rows = 0;
            if (list) {
                int n, kps;
                batch_split_keys((n_sel * block + kBaKeys - 1) / kBaKeys, (int)list_items, kBaWgs, kBaMinTiles, n,
                                 kps);
                check("listed workgroups", list_items * n, w.ctx_wgs);
                ctx_rows = n * rows * p.H;
            } else {
                check("context workgroups",
                      s.per_item ? (long)(s.per_item * p.H_kv + kBaXcds - 1) / kBaXcds * kBaXcds * s.chunks
                                 : s.workers,
                      w.ctx_wgs);
                ctx_rows = (long)(s.workers + s.items) * kBaRows;
            }
            check("context partial rows", ctx_rows, w.suf_part);
            // (the statistics take 16 bytes a row at most and end the workspace)
            check("suffix partial rows", w.suf_part + s.suf_n * rows * p.H, (w.total - w.part_s_off) / 16);
        }
    }
}

void steps(long n) {
    // One prompt of 112 rows on 64 / 8 heads; and ragged steps.
    step(make(4096, 64, 8, 64, 0), {0}, {112}, 0, 8, 64, 4);
    for (long i = 0; i < n; ++i) {
        const int Hkv = spread(1, 16), G = spread(1, 16), dtype = next() % 4 == 0;
        const int T = spread(1, 40000), n_seq = spread(1, 64);
        std::vector<int> past, news;
        const int most = spread(1, 150), before = spread(1, 500);
        for (int b = 0; b < n_seq; ++b) {
            past.push_back((int)(next() % (before + 1)));
            news.push_back(next() % 8 == 0 ? 0 : 1 + (int)(next() % most));
        }
        news[0] = most;
        const int block = 16 << next() % 4, nb = (T + block - 1) / block;
        step(make(T, Hkv * G, Hkv, next() % 2 ? 64 : 128, dtype), past, news,
             next() % 2 ? 0 : spread(1, 200), next() % 2 ? 1 : spread(1, 300), block, spread(1, std::min(nb, 2048)));
    }
}

void fits(const char* name, relaxkv_status st, size_t at_least) {
    char what[200];
    snprintf(what, sizeof what, "%s: status %d, %zu launches", name, st, launches.size());
    expect(st == RELAXKV_OK && launches.size() >= at_least, what);
    for (const Launch& l : launches) {
        const uint64_t x = (uint64_t)l.grid.x * l.block.x;
        snprintf(what, sizeof what, "%s: grid %u x %u x %u of %u threads", name, l.grid.x, l.grid.y, l.grid.z,
                 l.block.x);
        expect(x > 0 && x < 1ull << 32 && l.grid.y <= 65535 && l.grid.z <= 65535 && l.block.x <= 1024, what);
    }
    launches.clear();
}

void fresh() {
    char name[200];
    for (int dtype = 0; dtype < 2; ++dtype)
        for (int d = 64; d <= 128; d += 64)
            for (int H : {1, 16, 31, 32, 48, 64, 1024})
                for (int n : {1, 1024, 1025, (1 << 23), (1 << 24) - 1, 1 << 24, (1 << 24) + 1, (1 << 25) - 1,
                              RELAXKV_MAX_FRESH_ROWS}) {
                    const relaxkv_problem p = make(64, H, dtype && H == 1024 ? 64 : H, d, dtype);
                    const relaxkv_rope r = {(const float*)at(0x100), nullptr, nullptr, 0.f, 16, 0};
                    const relaxkv_rows in = {at(0x1000), nullptr, nullptr, 0, 0, 0, n};
                    snprintf(name, sizeof name, "fresh_rows of %d rows, %d heads, d %d", n, H, d);
                    fits(name, relaxkv_fresh_rows(&p, &r, &in, (const int32_t*)at(0x100), at(0x1000), nullptr,
                                                  nullptr, nullptr), 1);
                }
}

void batch() {
    char name[200];
    for (int dtype = 0; dtype < 2; ++dtype)
        for (int d = 64; d <= 128; d += 64)
            for (int H : {1, 64, 128, 1024})
                for (int Hkv : {1, H})
                    for (int T : {1, 64, 8192, 2048 * 16 + 1, 4096 * 16, 4096 * 16 + 1}) {
                        if (dtype && (H / Hkv > 256 || (int64_t)T * Hkv * d >= RELAXKV_MAX_BF16_LAYER_ELEMS)) continue;
                        const relaxkv_problem p = make(T, H, Hkv, d, dtype);
                        const int rows = std::min(RELAXKV_MAX_BATCH_ROWS, RELAXKV_MAX_BATCH_ROW_HEADS / H);
                        const int nb = (T + 15) / 16;
                        const relaxkv_batch b = bind(p, RELAXKV_MAX_SEQS, rows, 1000);
                        auto run = [&](const char* call, relaxkv_status st, size_t k) {
                            snprintf(name, sizeof name, "%s of %d rows, %d / %d heads, T %d, d %d, dtype %d", call,
                                     rows, H, Hkv, T, d, dtype);
                            fits(name, st, k);
                        };
                        const relaxkv_rope r = {(const float*)at(0x100), nullptr, nullptr, 0.f, 16, 0};
                        const relaxkv_rows in = {at(0x1000), at(0x2000), at(0x3000), 0, 0, 0, rows};
                        run("batch_plan", relaxkv_batch_plan(&p, &b, (int32_t*)at(0x100), (int32_t*)at(0x100), nullptr), 1);
                        run("batch_rows", relaxkv_batch_rows(&p, &r, &b, &in, at(0x1000), &kSuffix, nullptr), 1);
                        run("shared_attn", relaxkv_shared_attn(&p, &b, 0, at(0x2000), at(0x3000), at(0x4000), &kSuffix,
                                                               at(0x8000), nullptr, at(1 << 20), kAll, nullptr), 2);
                        run("block_means", relaxkv_block_means(&p, -1, at(0x2000), 16, at(0x8000), nullptr), 1);
                        for (int n_sel : {1, std::min(nb, RELAXKV_MAX_SELECTED_BLOCKS)}) {
                            run("block_select", relaxkv_block_select(&p, &b, 16, at(0x8000), at(0x4000), n_sel,
                                                                     (int32_t*)at(0x9000), at(1 << 20), kAll, nullptr), 1);
                            run("block_attn", relaxkv_block_attn(&p, &b, 0, at(0x2000), at(0x3000), 16,
                                                                 (int32_t*)at(0x9000), n_sel, at(0x4000), &kSuffix,
                                                                 at(0x8000), nullptr, at(1 << 20), kAll, nullptr), 2);
                        }
                    }
}

// block_select of `rows` rows and 8 KV heads over nb blocks takes n launches.
void select_launches(int d, int dtype, int nb, int rows, size_t n) {
    char what[200];
    const relaxkv_problem p = make(nb * 16, 8, 8, d, dtype);
    const relaxkv_batch b = bind(p, rows, rows, 8);
    launches.clear();
    expect(relaxkv_block_select(&p, &b, 16, at(0x8000), at(0x4000), 1, (int32_t*)at(0x9000), at(1 << 20), kAll,
                                nullptr) == RELAXKV_OK, "status");
    snprintf(what, sizeof what, "block_select: d %d, dtype %d, %d blocks, %d rows: %zu launches instead of %zu", d,
             dtype, nb, rows, launches.size(), n);
    expect(launches.size() == n, what);
}

void select() {
    for (int rows : {1, 32, 33})
        for (int nb : {1, 60, 256, 257, 500, 512, 1024, 1025}) {
            select_launches(64, 0, nb, rows, rows <= 32 && nb <= 1024 ? 1 : 2);
            select_launches(64, 1, nb, rows, rows <= 32 && nb <= 1024 ? 1 : 2);
            select_launches(128, 0, nb, rows, rows <= 32 && nb <= 256 ? 1 : 2);
            select_launches(128, 1, nb, rows, rows <= 32 && nb <= 256 ? 1 : 2);
        }
}

}  // namespace

// The runtime's launch of `kernel<<<grid, block>>>` in three calls.
#define TAKE extern "C" __attribute__((visibility("default")))
TAKE hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
    launches.push_back({grid, block});
    return hipSuccess;
}
TAKE hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* st) {
    *grid = launches.back().grid;
    *block = launches.back().block;
    *lds = 0;
    *st = nullptr;
    return hipSuccess;
}
TAKE hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) { return hipSuccess; }
TAKE hipError_t hipGetLastError() { return hipSuccess; }

int main(int argc, char** argv) {
    if (argc == 3 && !strcmp(argv[1], "steps")) steps(atol(argv[2]));
    else if (argc == 2 && !strcmp(argv[1], "fresh")) fresh();
    else if (argc == 2 && !strcmp(argv[1], "batch")) batch();
    else if (argc == 2 && !strcmp(argv[1], "select")) select();
    else return 2;
    if (n_bad) {
        fprintf(stderr, "%ld of %ld checks failed\n", n_bad, n_checks);
        return 1;
    }
    printf("ok %ld\n", n_checks);
    return 0;
}
