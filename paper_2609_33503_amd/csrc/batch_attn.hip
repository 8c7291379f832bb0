// Attention of a batch's rows over one shared context cache and, causally, each row's own
// request's suffix; and the same over listed context blocks instead of the whole context.
//
//   O_t = sum_j softmax_j(sigma <q_t, K_j>) V_j,   j over the context keys (all, or those of
//   the row's listed blocks) and then the suffix tokens of the row's request up to its own.
//
// bf16: one launch of independent work items, then a merge.
// - Context items.  Shared: the (token, head) rows of ALL requests of a KV head in chunks of
//   128, over key tiles, so K and V are read once for the batch and not once per request.
//   Listed: one token's group of heads, times one split of its listed keys; the list is
//   first compacted into LDS (full blocks, then copies of a partial last block), so that
//   every key below the count is one the row sees.
// - Suffix items: 128 rows of one request, times one split of its keys, causal.
// - How the items are split over workgroups (BatchSplit) follows from the step itself and
//   comes with its plan, so that the room of a batch does not change how a step is computed.  The
//   grids do follow the room, and a workgroup without an item takes its start and end: 64 decoding
//   rows of 40/8 heads over 32K in a batch of 64 rows, 512, 4096, 16384: 72, 69, 82, 132 us; over
//   2K listed keys 66, 68, 116, 297.
// - Each item streams 32-key K and V tiles through three swizzled LDS buffers by direct
//   loads; 48 KB of LDS and 167 registers let three workgroups share a CU, whose softmax,
//   matrix products and waits overlap.  A wave owns 32 rows (16 where that covers the item;
//   one row per lane): S^T = K Q^T, online softmax in the exp2 domain with a lazily raised
//   maximum, O^T += V^T P^T.
// - Probabilities are rounded to bf16 for the second product (2^-8 of each, independent over
//   keys: about as much as rounding O once; float32 products would take eight times the matrix
//   time).  The output is divided by the sum of the rounded ones, which keeps a row that
//   sees one key exact, the log-sum-exp uses the sum of the exact ones.
// - Every item writes its unnormalised output and (max, sums, scale); batch_merge adds them
//   with weights exp2(max_s - max) in a fixed order.  The outputs are written in 16 bits, half the
//   traffic of float32: as fp16 times a power of two that takes the row's largest element into
//   [2^14, 2^15) (an element is off by at most 2^-11 of itself, an eighth of what rounding O to
//   bf16 costs, down to 2^-28 of the largest, and by at most 2^-8 below, down to 2^-17 as scaled); a
//   row with a smaller element that is not 0, as bf16 (2^-8 of each, whatever their range).
// 64 decoding requests of 40/8 heads over 32K keys, d 128: 63 us and 7.0 of merge (its K and V once and
// the suffixes: 37 us at 6.07 TB/s); 20 questions of 761 tokens in all, 32/8 heads, over 8K: 115-120
// and 12 (85 at 1188 TFLOP/s).  While it runs MFMA and vector unit are busy 30-42% and 39-48%, rarely
// together, LDS 23%.  384 rows per KV head take 49-53 us more for 32K more keys, and as much without
// the fills, which alone take 33: the arithmetic at the clock that the power limit leaves.
// A row that sees no key gets O = 0 and lse = -inf.
// Loads never leave a run's keys (past its end they repeat its last key, masked), so cache
// rows past the context and suffix tokens past a request's length are never read.
//
// float32: the MFMA core of attn_f32.h over the same two kinds of items, 16 rows each: rows of all
// requests over a split of the context, rows of one request over a split of its suffix.  Each
// writes normalised outputs and log-sum-exps, which batch_merge_f32 adds in split order.
// Listed: a token's group of heads over its listed and suffix keys, which needs no merge
// where it is one split.

#include <math.h>

#include <algorithm>

#include "attn_f32.h"
#include "batch.h"
#include "dev_common.h"

namespace relaxkv {
namespace {

constexpr int kBaStages = 3;           // LDS ring depth
constexpr int kBaWaves = kBatchRowsBf16 / 32;
constexpr int kBaRing = 4;             // K fragments read ahead of their MFMA
constexpr int kBaRingV = 4;            // and V fragments
constexpr float kBaSlack = 8.0f;       // log2 units the running max may lag the true max
constexpr float kBaHuge = 1 << 20;     // log2 units from which half an ulp is near 2^-4

template <int N> struct Int { static constexpr int value = N; };

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

struct BaArgs {
    const uint16_t* q;       // [n_rows][H][D]
    const uint16_t *kc, *vc; // this layer's cache: key i of KV head g at g * c_sh + i * c_st
    const uint16_t *ks, *vs; // suffixes: key i of request b at b * s_ss + g * s_sh + i * s_st
    int64_t c_sh, c_st, s_ss, s_sh, s_st;
    const int32_t* counts;
    const int32_t* row_pos;
    const BatchTile* tiles;
    const int32_t* lists;    // [n_rows][Hkv][n_sel]
    // Partial rows: context ones first (shared: kBaRows per segment; listed: [split][Hkv][rows of
    // the step]), suffix ones ([split][Hkv][rows of the step]) from suf_part.
    _Float16* part_o;
    float4* part_s;          // (max, sum of rounded, sum of exact probabilities, scale; -1: a row of bf16)
    size_t suf_part;
    int T, H, Hkv, G, n_sel, bshift, nb, tail;
    int ctx_wgs, suf_wgs;    // workgroups of the launch for context and suffix items
    int list_tiles, list_items;   // listed: key tiles of a row at most, items of a token
    float sl2;               // softmax scale * log2(e)
};

// The step's split, through the scalar cache (it was written by an earlier kernel).  A step without
// rows may have no split at all (a zeroed buffer before its first plan): nothing is divided by it.
__device__ __forceinline__ BatchSplit load_split(const int32_t* counts) {
    typedef const __attribute__((address_space(4))) int32_t const_word;
    struct Words { int32_t w[sizeof(BatchSplit) / 4]; } words;
    const_word* p = (const_word*)(uintptr_t)(counts + kBatchSplitAt);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(BatchSplit) / 4); ++i) words.w[i] = p[i];
    return __builtin_bit_cast(BatchSplit, words);
}

// Listed keys of a row: splits, keys of each.
__device__ __forceinline__ void list_split(const BaArgs& a, int rows, int& n, int& kps) {
    const int tiles = a.list_tiles;
    batch_split_keys(tiles, rows * a.list_items, kBaWgs, kBaMinTiles, n, kps);
    kps *= kBaKeys;
}

// MFMA blocks of NR (token, head) rows: the lane's row is lane % NR, its group lane / NR.
// Value v of a 32-key tile's logits is key key0(v) + 4 kg, value v of an output block is element
// key0(v) + 4 group of the block's NR ones (key0: 8 (v/4) + v%4 for 32 rows, 16 (v/4) + v%4 for 16).
// kg is the group; for 16 rows the middle two of the four change places (the K rows that are fed
// to the product do), so that the V rows that 32 lanes read, 0 - 3 and 8 - 11, lie in different
// banks under the tiles' swizzle.
template <int NR> struct RowBlock;
template <> struct RowBlock<32> {
    typedef f32x16 Acc;
    static constexpr int key_sub = 1, kdim = 16;       // 32-key tile: one block of logits
    static __device__ __forceinline__ Acc mac(bf16x8 a, bf16x8 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    template <typename F> static __device__ __forceinline__ float groups(float x, F f) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
};
template <> struct RowBlock<16> {
    typedef f32x4 Acc;
    static constexpr int key_sub = 2, kdim = 32;       // two blocks of 16 keys
    static __device__ __forceinline__ Acc mac(bf16x8 a, bf16x8 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    template <typename F> static __device__ __forceinline__ float groups(float x, F f) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return RowBlock<32>::groups(f(__uint_as_float(r[0]), __uint_as_float(r[1])), f);
    }
};
template <int NR> __device__ __forceinline__ float ba_group_max(float x) {
    return RowBlock<NR>::groups(x, [](float a, float b) { return fmaxf(a, b); });
}
template <int NR> __device__ __forceinline__ float ba_group_sum(float x) {
    return RowBlock<NR>::groups(x, [](float a, float b) { return a + b; });
}

// Whether x is NaN, by its bits (this file is compiled for maxima and compares without NaN).
__device__ __forceinline__ bool is_nan(float x) {
    uint32_t u = __float_as_uint(x);
    asm volatile("" : "+v"(u));
    return (u & 0x7fffffffu) > 0x7f800000u;
}

// fill_lds16 with a wave-uniform base and a 32-bit byte offset per lane.
__device__ __forceinline__ void fill_lds16_u(const void* base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0"
                 :: "s"(base), "v"(off), "s"(lds) : "memory", "m0");
}

// Wave 0 compacts a block list into lst: entries in [0, nb) that are full blocks in list
// order; cnt[0] of them, cnt[1] copies of the partial last block.  Other entries are dropped.
__device__ __forceinline__ void compact_list(const int32_t* list, int n, int nb, int tail, int* lst,
                                             int* cnt) {
    const int lane = threadIdx.x & 63;
    if (threadIdx.x < 64) {
        int nf = 0, nt = 0;
        for (int i0 = 0; i0 < n; i0 += 64) {
            const int b = i0 + lane < n ? list[i0 + lane] : -1;
            const bool part = tail > 0 && b == nb - 1;
            const bool full = b >= 0 && b < nb && !part;
            const uint64_t m = __ballot(full);
            if (full) lst[nf + lanes_below(m)] = b;
            nf += __popcll(m);
            nt += __popcll(__ballot(part));
        }
        if (lane == 0) {
            cnt[0] = nf;
            cnt[1] = nt;
        }
    }
    __syncthreads();
}

// Position of key c of a compacted list.
__device__ __forceinline__ int list_key(int c, const int* lst, int nf, int bshift, int nb, int tail) {
    const int cf = nf << bshift;
    if (c < cf) return (lst[c >> bshift] << bshift) + (c & ((1 << bshift) - 1));
    return ((nb - 1) << bshift) + (c - cf) % tail;
}

template <int D, bool LIST>
__global__ __launch_bounds__(kBaWaves * 64, 3) void battn_bf16(BaArgs a) {
    constexpr int TK = kBaKeys, ST = kBaStages, NW = kBaWaves;
    constexpr int ROWB = 2 * D;            // tile row bytes
    constexpr int CH = D / 8;              // 16-byte chunks per row
    constexpr int RPI = 64 / CH;           // rows per wave-wide load
    constexpr int NL = TK / RPI;           // wave-wide loads per tile and tensor
    constexpr int NI = NL / NW;            // of them per wave
    constexpr int LPW = 2 * NI;            // K and V
    static_assert(NL % NW == 0 && TK == 32 && ST == 3, "tile shape");
    __shared__ __attribute__((aligned(1024))) uint16_t tiles[2 * ST * TK * D];   // K, then V
    extern __shared__ int lst[];                         // listed: n_sel blocks
    __shared__ int cnt[2];

    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const BatchSplit sp = load_split(a.counts);
    const int ctx0 = sp.suffix_first ? a.suf_wgs : 0, suf0 = sp.suffix_first ? 0 : a.ctx_wgs;
    const bool ctx = sp.suffix_first ? (int)blockIdx.x >= a.suf_wgs : (int)blockIdx.x < a.ctx_wgs;
    const int wg = (int)blockIdx.x - (ctx ? ctx0 : suf0);
    const size_t R = (size_t)sp.rows * a.G;              // rows of the step per KV head

    // Shared context: the worker's tiles x .. x_end - 1.
    int worker = 0;
    int64_t x = 0, x_end = 0;
    if (sp.rows == 0) return;
    if (ctx && !LIST) {
        const int j = wg / kBaXcds, xcd = wg % kBaXcds;   // (both counts are multiples of the XCDs)
        if (sp.per_item) {
            // (the chunks of one key range are consecutive workgroups of one XCD)
            const int pair = j / sp.chunks * kBaXcds + xcd;
            if (pair >= sp.per_item * a.Hkv) return;
            worker = (pair % a.Hkv * sp.chunks + j % sp.chunks) * sp.per_item + pair / a.Hkv;
        } else {
            worker = xcd * (kBaWgs / kBaXcds) + j;       // (neighbours share an XCD)
        }
        if (worker >= sp.workers) return;
        x = (int64_t)worker * sp.quota;
        x_end = min(x + sp.quota, (int64_t)sp.items * sp.len);
    }

  for (;;) {
    // Made opaque per item, so that what is derived from it is not kept live across the loop.
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    // The item: KV head g, the wave's first partial row and number of rows (consecutive ones),
    // the lane's row (token t, head hh of the group, last visible key lim), and the keys key0 ..
    // key0 + nk - 1 of a run (base pointers, stride); the first `open` of them every row sees.
    // An item of at most 64 rows gives each wave 16 of them instead of 32: half the products and
    // softmax of a wave, and a decoding request's few heads do not wait for 32 rows' (16 rows
    // over 4096 listed keys each: 11.6 us, 14.1 with 32; 64 requests of 5 rows over suffixes of
    // 300: 73.2, 76.6).
    int g, t, hh, lim, key0, nk, open, n_val;
    bool small;
    const uint16_t *kb, *vb;
    int64_t st;
    size_t part;
    bool listed = false;
    if (ctx) {
        if constexpr (LIST) {
            int y = wg, list_n, list_kps;
            list_split(a, sp.rows, list_n, list_kps);
            const int split = y % list_n;
            y /= list_n;
            int chunk = 0;
            if (a.G > kBaRows) {
                const int chunks = (a.G + kBaRows - 1) / kBaRows;
                chunk = y % chunks;
                y /= chunks;
            }
            g = y % a.Hkv;
            t = y / a.Hkv;
            if (t >= sp.rows) return;
            compact_list(a.lists + ((size_t)t * a.Hkv + g) * a.n_sel, a.n_sel, a.nb, a.tail, lst, cnt);
            small = a.G - chunk * kBaRows <= 64;
            const int rw = small ? 16 : 32, r = lane & (rw - 1);
            const int h0 = chunk * kBaRows + w * rw;
            n_val = min(a.G - h0, rw);
            hh = r < n_val ? h0 + r : 0;
            part = ((size_t)split * a.Hkv + g) * R + (size_t)t * a.G + h0;
            key0 = split * list_kps;
            const int n = __builtin_amdgcn_readfirstlane((cnt[0] << a.bshift) + cnt[1] * a.tail);
            nk = min(list_kps, n - key0);
            if (nk <= 0) {                               // nothing in this split
                if (lane < n_val) a.part_s[part + lane] = float4{-INFINITY, 0.f, 0.f, 0.f};
                return;
            }
            listed = true;
        } else {
            const int item = (int)(x / sp.len), t0 = (int)(x - (int64_t)item * sp.len);
            const int left = (int)(x_end - x), nt = min(left, sp.tiles - t0);
            x += min(left, sp.len - t0);                 // (the next item's first tile)
            if (nt <= 0) return;                         // (padding, which ends a range)
            g = item / sp.chunks;
            const int row0 = (item - g * sp.chunks) * kBaRows;
            small = sp.rows * a.G - row0 <= 64;
            const int rw = small ? 16 : 32, r = lane & (rw - 1);
            const int rho0 = row0 + w * rw;
            n_val = min(sp.rows * a.G - rho0, rw);
            const int rho = r < n_val ? rho0 + r : 0;
            t = rho / a.G;
            hh = rho - t * a.G;
            part = (size_t)(worker + item) * kBaRows + w * rw;
            key0 = t0 * TK;
            nk = min(nt * TK, a.T - key0);
        }
        lim = nk - 1;
        open = nk;
        kb = a.kc + g * a.c_sh;
        vb = a.vc + g * a.c_sh;
        st = a.c_st;
    } else {
        int y = wg;
        const int split = y % sp.suf_n;
        y /= sp.suf_n;
        g = y % a.Hkv;
        y /= a.Hkv;
        if (y >= sp.row_tiles) return;
        BatchTile tl = a.tiles[y];
        tl.seq = __builtin_amdgcn_readfirstlane(tl.seq);
        tl.row_begin = __builtin_amdgcn_readfirstlane(tl.row_begin);
        tl.n_new = __builtin_amdgcn_readfirstlane(tl.n_new);
        tl.past = __builtin_amdgcn_readfirstlane(tl.past);
        tl.row0 = __builtin_amdgcn_readfirstlane(tl.row0);
        key0 = split * sp.suf_kps;
        const int n_th = tl.n_new * a.G;                 // (token, head) rows of the request
        const int last = (min(tl.row0 + kBaRows, n_th) - 1) / a.G;
        nk = min(sp.suf_kps, tl.past + last + 1 - key0);
        if (nk <= 0) return;
        small = n_th - tl.row0 <= 64;
        const int rw = small ? 16 : 32, r = lane & (rw - 1);
        const int rq0 = tl.row0 + w * rw;
        n_val = min(n_th - rq0, rw);
        const int rq = r < n_val ? rq0 + r : 0;
        const int tr = rq / a.G;
        hh = rq - tr * a.G;
        t = tl.row_begin + tr;
        part = a.suf_part + ((size_t)split * a.Hkv + g) * R + (size_t)tl.row_begin * a.G + rq0;
        lim = tl.past + tr - key0;                       // (below 0: the merge skips the split)
        open = min(nk, tl.past + tl.row0 / a.G + 1 - key0);
        kb = a.ks + tl.seq * a.s_ss + g * a.s_sh;
        vb = a.vs + tl.seq * a.s_ss + g * a.s_sh;
        st = a.s_st;
    }
    const bool live = n_val > 0;
    const int ntile = (nk + TK - 1) / TK;

    // Loader: load jj = w + NW i fills tile rows jj RPI ..; lane l writes (row l / CH, chunk
    // l % CH) and fetches the chunk that belongs there.  The swizzle of a lane's rows is the
    // same for every i (NW RPI is a multiple of its period), so in full tiles of a run a
    // lane's byte offset is constant and the base is wave-uniform.
    const int lrow = lane / CH, pchunk = lane % CH;
    static_assert((NW * RPI) % 16 == 0, "the swizzle repeats every 16 rows");
    const int ch8 = (pchunk ^ tile_swz<D>(w * RPI + lrow)) << 3;
    const uint32_t lane_off = (uint32_t)(lrow * (int)st + ch8) * 2u;
    const uint32_t kt0 = lds_addr(tiles) + w * RPI * ROWB, vt0 = kt0 + ST * TK * ROWB;
    auto issue = [&](int tt) {
        const uint32_t so = (uint32_t)(tt % ST) * (TK * ROWB);
        if (!listed && (tt + 1) * TK <= nk) {
            const int64_t e0 = (int64_t)(key0 + tt * TK + w * RPI) * st;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int64_t e = e0 + (int64_t)(NW * RPI * i) * st;
                fill_lds16_u(kb + e, lane_off, kt0 + so + i * (NW * RPI * ROWB));
                fill_lds16_u(vb + e, lane_off, vt0 + so + i * (NW * RPI * ROWB));
            }
        } else {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                int c = key0 + min(tt * TK + (w + NW * i) * RPI + lrow, nk - 1);
                if constexpr (LIST)
                    if (listed) c = list_key(c, lst, cnt[0], a.bshift, a.nb, a.tail);
                const int64_t e = c * st + ch8;
                fill_lds16(kb + e, kt0 + so + i * (NW * RPI * ROWB));
                fill_lds16(vb + e, vt0 + so + i * (NW * RPI * ROWB));
            }
        }
    };

    auto run = [&](auto nr_t) {
        constexpr int NR = decltype(nr_t)::value;
        typedef RowBlock<NR> RB;
        typedef typename RB::Acc Acc;
        constexpr int NV = sizeof(Acc) / 4, KB = RB::key_sub, NS = KB * NV;   // logits of a lane
        constexpr int KS = D / RB::kdim;               // k-steps of QK^T
        constexpr int DB = D / NR, PK = 32 / RB::kdim; // d blocks of O^T, products of each per tile
        constexpr int VSTEP = NR == 32 ? 8 : 16;       // keys between a lane's runs of four
        const int row = lane & (NR - 1), grp = lane / NR;
        const int kg = NR == 16 ? grp >> 1 | (grp & 1) << 1 : grp;
        const int krow = NR == 16 ? (row & 3) | (row & 4) << 1 | (row & 8) >> 1 : row;
        const int lim4 = lim - 4 * kg;
        bf16x8 qf[KS];
        {
            const uint16_t* qrow = a.q + ((size_t)t * a.H + g * a.G + hh) * D;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const bf16x8*)(qrow + ks * RB::kdim + grp * 8);
            // Consumed here, so the compiler's waits for these loads stay before the loop.
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
        }
        Acc o[DB];
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = Acc{};
        // The row's reference maximum, what the logits are compared with, and subtracted from them.
        float m_run = -INFINITY, thr = -INFINITY, m_ref = 0.f;
        float l0 = 0.f, l1 = 0.f, e0 = 0.f, e1 = 0.f;  // sums of rounded and exact probabilities
        const float inv_sl2 = 1.0f / a.sl2;

        // Fragment byte offsets: K rows `krow` (+ 16), chunk grp (+ the k-step's); V by transposing
        // reads, 16 lanes taking 4 keys x 16 elements.
        const int k_base = krow * ROWB | ((grp ^ tile_swz<D>(krow)) << 4);
        const int rl = 4 * kg + ((lane & 15) >> 2);
        const int cl = (NR == 32 ? ((lane >> 4) & 1) * 2 : 0) + ((lane & 3) >> 1);
        const int v_base0 = rl * ROWB | ((cl ^ tile_swz<D>(rl)) << 4) | ((lane & 1) << 3);
        const int v_base1 = (rl + VSTEP) * ROWB | ((cl ^ tile_swz<D>(rl + VSTEP)) << 4) | ((lane & 1) << 3);
        const char* kst = (const char*)tiles;
        const uint32_t vlds = lds_addr(tiles) + ST * TK * ROWB;

        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        auto step = [&](uint32_t stage, int c0) {
            int kbo = k_base + (int)stage;
            uint32_t vb0 = v_base0 + vlds + stage, vb1 = v_base1 + vlds + stage;
            asm volatile("" : "+v"(kbo), "+v"(vb0), "+v"(vb1));
            // S^T = K Q^T
            Acc sa[KB];
            constexpr int NX = KS * KB;                // fragment x: k-step x / KB, keys x % KB
            auto frag = [&](int x) {
                return *(const bf16x8*)(kst + (x % KB) * 16 * ROWB + (kbo ^ ((x / KB) * (2 * RB::kdim))));
            };
            bf16x8 kf[kBaRing];
#pragma unroll
            for (int i = 0; i < kBaRing; ++i) kf[i] = frag(i);
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                const bf16x8 cur = kf[x % kBaRing];
                if (x + kBaRing < NX) kf[x % kBaRing] = frag(x + kBaRing);
                sa[x % KB] = RB::mac(cur, qf[x / KB], x < KB ? Acc{} : sa[x % KB]);
            }
            // V fragments, the first ones read ahead of the softmax: y = PK db + k2
            constexpr int NY = DB * PK;
            auto vfrag = [&](int y) {
                const uint32_t rowo = (y % PK) * 16 * ROWB;
                const v4i16 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_v4i16*)(uintptr_t)((vb0 ^ (y / PK * (2 * NR))) + rowo));
                const v4i16 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_v4i16*)(uintptr_t)((vb1 ^ (y / PK * (2 * NR))) + rowo));
                return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
            };
            bf16x8 vf[kBaRingV];
#pragma unroll
            for (int i = 0; i < kBaRingV; ++i) vf[i] = vfrag(i);
            __builtin_amdgcn_sched_group_barrier(0x100, kBaRing, 0);
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (x + kBaRing < NX) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                else __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            // The softmax before other waves' matrix products: the vector unit is the busier one (the
            // reverse order, or none, takes 3-4% longer).
            __builtin_amdgcn_s_setprio(1);
            float s[NS];
#pragma unroll
            for (int v = 0; v < NS; ++v) s[v] = sa[v / NV][v % NV];
            if (c0 + TK > open) {                      // the run's tail, or the causal future
                const int e = lim4 - c0;
#pragma unroll
                for (int v = 0; v < NS; ++v)
                    if (VSTEP * (v >> 2) + (v & 3) > e) s[v] = -INFINITY;
            }
            float mk = fmaxf(s[0], s[1]), mk2 = fmaxf(s[2], s[3]);
#pragma unroll
            for (int v = 4; v < NS; v += 4) {
                mk = fmaxf(fmaxf(mk, s[v]), s[v + 1]);
                mk2 = fmaxf(fmaxf(mk2, s[v + 2]), s[v + 3]);
            }
            const float top = ba_group_max<NR>(fmaxf(mk, mk2));
            if (__any(top > thr)) {
                const float mx = top * a.sl2;
                const float m_new = mx > m_run + kBaSlack ? mx : m_run;
                const float alpha = m_new == m_run ? 1.f : fast_exp2(m_run - m_new);
                l0 *= alpha;
                l1 *= alpha;
                e0 *= alpha;
                e1 *= alpha;
#pragma unroll
                for (int db = 0; db < DB; ++db) o[db] *= alpha;
                m_run = m_new;
                // The maximum is rounded, the product in the multiply-add below is not: where
                // logits are huge (a split of keys at the type's lowest value), what the rounding
                // cut off would be an exponent of its own.  Such a row enters here for every tile,
                // has the product rounded too and its logits moved to a maximum of 0.
                const bool none = m_run == -INFINITY, huge = !none && fabsf(m_run) > kBaHuge;
                m_ref = none || huge ? 0.f : m_run;    // (no visible key so far: exact zeros)
                thr = huge ? -INFINITY : (m_run + kBaSlack) * inv_sl2;
                if (__any(huge)) {
#pragma unroll
                    for (int v = 0; v < NS; ++v) {
                        float x = s[v] * a.sl2;
                        asm volatile("" : "+v"(x));    // (not a multiply-add)
                        s[v] = huge ? (x - m_run) * inv_sl2 : s[v];
                    }
                }
            }
            bf16x8 pb[PK];
#pragma unroll
            for (int v = 0; v < NS; ++v) {
                const float p = fast_exp2(fmaf(s[v], a.sl2, -m_ref));
                (v & 1 ? e1 : e0) += p;
                pb[v >> 3][v & 7] = (__bf16)p;
            }
            const bf16x2 one2 = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
            for (int k2 = 0; k2 < PK; ++k2) {
                const bf16x8 q8 = pb[k2];
                l0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(q8, q8, 0, 1), one2, l0, false);
                l1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(q8, q8, 2, 3), one2, l1, false);
                l0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(q8, q8, 4, 5), one2, l0, false);
                l1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(q8, q8, 6, 7), one2, l1, false);
            }
            __builtin_amdgcn_s_setprio(0);
            // O^T += V^T P^T
#pragma unroll
            for (int y = 0; y < NY; ++y) {
                const bf16x8 cur = vf[y % kBaRingV];
                if (y + kBaRingV < NY) vf[y % kBaRingV] = vfrag(y + kBaRingV);
                o[y / PK] = RB::mac(cur, pb[y % PK], o[y / PK]);
            }
        };

#pragma unroll
        for (int tt = 0; tt < ST - 1; ++tt)
            if (tt < ntile) issue(tt);
        for (int tt = 0; tt < ntile; ++tt) {
            // Tile tt has landed (the later one of the ring may be in flight), and every wave is
            // done with the buffer that is filled next.
            if (tt + 1 < ntile) wait_loads_barrier<LPW>();
            else wait_loads_barrier<0>();
            if (tt + ST - 1 < ntile) issue(tt + ST - 1);
            if (live) step((uint32_t)(tt % ST) * (TK * ROWB), tt * TK);
        }

        // The partial rows: in 16 bits, transposed through LDS (the tiles are done with) and
        // written as whole rows.
        const float l_tot = ba_group_sum<NR>(l0 + l1), l_ex = ba_group_sum<NR>(e0 + e1);
        asm volatile("" : "+v"(lane));
        __syncthreads();
        constexpr int OROW = 2 * D + 16;               // bytes of a row in LDS
        static_assert(kBaRows * OROW <= (int)sizeof(tiles), "the rows fit the tiles");
        char* orow = (char*)tiles + (w * NR) * OROW;
        if (live) {
            // The largest finite element, and the smallest that is not 0 (its bits without the sign,
            // less one: 0 is then above every number).
            float top = 0.f;
            uint32_t low = ~0u;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const float x = fabsf(o[db][v]);
                    top = x <= 3.4028235e38f ? fmaxf(top, x) : top;
                    low = min(low, (__float_as_uint(o[db][v]) << 1) - 1u);
                }
            top = ba_group_max<NR>(top);
            // Exponent of the largest (of 2^-112 at least, so that scale and inverse are normal
            // numbers; what fp16 then cuts off is below float32's smallest).
            const int ex = top > 0.f ? max((int)(__float_as_uint(top) >> 23), 15) : 141;
            const float inv = __uint_as_float((uint32_t)(268 - ex) << 23);
            const bool far = ba_group_max<NR>(ex > 31 && low < ((uint32_t)(ex - 31) << 24) - 1u ? 1.f : 0.f) > 0.f;
            const float scale = far ? -1.f : __uint_as_float((uint32_t)(ex - 14) << 23);
            typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
            auto half = [&](float x) { return __builtin_bit_cast(uint16_t, (_Float16)(x * inv)); };
            auto write = [&](auto bits) {
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int j = 0; j < NV / 4; ++j)
                        *(u16x4*)(orow + (lane & (NR - 1)) * OROW + 2 * (db * NR + 8 * j + 4 * (lane / NR))) =
                            u16x4{bits(o[db][4 * j]), bits(o[db][4 * j + 1]), bits(o[db][4 * j + 2]),
                                  bits(o[db][4 * j + 3])};
            };
            if (__any(far))
                write([&](float x) { return far ? __builtin_bit_cast(uint16_t, (__bf16)x) : half(x); });
            else
                write(half);
            // (a NaN sum under a maximum of -inf, where no logit is a number, must not pass for a
            // split without keys)
            if (lane < n_val) a.part_s[part + lane] = float4{is_nan(l_ex) ? 0.f : m_run, l_tot, l_ex, scale};
            __builtin_amdgcn_wave_barrier();
            _Float16* dst = a.part_o + part * D + lane * 8;
#pragma unroll
            for (int i = 0; i < NR / RPI; ++i) {
                const int r = i * RPI + lane / CH;
                const u32x4 v = *(const u32x4*)(orow + r * OROW + (lane % CH) * 16);
                if (r < n_val) *(u32x4*)(dst + i * 512) = v;
            }
        }
    };
    if (small) run(Int<16>{});
    else run(Int<32>{});
    if (!ctx || LIST || x >= x_end) return;
    __syncthreads();                                     // (the next item fills the tiles)
  }
}

// LN lanes per (token, head): its partials are the context's in order, then the suffix splits
// that hold one of the row's keys.  Lane i takes the statistics of partial i (then i + LN, ..);
// the outputs are loaded by groups of D/8 lanes, partial by partial in turn, four each at a
// time with the weights handed round, so a row waits for memory about twice.
template <int D, bool LIST, int LN>
__device__ __forceinline__ void merge_row(const BaArgs& a, const BatchSplit& sp, long th,
                                          uint16_t* __restrict__ out, float* __restrict__ lse) {
    constexpr int LPR = D / 8, NG = LN / LPR, U = 4;
    typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
    const int wl = threadIdx.x & 63, base = wl / LN * LN, lane = wl - base;
    const int grp = lane / LPR, col = lane % LPR;
    const int t0 = (int)(th / a.H);
    // (surplus lanes of a wave follow a real row, so that the exchanges below stay whole)
    const bool real = t0 < sp.rows;
    if (!__any(real)) return;
    const int t = real ? t0 : 0, h = real ? (int)(th - (long)t0 * a.H) : 0;
    const int g = h / a.G, rho = t * a.G + (h - g * a.G);
    const size_t R = (size_t)sp.rows * a.G;
    int n_ctx;
    size_t first, step;                                  // context partial s: first + s * step
    if constexpr (LIST) {
        int kps;
        list_split(a, sp.rows, n_ctx, kps);
        first = (size_t)g * R + rho;
        step = (size_t)a.Hkv * R;
    } else {
        const int chunk = rho / kBaRows, item = g * sp.chunks + chunk;
        const int64_t x0 = (int64_t)item * sp.len;
        const int w0 = (int)(x0 / sp.quota);
        n_ctx = (int)((x0 + sp.tiles - 1) / sp.quota) - w0 + 1;
        first = (size_t)(w0 + item) * kBaRows + (rho - chunk * kBaRows);
        step = kBaRows;
    }
    const size_t suf = a.suf_part + (size_t)g * R + rho, suf_step = (size_t)a.Hkv * R;
    const f32x4* part_s = (const f32x4*)a.part_s;
    auto at = [&](int s) { return s < n_ctx ? first + s * step : suf + (s - n_ctx) * suf_step; };
    // The first statistics and outputs are loaded beside the row's position, which says how many
    // suffix splits there are: up to all of them (what a split did not write gets weight 0).
    const int n_all = n_ctx + sp.suf_n;
    const f32x4 none = {-INFINITY, 0.f, 0.f, 0.f};
    f32x4 st0 = part_s[at(min(lane, n_all - 1))];
    f16x8 v0[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        v0[u] = *(const f16x8*)(a.part_o + at(min(u * NG + grp, n_all - 1)) * D + col * 8);
    const int n = n_ctx + (a.row_pos[t] - a.T) / sp.suf_kps + 1;
    st0 = lane < n ? st0 : none;
    float M = st0[0];
    for (int s = lane + LN; s < n; s += LN) M = fmaxf(M, part_s[at(s)][0]);
#pragma unroll
    for (int o = LN / 2; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
    float acc[8], z = 0.f, ze = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    for (int c0 = 0; __any(c0 < n); c0 += LN) {
        f32x4 st = st0;
        if (c0 > 0) st = c0 + lane < n ? part_s[at(c0 + lane)] : none;
        const float e = st[0] == -INFINITY ? 0.f : fast_exp2(st[0] - M);
        z = fmaf(e, st[1], z);
        ze = fmaf(e, st[2], ze);
        const float wt = e * st[3];                       // (0 past the last partial, below 0: bf16)
        if (__any(st[3] < 0.f)) {                         // (rare: one partial at a time)
            for (int j0 = 0; j0 < LN && __any(c0 + j0 < n); j0 += NG) {
                const int j = j0 + grp;
                const float wj = __shfl(wt, base + (j & (LN - 1)), 64);
                const f16x8 v = *(const f16x8*)(a.part_o + at(min(c0 + j, n - 1)) * D + col * 8);
                const bf16x8 b = __builtin_bit_cast(bf16x8, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {            // (weight 0: the output may not be written)
                    const float x = wj < 0.f ? (float)b[i] : (float)v[i];
                    acc[i] = wj != 0.f ? fmaf(fabsf(wj), x, acc[i]) : acc[i];
                }
            }
            continue;
        }
        for (int j0 = 0; j0 < LN && __any(c0 + j0 < n); j0 += NG * U) {
            f16x8 v[U];
            float wj[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u * NG + grp;
                wj[u] = __shfl(wt, base + (j & (LN - 1)), 64);
                v[u] = c0 + j0 == 0 ? v0[u]
                                    : *(const f16x8*)(a.part_o + at(min(c0 + j, n - 1)) * D + col * 8);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i)              // (weight 0: the output may not be written)
                    acc[i] = wj[u] != 0.f ? fmaf(wj[u], (float)v[u][i], acc[i]) : acc[i];
        }
    }
#pragma unroll
    for (int o = LN / 2; o > 0; o >>= 1) {
        z += __shfl_xor(z, o, 64);
        ze += __shfl_xor(ze, o, 64);
    }
#pragma unroll
    for (int o = LPR; o < LN; o <<= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += __shfl_xor(acc[i], o, 64);
    if (!real) return;
    const float inv = M == -INFINITY ? 0.f : 1.0f / z;
    if (grp == 0) {
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r[i] = (uint32_t)f32_to_bf16_bits(acc[2 * i] * inv) |
                   ((uint32_t)f32_to_bf16_bits(acc[2 * i + 1] * inv) << 16);
        *(u32x4*)(out + (size_t)th * D + col * 8) = r;
    }
    if (lse && lane == 0) lse[th] = M == -INFINITY ? -INFINITY : (M + __log2f(ze)) * kLn2;
}

// A row takes a wave where it has many partials, or several and few rows (33 partials of 2440
// rows: 9.0 us, 10.2 with D/8 lanes per row; 9 of 256: 4.4, 5.7); else D/8 lanes (5 partials of
// 24352 rows: 12.3 us, 20.7 with a wave; 4 of 2328: 4.1, 6.3).
constexpr int kBaManyPartials = 16, kBaSomePartials = 8, kBaFewRows = 4096;
template <int D, bool LIST>
__global__ __launch_bounds__(256) void batch_merge(BaArgs a, uint16_t* __restrict__ out,
                                                   float* __restrict__ lse) {
    constexpr int LPR = D / 8;
    const BatchSplit sp = load_split(a.counts);
    if (sp.rows == 0) return;
    int n_ctx, kps;
    if constexpr (LIST) list_split(a, sp.rows, n_ctx, kps);
    else n_ctx = sp.tiles / sp.quota + 1;
    const int n = n_ctx + sp.suf_n;
    if (n > kBaManyPartials || (n >= kBaSomePartials && sp.rows * a.H <= kBaFewRows))
        merge_row<D, LIST, 64>(a, sp, blockIdx.x * 4l + (threadIdx.x >> 6), out, lse);
    else
        merge_row<D, LIST, LPR>(a, sp, (long)blockIdx.x * (256 / LPR) + threadIdx.x / LPR, out, lse);
}

// float32, listed: key c is listed key c below their count, suffix token c - count from there.
struct BaF32Args {
    const float *q, *kc, *vc, *ks, *vs;
    int64_t c_sh, c_st, s_ss, s_sh, s_st;
    const int32_t *counts, *row_seq, *row_pos, *lists;
    const BatchTile* tiles;
    int T, H, Hkv, G, n_sel, bshift, nb, tail;
    int list_tiles, list_items;      // listed: kBaF32ListKeys of a row at most, items of a token
    float scale;
    float *out, *lse;
    float *part_o, *part_l;          // [split][rows of the step][H] (D)
};

// Listed: splits of an item's keys.
__device__ __forceinline__ void list_split_f32(const BaF32Args& a, int rows, int& n, int& kps) {
    batch_split_keys(a.list_tiles + (a.counts[2] + kBaF32ListKeys - 1) / kBaF32ListKeys,
                     rows * a.list_items, kBaF32ListWgs, 1, n, kps);
    kps *= kBaF32ListKeys;
}

template <bool LIST> constexpr int f32_waves() { return LIST ? kBaF32ListWaves : kBaF32Waves; }
template <int D, bool LIST>
__global__ __launch_bounds__(f32_waves<LIST>() * 64, 4) void battn_f32(BaF32Args a) {
    constexpr int R = kBatchRowsF32, NW = f32_waves<LIST>();
    extern __shared__ __attribute__((aligned(16))) char f32_lds[];
    typedef AttnF32Lds<D, R, NW> Lds;
    Lds& sm = *(Lds*)f32_lds;
    int* lst = (int*)(f32_lds + sizeof(Lds));
    const int rl = threadIdx.x % R;
    const BatchSplit sp = load_split(a.counts);
    if (sp.rows == 0) return;
    int x = (int)(blockIdx.y * gridDim.x + blockIdx.x);
    bool ctx = false;
    int n_split, kps;
    if constexpr (LIST) {
        list_split_f32(a, sp.rows, n_split, kps);
    } else {
        const int ctx_wgs = (sp.rows * a.G + R - 1) / R * a.Hkv * sp.f32_n;
        ctx = x < ctx_wgs;
        if (!ctx) x -= ctx_wgs;
        n_split = ctx ? sp.f32_n : sp.f32_sn;
        kps = ctx ? sp.f32_kps : sp.f32_skps;
    }
    const int split = x % n_split;
    x /= n_split;
    const int g = x % a.Hkv;
    x /= a.Hkv;
    // Keys 0 .. n_ctx - 1 are context keys (or listed ones), the others suffix tokens; the row sees
    // those up to n_ctx + own, a row of the item those up to n_ctx + last_own.
    int t, hh, seq, own, last_own, n_ctx = 0;
    bool valid;
    if constexpr (LIST) {
        const int chunks = (a.G + R - 1) / R;
        t = x / chunks;
        if (t >= sp.rows) return;
        hh = (x - t * chunks) * R + rl;
        valid = hh < a.G;
        if (!valid) hh = a.G - 1;
        compact_list(a.lists + ((size_t)t * a.Hkv + g) * a.n_sel, a.n_sel, a.nb, a.tail, lst + 2, lst);
        n_ctx = (lst[0] << a.bshift) + lst[1] * a.tail;
        seq = a.row_seq[t];
        own = last_own = a.row_pos[t] - a.T;
    } else if (ctx) {
        const int rho0 = x * R + rl, n_th = sp.rows * a.G;
        valid = rho0 < n_th;
        const int rho = valid ? rho0 : n_th - 1;
        t = rho / a.G;
        hh = rho - t * a.G;
        seq = 0;
        n_ctx = a.T;
        own = last_own = -1;
    } else {
        if (x >= sp.row_tiles) return;
        const BatchTile tl = a.tiles[x];
        const int n_th = tl.n_new * a.G, last = min(tl.row0 + R, n_th) - 1;
        const int rq0 = tl.row0 + rl;
        valid = rq0 < n_th;
        const int rq = valid ? rq0 : last;
        const int tr = rq / a.G;
        hh = rq - tr * a.G;
        t = tl.row_begin + tr;
        seq = tl.seq;
        own = tl.past + tr;
        last_own = tl.past + last / a.G;
    }
    const uint32_t orow = (uint32_t)t * a.H + g * a.G + hh;
    float *out = a.out, *lse = a.lse;
    if (!LIST || n_split > 1) {
        const size_t part = (size_t)(LIST || ctx ? split : sp.f32_n + split) * sp.rows * a.H;
        out = a.part_o + part * D;
        lse = a.part_l + part;
    }
    // (a row that sees no key of the split: output 0, log-sum-exp -inf)
    const int key0 = split * kps, n_keys = min(kps, n_ctx + last_own + 1 - key0);
    if (n_keys <= 0) {
        if (valid && threadIdx.x < R) lse[orow] = -INFINITY;
        return;
    }
    auto id_of = [&](int c0) {
        const int c = c0 + key0;
        if (c >= n_ctx) return c - n_ctx;
        if constexpr (LIST) return ~list_key(c, lst + 2, lst[0], a.bshift, a.nb, a.tail);
        else return ~c;
    };
    const int64_t sb = seq * a.s_ss + g * a.s_sh;
    attn_f32_rows<D, R, 4, NW>(sm, a.ks + sb, a.vs + sb, a.s_st, a.kc + g * a.c_sh, a.vc + g * a.c_sh,
                               a.c_st, id_of, n_keys, a.q + (size_t)orow * D,
                               max(-1, min(n_keys - 1, n_ctx + own - key0)), a.scale, valid, out, lse, orow);
}

// One wave per (token, head): lane s takes split s's log-sum-exp, D/4 lanes (twice at d 64) then
// add the splits' outputs.
template <int D, bool LIST>
__global__ __launch_bounds__(256) void batch_merge_f32(BaF32Args a) {
    constexpr int LPR = D / 4, NG = 64 / LPR;
    const int lane = threadIdx.x & 63, grp = lane / LPR, col = lane % LPR;
    const long th = blockIdx.x * 4l + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const BatchSplit sp = load_split(a.counts);
    if (sp.rows == 0) return;
    int n = sp.f32_n + sp.f32_sn, kps;
    if constexpr (LIST) list_split_f32(a, sp.rows, n, kps);
    const long rows = (long)sp.rows * a.H;
    if (n == 1 || th >= rows) return;
    float M = -INFINITY;
    for (int s = lane; s < n; s += 64) {
        const float l = a.part_l[s * rows + th];
        M = fmaxf(M, is_nan(l) ? 0.f : l);               // (not a row without keys)
    }
    M = wave_max(M);
    const float ref = M == -INFINITY ? 0.f : M;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float z = 0.f;
    for (int c0 = 0; c0 < n; c0 += 64) {
        const float w = c0 + lane < n ? expf(a.part_l[(c0 + lane) * rows + th] - ref) : 0.f;
        z += w;
        const int m = min(64, n - c0);
        for (int j0 = 0; j0 < m; j0 += NG) {             // (one load after another)
            const int j = min(j0 + grp, m - 1);
            float wj = __shfl(w, j, 64);
            wj = j0 + grp < m ? wj : 0.f;
            const f32x4 v = *(const f32x4*)(a.part_o + ((c0 + j) * rows + th) * D + col * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)                  // (weight 0: the output may not be written)
                acc[i] = wj != 0.f ? fmaf(wj, v[i], acc[i]) : acc[i];
        }
    }
    z = wave_sum(z);
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor(acc[i], o, 64);
    const float inv = M == -INFINITY ? 0.f : 1.0f / z;
    if (grp == 0) *(f32x4*)(a.out + th * D + col * 4) = acc * inv;
    if (a.lse && lane == 0) a.lse[th] = M == -INFINITY ? M : M + logf(z);
}

}  // namespace

// Workgroups of the launch and partial rows of each part: a step of fewer rows than the batch
// has room for is split further, up to kBaWgs workgroups of kBaRows rows.  float32: never into more
// splits than its keys fill, since empty workgroups cost too (of 16 waves, 2 requests over 2732
// keys: 20.6 us with room for kBaF32Parts of them, 14.2).
BatchAttnWorkspace batch_attn_layout(const relaxkv_problem& p, const relaxkv_batch& b, int block,
                                     int n_sel) {
    BatchAttnWorkspace w = {};
    if (b.n_rows == 0) return w;
    const long G = p.H / p.H_kv, rows = (long)b.n_rows * p.H;
    if (p.dtype == RELAXKV_DTYPE_F32) {
        // (with more than one split, kBaF32Parts workgroups of kBatchRowsF32 rows at most; listed, one
        // round)
        const long most = n_sel == 0 ? kBaF32Parts : kBaF32ListWgs;
        auto wgs = [&](long items, long keys) {
            const int unit = n_sel == 0 ? kBaF32Keys : kBaF32ListKeys;
            items *= p.H_kv;
            // (a step of i <= items takes one split, or as many as are kBaF32Wgs workgroups, and
            // kBaF32More)
            const long i = std::min(items, (long)kBaF32Items);
            const long round = n_sel == 0 ? std::min(std::max(i, (long)kBaF32Wgs) + i * kBaF32More, most) : most;
            return std::min(std::max(items, round), items * ((keys + unit - 1) / unit));
        };
        const size_t parts = n_sel == 0 ? 2 * std::max(most * kBatchRowsF32, rows) : most * kBatchRowsF32;
        w.ctx_wgs = (int)(n_sel == 0 ? wgs((b.n_rows * G + kBatchRowsF32 - 1) / kBatchRowsF32, p.T_c) +
                                           wgs(b.tile_cap, b.max_suffix)
                                     : wgs(b.n_rows * ((G + kBatchRowsF32 - 1) / kBatchRowsF32),
                                           (long)n_sel * block + b.max_suffix + kBaF32ListKeys));
        w.part_s_off = parts * p.d * 4;
        w.total = w.part_s_off + parts * 4;
        return w;
    }
    const long least = (long)kBaWgs * kBaRows;
    const long item_cap = (b.n_rows * G + kBaRows - 1) / kBaRows * p.H_kv;
    const long list_items = (long)b.n_rows * p.H_kv * ((G + kBaRows - 1) / kBaRows);
    const long suf_items = (long)b.tile_cap * p.H_kv;
    auto wgs = [](long items) {
        return (int)((items > kBaWgs ? items + kBaXcds - 1 : kBaWgs) / kBaXcds * kBaXcds);
    };
    w.ctx_wgs = n_sel == 0 ? kBaWgs : wgs(list_items);
    w.suf_wgs = wgs(suf_items);
    w.suf_part = n_sel == 0 ? (kBaWgs + item_cap) * kBaRows : rows > least ? rows : least;
    const size_t parts = w.suf_part + (rows > least ? rows : least);
    w.part_s_off = (parts * p.d * 2 + 255) / 256 * 256;
    w.total = w.part_s_off + (parts * 16 + 255) / 256 * 256;
    return w;
}

hipError_t launch_batch_attn(const relaxkv_problem& p, const relaxkv_batch& b, int layer,
                             const void* k_cache, const void* v_cache, const void* q,
                             const relaxkv_suffix& suf, int block, const int32_t* blocks, int n_sel,
                             void* out, float* lse_out, char* ws, hipStream_t st) {
    const int G = p.H / p.H_kv;
    const bool list = n_sel > 0;
    const float scale = p.softmax_scale > 0.f ? p.softmax_scale : 1.0f / sqrtf((float)p.d);
    const KvStrides ks = kv_strides(p);
    const SuffixStrides ss = suffix_strides(p, b, suf);
    const size_t layer_off = (size_t)(layer * ks.layer);
    const int bshift = list ? __builtin_ctz(block) : 0;
    const int nb = list ? block_count(p, block) : 0;
    const int tail = list ? p.T_c % block : 0;
    if (p.dtype == RELAXKV_DTYPE_F32) {
        BaF32Args a;
        a.q = (const float*)q;
        a.kc = (const float*)k_cache + layer_off;
        a.vc = (const float*)v_cache + layer_off;
        a.ks = (const float*)suf.k;
        a.vs = (const float*)suf.v;
        a.c_sh = ks.head;
        a.c_st = ks.token;
        a.s_ss = ss.seq;
        a.s_sh = ss.head;
        a.s_st = ss.token;
        a.counts = b.counts;
        a.row_seq = b.row_seq;
        a.row_pos = b.row_pos;
        a.lists = blocks;
        a.tiles = (const BatchTile*)b.tiles;
        a.T = p.T_c;
        a.H = p.H;
        a.Hkv = p.H_kv;
        a.G = G;
        a.n_sel = n_sel;
        a.bshift = bshift;
        a.nb = nb;
        a.tail = tail;
        a.scale = scale;
        a.out = (float*)out;
        a.lse = lse_out;
        const BatchAttnWorkspace w = batch_attn_layout(p, b, block, n_sel);
        a.list_items = p.H_kv * ((G + kBatchRowsF32 - 1) / kBatchRowsF32);
        a.list_tiles = (int)(((long)n_sel * block + kBaF32ListKeys - 1) / kBaF32ListKeys);
        a.part_o = (float*)ws;
        a.part_l = (float*)(ws + w.part_s_off);
        auto go = [&](auto d_t, auto list_t) {
            constexpr int D = decltype(d_t)::value;
            constexpr bool LIST = decltype(list_t)::value;
            // (a launch dimension holds fewer than 2^32 threads)
            const unsigned nx = std::min(w.ctx_wgs, 1 << 20);
            hipLaunchKernelGGL((battn_f32<D, LIST>), dim3(nx, (w.ctx_wgs + nx - 1) / nx), dim3(f32_waves<LIST>() * 64),
                               sizeof(AttnF32Lds<D, kBatchRowsF32, f32_waves<LIST>()>) + (LIST ? (n_sel + 2) * sizeof(int) : 0),
                               st, a);
            hipLaunchKernelGGL((batch_merge_f32<D, LIST>), dim3((unsigned)(((long)b.n_rows * p.H + 3) / 4)),
                               dim3(256), 0, st, a);
        };
        if (p.d == 128) {
            if (list) go(Int<128>{}, Int<1>{});
            else go(Int<128>{}, Int<0>{});
        } else {
            if (list) go(Int<64>{}, Int<1>{});
            else go(Int<64>{}, Int<0>{});
        }
        return hipGetLastError();
    }
    const BatchAttnWorkspace w = batch_attn_layout(p, b, block, n_sel);
    BaArgs a;
    a.q = (const uint16_t*)q;
    a.kc = (const uint16_t*)k_cache + layer_off;
    a.vc = (const uint16_t*)v_cache + layer_off;
    a.ks = (const uint16_t*)suf.k;
    a.vs = (const uint16_t*)suf.v;
    a.c_sh = ks.head;
    a.c_st = ks.token;
    a.s_ss = ss.seq;
    a.s_sh = ss.head;
    a.s_st = ss.token;
    a.counts = b.counts;
    a.row_pos = b.row_pos;
    a.tiles = (const BatchTile*)b.tiles;
    a.lists = blocks;
    a.part_o = (_Float16*)ws;
    a.part_s = (float4*)(ws + w.part_s_off);
    a.suf_part = w.suf_part;
    a.T = p.T_c;
    a.H = p.H;
    a.Hkv = p.H_kv;
    a.G = G;
    a.n_sel = n_sel;
    a.bshift = bshift;
    a.nb = nb;
    a.tail = tail;
    a.ctx_wgs = w.ctx_wgs;
    a.suf_wgs = w.suf_wgs;
    a.list_items = p.H_kv * ((G + kBaRows - 1) / kBaRows);
    a.list_tiles = (int)(((long)n_sel * block + kBaKeys - 1) / kBaKeys);
    a.sl2 = scale * kLog2e;
    // (workgroups for a wave per row; with D/8 lanes per row most of them have none)
    const unsigned merges = (unsigned)(((long)b.n_rows * p.H + 3) / 4);
    auto go = [&](auto d_t, auto list_t) {
        constexpr int D = decltype(d_t)::value;
        constexpr bool LIST = decltype(list_t)::value;
        hipLaunchKernelGGL((battn_bf16<D, LIST>), dim3(w.ctx_wgs + w.suf_wgs), dim3(kBaWaves * 64),
                           LIST ? n_sel * sizeof(int) : 0, st, a);
        hipLaunchKernelGGL((batch_merge<D, LIST>), dim3(merges), dim3(256), 0, st, a, (uint16_t*)out,
                           lse_out);
    };
    if (p.d == 128) {
        if (list) go(Int<128>{}, Int<1>{});
        else go(Int<128>{}, Int<0>{});
    } else {
        if (list) go(Int<64>{}, Int<1>{});
        else go(Int<64>{}, Int<0>{});
    }
    return hipGetLastError();
}

}  // namespace relaxkv
