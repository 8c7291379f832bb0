// Attention of a batch's rows over one shared context cache and, causally, each row's own
// request's suffix; and the same over listed context blocks instead of the whole context.
//
//   O_t = sum_j softmax_j(sigma <q_t, K_j>) V_j,   j over the context keys (all, or those of
//   the row's listed blocks) and then the suffix tokens of the row's request up to its own.
//
// bf16: one launch of independent work items, then a merge.
// - Context items.  Shared: the (token, head) rows of ALL requests of a KV head in chunks of
//   128, times one split of the keys, so K and V are read once for the batch and not
//   once per request.  The chunks of one split are consecutive on one XCD, whose L2 then
//   serves all but the first.  Listed: one token's group of heads, times one split of its
//   listed keys; the list is first compacted into LDS (full blocks, then copies of a
//   partial last block), so that every key below the count is one the row sees.
// - Suffix items: 128 rows of one request, times one split of its keys, causal.
// - Each item streams 64-key K and V tiles through two swizzled LDS buffers by direct loads;
//   64 KB of LDS let two workgroups share a CU, so that one's softmax and waits overlap
//   the other's matrix products.  A wave owns 32 rows (one per lane): S^T = K Q^T, online
//   softmax in the exp2 domain with a lazily raised maximum, O^T += V^T P^T.
// - Probabilities are rounded to bf16 for the second product (2^-9 of each, independent over
//   keys: about as much as rounding O once; fp32 products would take eight times the matrix
//   time).  The output is divided by the sum of the rounded ones, which keeps a row that
//   sees one key exact, the log-sum-exp uses the sum of the exact ones.
// - Every item writes its unnormalised float32 output and (max, sums); batch_merge adds them
//   with weights exp2(max_s - max) in a fixed order.
// A row that sees no key gets O = 0 and lse = -inf.
// Loads never leave a run's keys (past its end they repeat its last key, masked), so cache
// rows past the context and suffix tokens past a request's length are never read.
//
// float32: the MFMA core of attn_f32.h, 16 rows of one request per workgroup over all of
// their keys.

#include <math.h>

#include "attn_f32.h"
#include "batch.h"
#include "dev_common.h"

namespace relaxkv {
namespace {

constexpr int kBaKeys = 64;            // keys per tile
constexpr int kBaStages = 2;           // LDS ring depth
constexpr int kBaWaves = kBatchRowsBf16 / 32;
constexpr int kBaRing = 4;             // K fragments read ahead of their MFMA
constexpr float kBaSlack = 8.0f;       // log2 units the running max may lag the true max
constexpr long kBaWgs = 512;           // workgroups the key splits aim for (two per CU)
constexpr long kBaMinSplit = 256;      // fewest keys per split
constexpr int kBaXcds = 8;

template <int N> struct Int { static constexpr int value = N; };

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

struct BaArgs {
    const uint16_t* q;       // [n_rows][H][D]
    const uint16_t *kc, *vc; // this layer's cache: key i of KV head g at g * c_sh + i * c_st
    const uint16_t *ks, *vs; // suffixes: key i of request b at b * s_ss + g * s_sh + i * s_st
    int64_t c_sh, c_st, s_ss, s_sh, s_st;
    const int32_t* counts;
    const BatchTile* tiles;
    const int32_t* lists;    // [n_rows][Hkv][n_sel]
    float* part_o;           // [slot][Hkv][n_rows * G][D]
    float4* part_s;          // [slot][Hkv][n_rows * G]
    int T, H, Hkv, G, n_rows, n_sel, bshift, nb, tail;
    int n_ctx, kps, n_suf, kss, n_chunks, ctx_items;
    float sl2;               // softmax scale * log2(e)
};

__device__ __forceinline__ float ba_pair_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float ba_pair_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
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
__global__ __launch_bounds__(kBaWaves * 64, 2) void battn_bf16(BaArgs a) {
    constexpr int TK = kBaKeys, ST = kBaStages, NW = kBaWaves;
    constexpr int KS = D / 16;             // k-steps of QK^T
    constexpr int DB = D / 32;             // 32-wide d blocks of O^T
    constexpr int NKB = TK / 32;
    constexpr int ROWB = 2 * D;            // tile row bytes
    constexpr int CH = D / 8;              // 16-byte chunks per row
    constexpr int RPI = 64 / CH;           // rows per wave-wide load
    constexpr int NL = TK / RPI;           // wave-wide loads per tile and tensor
    constexpr int NI = NL / NW;            // of them per wave
    constexpr int LPW = 2 * NI;            // K and V
    static_assert(NL % NW == 0, "loader shape");
    __shared__ __attribute__((aligned(1024))) uint16_t Kt[ST][TK * D];
    __shared__ __attribute__((aligned(1024))) uint16_t Vt[ST][TK * D];
    __shared__ int lst[LIST ? RELAXKV_MAX_SELECTED_BLOCKS : 1], cnt[2];

    const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, hf = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int id = blockIdx.x;
    const int rows = min(a.counts[0], a.n_rows);
    const bool ctx = id < a.ctx_items;

    // The item: KV head g, partial slot, the lane's row (token t, head hh of the group, last
    // visible key lim), and its keys key0 .. key0 + nk - 1 of a run (base pointers, stride).
    int g, slot, t, hh, lim, key0, nk, open;             // open: keys that every row sees
    bool valid;
    const uint16_t *kb, *vb;
    int64_t st;
    bool listed = false;
    if (ctx) {
        if constexpr (LIST) {
            slot = id % a.n_ctx;
            int x = id / a.n_ctx;
            const int chunk = x % a.n_chunks;
            x /= a.n_chunks;
            g = x % a.Hkv;
            t = x / a.Hkv;
            if (t >= rows) return;
            compact_list(a.lists + ((size_t)t * a.Hkv + g) * a.n_sel, a.n_sel, a.nb, a.tail, lst, cnt);
            hh = chunk * kBatchRowsBf16 + w * 32 + r32;
            valid = hh < a.G;
            if (!valid) hh = 0;
            key0 = slot * a.kps;
            const int n = __builtin_amdgcn_readfirstlane((cnt[0] << a.bshift) + cnt[1] * a.tail);
            nk = min(a.kps, n - key0);
            if (nk <= 0) {                               // nothing in this split
                if (valid && hf == 0)
                    a.part_s[((size_t)slot * a.Hkv + g) * ((size_t)a.n_rows * a.G) + (size_t)t * a.G + hh] =
                        float4{-INFINITY, 0.f, 0.f, 0.f};
                return;
            }
            listed = true;
        } else {
            // (the chunks of one (split, head) pair are consecutive workgroups of one XCD)
            const int x = id / kBaXcds, chunk = x % a.n_chunks;
            const int pair = x / a.n_chunks * kBaXcds + id % kBaXcds;
            if (pair >= a.n_ctx * a.Hkv) return;
            g = pair % a.Hkv;
            slot = pair / a.Hkv;
            const int row0 = chunk * kBatchRowsBf16;
            if (row0 >= rows * a.G) return;
            const int rho = row0 + w * 32 + r32;
            valid = rho < rows * a.G;
            t = valid ? rho / a.G : 0;
            hh = valid ? rho - t * a.G : 0;
            key0 = slot * a.kps;
            nk = min(a.kps, a.T - key0);
        }
        lim = nk - 1;
        open = nk;
        kb = a.kc + g * a.c_sh;
        vb = a.vc + g * a.c_sh;
        st = a.c_st;
    } else {
        int x = id - a.ctx_items;
        const int split = x % a.n_suf;
        x /= a.n_suf;
        g = x % a.Hkv;
        x /= a.Hkv;
        const int n_tiles = a.counts[1];
        BatchTile tl = a.tiles[x];                       // (tiles past the count: unspecified)
        if (x >= n_tiles) return;
        tl.seq = __builtin_amdgcn_readfirstlane(tl.seq);
        tl.row_begin = __builtin_amdgcn_readfirstlane(tl.row_begin);
        tl.n_new = __builtin_amdgcn_readfirstlane(tl.n_new);
        tl.past = __builtin_amdgcn_readfirstlane(tl.past);
        tl.row0 = __builtin_amdgcn_readfirstlane(tl.row0);
        slot = a.n_ctx + split;
        key0 = split * a.kss;
        const int n_th = tl.n_new * a.G;                 // (token, head) rows of the request
        const int last = (min(tl.row0 + kBatchRowsBf16, n_th) - 1) / a.G;
        nk = min(a.kss, tl.past + last + 1 - key0);
        if (nk <= 0) return;
        const int rq = tl.row0 + w * 32 + r32;
        valid = rq < n_th;
        const int tr = valid ? rq / a.G : 0;
        hh = valid ? rq - tr * a.G : 0;
        t = tl.row_begin + tr;
        lim = tl.past + tr - key0;
        open = min(nk, tl.past + tl.row0 / a.G + 1 - key0);
        valid = valid && lim >= 0;                       // (the merge reads no others)
        kb = a.ks + tl.seq * a.s_ss + g * a.s_sh;
        vb = a.vs + tl.seq * a.s_ss + g * a.s_sh;
        st = a.s_st;
    }
    const bool live = __any(valid);
    const int ntile = (nk + TK - 1) / TK;

    bf16x8 qf[KS];
    {
        const uint16_t* qrow = a.q + ((size_t)t * a.H + g * a.G + hh) * D;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const bf16x8*)(qrow + ks * 16 + hf * 8);
        // Consumed here, so the compiler's waits for these loads stay before the loop.
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
    }
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x16{};
    float m_run = -INFINITY, l_run = 0.f, l_exact = 0.f;

    // Loader: load jj = w + NW i fills tile rows jj RPI ..; lane l writes (row l / CH, chunk
    // l % CH) and fetches the chunk that belongs there.  The swizzle of a lane's rows is the
    // same for every i (NW RPI is a multiple of its period), so in full tiles of a run a
    // lane's byte offset is constant and the base is wave-uniform.
    const int lrow = lane / CH, pchunk = lane % CH;
    static_assert((NW * RPI) % 16 == 0, "the swizzle repeats every 16 rows");
    const int ch8 = (pchunk ^ tile_swz<D>(w * RPI + lrow)) << 3;
    const uint32_t lane_off = (uint32_t)(lrow * (int)st + ch8) * 2u;
    const uint32_t kt0 = lds_addr(Kt[0]) + w * RPI * ROWB, vt0 = lds_addr(Vt[0]) + w * RPI * ROWB;
    auto issue = [&](int tt) {
        const uint32_t so = (uint32_t)(tt % ST) * (TK * ROWB);
        if (!listed && (tt + 1) * TK <= nk) {
            const int64_t e0 = (int64_t)(key0 + tt * TK + w * RPI) * st;
            const uint16_t *kp = kb + e0, *vp = vb + e0;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                fill_lds16_u(kp + (int64_t)(NW * RPI * i) * st, lane_off, kt0 + so + i * (NW * RPI * ROWB));
                fill_lds16_u(vp + (int64_t)(NW * RPI * i) * st, lane_off, vt0 + so + i * (NW * RPI * ROWB));
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

    // Fragment byte offsets: K rows r32 (+ 32 kb), chunk hf (+ 2 ks); V by transposing reads.
    const int k_base = r32 * ROWB | ((hf ^ tile_swz<D>(r32)) << 4);
    const int rl = 4 * (lane >> 5) + ((lane & 15) >> 2);
    const int cl = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    const int v_base0 = rl * ROWB | ((cl ^ tile_swz<D>(rl)) << 4) | ((lane & 1) << 3);
    const int v_base1 = (rl + 8) * ROWB | ((cl ^ tile_swz<D>(rl + 8)) << 4) | ((lane & 1) << 3);
    const char* kst = (const char*)Kt[0];
    const uint32_t vlds = lds_addr(Vt[0]);

    auto step = [&](uint32_t stage, int c0, bool masked) {
        int kbo = k_base + (int)stage;
        uint32_t vb0 = v_base0 + vlds + stage, vb1 = v_base1 + vlds + stage;
        asm volatile("" : "+v"(kbo), "+v"(vb0), "+v"(vb1));
        // S^T = K Q^T: s[kb][v] = S[row][key c0 + 32kb + 8(v/4) + 4hf + v%4]
        f32x16 s[NKB];
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) s[kb] = f32x16{};
        auto frag = [&](int x) {                       // x = NKB ks + kb
            return *(const bf16x8*)(kst + (x % NKB) * 32 * ROWB + (kbo ^ ((x / NKB) << 5)));
        };
        bf16x8 kf[kBaRing];
#pragma unroll
        for (int i = 0; i < kBaRing; ++i) kf[i] = frag(i);
#pragma unroll
        for (int x = 0; x < NKB * KS; ++x) {
            const bf16x8 cur = kf[x % kBaRing];
            if (x + kBaRing < NKB * KS) kf[x % kBaRing] = frag(x + kBaRing);
            s[x % NKB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cur, qf[x / NKB], s[x % NKB], 0, 0, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, kBaRing, 0);
#pragma unroll
        for (int x = 0; x < NKB * KS; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (x + kBaRing < NKB * KS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        if (masked) {                                  // the run's tail, or the causal future
            const int e = lim - c0 - 4 * hf;
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (32 * kb + 8 * (v >> 2) + (v & 3) > e) s[kb][v] = -INFINITY;
        }
        float mk[NKB];
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
            mk[kb] = fmaxf(s[kb][0], s[kb][1]);
#pragma unroll
            for (int v = 2; v < 16; v += 2) mk[kb] = fmaxf(fmaxf(mk[kb], s[kb][v]), s[kb][v + 1]);
        }
        const float mx = ba_pair_max(fmaxf(mk[0], mk[NKB - 1])) * a.sl2;
        if (__any(mx > m_run + kBaSlack)) {
            const float m_new = mx > m_run + kBaSlack ? mx : m_run;
            const float alpha = m_new == m_run ? 1.f : fast_exp2(m_run - m_new);
            l_run *= alpha;
            l_exact *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db] *= alpha;
            m_run = m_new;
        }
        // (a row with no visible key so far adds exact zeros)
        const float m_ref = m_run == -INFINITY ? 0.f : m_run;
        bf16x8 pb[NKB][2];
        float e0 = 0.f, e1 = 0.f, e2 = 0.f, e3 = 0.f;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float p = fast_exp2(fmaf(s[kb][v], a.sl2, -m_ref));
                ((v & 3) == 0 ? e0 : (v & 3) == 1 ? e1 : (v & 3) == 2 ? e2 : e3) += p;
                pb[kb][v >> 3][v & 7] = (__bf16)p;
            }
        l_exact += (e0 + e1) + (e2 + e3);
        {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            const bf16x2 one2 = {(__bf16)1.0f, (__bf16)1.0f};
            float ls0 = 0.f, ls1 = 0.f, ls2 = 0.f, ls3 = 0.f;
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                for (int k2 = 0; k2 < 2; ++k2) {
                    const bf16x8 q8 = pb[kb][k2];
                    ls0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(q8, q8, 0, 1), one2, ls0, false);
                    ls1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(q8, q8, 2, 3), one2, ls1, false);
                    ls2 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(q8, q8, 4, 5), one2, ls2, false);
                    ls3 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(q8, q8, 6, 7), one2, ls3, false);
                }
            l_run += (ls0 + ls1) + (ls2 + ls3);
        }
        // O^T += V^T P^T
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int k2 = 0; k2 < 2; ++k2) {
                    const uint32_t rowo = (kb * 32 + k2 * 16) * ROWB;
                    const v4i16 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (lds_v4i16*)(uintptr_t)((vb0 ^ (db << 6)) + rowo));
                    const v4i16 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (lds_v4i16*)(uintptr_t)((vb1 ^ (db << 6)) + rowo));
                    const bf16x8 vv = __builtin_bit_cast(
                        bf16x8, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vv, pb[kb][k2], o[db], 0, 0, 0);
                }
    };

#pragma unroll
    for (int tt = 0; tt < ST - 1; ++tt)
        if (tt < ntile) issue(tt);
    for (int tt = 0; tt < ntile; ++tt) {
        // Tile tt has landed, and every wave is done with the buffer that is filled next.
        wait_loads_barrier<0>();
        if (tt + ST - 1 < ntile) issue(tt + ST - 1);
        if (live) step((uint32_t)(tt % ST) * (TK * ROWB), tt * TK, (tt + 1) * TK > open);
    }

    const float l_tot = ba_pair_sum(l_run), l_ex = ba_pair_sum(l_exact);
    if (!valid) return;
    const size_t prow = ((size_t)slot * a.Hkv + g) * ((size_t)a.n_rows * a.G) + (size_t)t * a.G + hh;
    float* po = a.part_o + prow * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            *(f32x4*)(po + db * 32 + 8 * j + 4 * hf) =
                f32x4{o[db][4 * j], o[db][4 * j + 1], o[db][4 * j + 2], o[db][4 * j + 3]};
    if (hf == 0) a.part_s[prow] = float4{m_run, l_tot, l_ex, 0.f};
}

// D/4 lanes per (token, head): the context slots in order, then the suffix slots that hold
// one of the row's keys.
template <int D>
__global__ __launch_bounds__(256) void batch_merge(const float* __restrict__ part_o,
                                                   const float4* __restrict__ part_s, int n_ctx,
                                                   int kss, const int32_t* __restrict__ counts,
                                                   const int32_t* __restrict__ row_pos, int T, int H,
                                                   int Hkv, int G, int n_rows,
                                                   uint16_t* __restrict__ out,
                                                   float* __restrict__ lse) {
    constexpr int LPR = D / 4;
    const int lane = threadIdx.x % LPR;
    const long th = (long)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int t = (int)(th / H), h = (int)(th - (long)t * H);
    if (t >= min(counts[0], n_rows)) return;
    const int g = h / G;
    const int n = n_ctx + (row_pos[t] - T) / kss + 1;
    const size_t stride = (size_t)Hkv * n_rows * G;           // between slots
    const size_t row = (size_t)g * n_rows * G + (size_t)t * G + (h - g * G);
    float M = -INFINITY;
    for (int s = lane; s < n; s += LPR) M = fmaxf(M, part_s[s * stride + row].x);
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float z = 0.f, ze = 0.f;
#pragma unroll 4
    for (int s = 0; s < n; ++s) {
        const float4 st = part_s[s * stride + row];
        if (st.x == -INFINITY) continue;                      // (its output is not written)
        const f32x4 v = *(const f32x4*)(part_o + (s * stride + row) * D + lane * 4);
        const float wt = fast_exp2(st.x - M);
        z = fmaf(wt, st.y, z);
        ze = fmaf(wt, st.z, ze);
        acc += wt * v;
    }
    const float inv = M == -INFINITY ? 0.f : 1.0f / z;
    uint16_t* dst = out + (size_t)th * D + lane * 4;
    u32x2 r;
    r[0] = (uint32_t)f32_to_bf16_bits(acc[0] * inv) | ((uint32_t)f32_to_bf16_bits(acc[1] * inv) << 16);
    r[1] = (uint32_t)f32_to_bf16_bits(acc[2] * inv) | ((uint32_t)f32_to_bf16_bits(acc[3] * inv) << 16);
    *(u32x2*)dst = r;
    if (lse && lane == 0) lse[th] = M == -INFINITY ? -INFINITY : (M + __log2f(ze)) * kLn2;
}

// float32: rows of one request per workgroup; key c is context key c (or listed key c) below
// the context count, suffix token c - count from there.
struct BaF32Args {
    const float *q, *kc, *vc, *ks, *vs;
    int64_t c_sh, c_st, s_ss, s_sh, s_st;
    const int32_t *counts, *row_seq, *row_pos, *lists;
    const BatchTile* tiles;
    int T, H, Hkv, G, n_rows, n_sel, bshift, nb, tail;
    float scale;
    float *out, *lse;
};

template <int D, bool LIST>
__global__ __launch_bounds__(MfmaF32<16>::waves * 64) void battn_f32(BaF32Args a) {
    constexpr int R = kBatchRowsF32;
    extern __shared__ __attribute__((aligned(16))) char f32_lds[];
    AttnF32Lds<D, R>& sm = *(AttnF32Lds<D, R>*)f32_lds;
    int* lst = (int*)(f32_lds + sizeof(AttnF32Lds<D, R>));
    const int g = blockIdx.y, rl = threadIdx.x % R;
    const int rows = min(a.counts[0], a.n_rows);
    int t, hh, seq, own, last_own, n_ctx = a.T;
    bool valid;
    if constexpr (LIST) {
        const int chunks = (a.G + R - 1) / R;
        t = blockIdx.x / chunks;
        if (t >= rows) return;
        hh = (blockIdx.x % chunks) * R + rl;
        valid = hh < a.G;
        if (!valid) hh = a.G - 1;
        compact_list(a.lists + ((size_t)t * a.Hkv + g) * a.n_sel, a.n_sel, a.nb, a.tail, lst + 2, lst);
        n_ctx = (lst[0] << a.bshift) + lst[1] * a.tail;
        seq = a.row_seq[t];
        own = last_own = a.row_pos[t] - a.T;
    } else {
        if ((int)blockIdx.x >= a.counts[1]) return;
        const BatchTile tl = a.tiles[blockIdx.x];
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
    const int h = g * a.G + hh;
    const uint32_t orow = (uint32_t)t * a.H + h;
    auto id_of = [&](int c) {
        if (c >= n_ctx) return c - n_ctx;
        if constexpr (LIST) return ~list_key(c, lst + 2, lst[0], a.bshift, a.nb, a.tail);
        else return ~c;
    };
    const int64_t sb = seq * a.s_ss + g * a.s_sh;
    attn_f32_rows<D, R>(sm, a.ks + sb, a.vs + sb, a.s_st, a.kc + g * a.c_sh, a.vc + g * a.c_sh,
                        a.c_st, id_of, n_ctx + last_own + 1, a.q + (size_t)orow * D, n_ctx + own,
                        a.scale, valid, a.out, a.lse, orow);
}

}  // namespace

BatchAttnWorkspace batch_attn_layout(const relaxkv_problem& p, const relaxkv_batch& b, int block,
                                     int n_sel) {
    BatchAttnWorkspace w = {};
    if (p.dtype != RELAXKV_DTYPE_BF16) return w;
    const int G = p.H / p.H_kv;
    const bool list = n_sel > 0;
    // Keys per split so that about kBaWgs workgroups are launched, whole tiles, not too few.
    auto split = [](long keys, long items, int& kps, int& n) {
        const long want = items >= kBaWgs ? 1 : kBaWgs / items;
        long k = (keys + want - 1) / want;
        k = (k + kBaKeys - 1) / kBaKeys * kBaKeys;
        kps = (int)(k < kBaMinSplit ? kBaMinSplit : k);
        n = (int)((keys + kps - 1) / kps);
    };
    const long rows = (long)b.n_rows * G;
    w.n_chunks = list ? (G + kBatchRowsBf16 - 1) / kBatchRowsBf16
                      : (int)((rows + kBatchRowsBf16 - 1) / kBatchRowsBf16);
    const long ctx_items = (list ? (long)b.n_rows : 1) * p.H_kv * w.n_chunks;
    const long ctx_keys = list ? (long)n_sel * block : p.T_c;
    split(ctx_keys, ctx_items > 0 ? ctx_items : 1, w.kps, w.n_ctx);
    const long suf_items = (long)b.tile_cap * p.H_kv;
    split(b.max_suffix, suf_items > 0 ? suf_items : 1, w.kss, w.n_suf);
    const size_t slots = (size_t)(w.n_ctx + w.n_suf) * p.H_kv * (size_t)rows;
    w.part_s_off = (slots * p.d * 4 + 255) / 256 * 256;
    w.total = w.part_s_off + (slots * 16 + 255) / 256 * 256;
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
        a.n_rows = b.n_rows;
        a.n_sel = n_sel;
        a.bshift = bshift;
        a.nb = nb;
        a.tail = tail;
        a.scale = scale;
        a.out = (float*)out;
        a.lse = lse_out;
        const int chunks = (G + kBatchRowsF32 - 1) / kBatchRowsF32;
        const unsigned gx = list ? (unsigned)(b.n_rows * chunks) : (unsigned)b.tile_cap;
        auto go = [&](auto kernel, size_t lds) {
            hipLaunchKernelGGL(kernel, dim3(gx, p.H_kv), dim3(MfmaF32<16>::waves * 64),
                               lds + (list ? (n_sel + 2) * sizeof(int) : 0), st, a);
        };
        if (p.d == 128) {
            if (list) go(battn_f32<128, true>, sizeof(AttnF32Lds<128, 16>));
            else go(battn_f32<128, false>, sizeof(AttnF32Lds<128, 16>));
        } else {
            if (list) go(battn_f32<64, true>, sizeof(AttnF32Lds<64, 16>));
            else go(battn_f32<64, false>, sizeof(AttnF32Lds<64, 16>));
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
    a.tiles = (const BatchTile*)b.tiles;
    a.lists = blocks;
    a.part_o = (float*)ws;
    a.part_s = (float4*)(ws + w.part_s_off);
    a.T = p.T_c;
    a.H = p.H;
    a.Hkv = p.H_kv;
    a.G = G;
    a.n_rows = b.n_rows;
    a.n_sel = n_sel;
    a.bshift = bshift;
    a.nb = nb;
    a.tail = tail;
    a.n_ctx = w.n_ctx;
    a.kps = w.kps;
    a.n_suf = w.n_suf;
    a.kss = w.kss;
    a.n_chunks = w.n_chunks;
    a.sl2 = scale * kLog2e;
    const int pairs = w.n_ctx * p.H_kv;
    a.ctx_items = list ? b.n_rows * p.H_kv * w.n_chunks * w.n_ctx
                       : (pairs + kBaXcds - 1) / kBaXcds * kBaXcds * w.n_chunks;
    const unsigned items = (unsigned)a.ctx_items + (unsigned)(b.tile_cap * p.H_kv * w.n_suf);
    const unsigned merges = (unsigned)(((long)b.n_rows * p.H * (p.d / 4) + 255) / 256);
    auto go = [&](auto d_t) {
        constexpr int D = decltype(d_t)::value;
        if (list) hipLaunchKernelGGL((battn_bf16<D, true>), dim3(items), dim3(kBaWaves * 64), 0, st, a);
        else hipLaunchKernelGGL((battn_bf16<D, false>), dim3(items), dim3(kBaWaves * 64), 0, st, a);
        hipLaunchKernelGGL((batch_merge<D>), dim3(merges), dim3(256), 0, st, (const float*)a.part_o,
                           (const float4*)a.part_s, a.n_ctx, a.kss, b.counts, b.row_pos, p.T_c, p.H,
                           p.H_kv, G, b.n_rows, (uint16_t*)out, lse_out);
    };
    if (p.d == 128) go(Int<128>{});
    else go(Int<64>{});
    return hipGetLastError();
}

}  // namespace relaxkv
