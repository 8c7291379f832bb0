// Block means of the cached keys, and the context blocks that a score by those means
// selects for each row and KV head.
//
//   m_j = (1 / n_j) sum_{i in block j} k_i                          (64-bit sums, rounded once)
//   s_j = float32( sum_c (sum_{h in group} q_{h,c}) m_{j,c} )       (64-bit sums)
//   the n_sel largest s_j, equal ones to the lower block, in ascending block order.
//
// A selection is only as reproducible as its scores: float32 sums of another order differ in
// the last bits and swap blocks near the border.  Products of two bf16 (or float32) values
// are exact in 64 bits and their sums there are off by 2^-53, so the score that is
// rounded to float32 is, but for one in about 2^28, the same whatever the order of its sum.
// The 64-bit rate of the chip (half its float32 rate) makes that cheap: 2 nb d operations
// per row and KV head, against 4 G d per key of the attention that follows.
//
// block_means is memory bound (reads every key once: 40 layers of 8 heads, 16K keys, d 128 in 234 us,
// 5.8 TB/s); the scores' products are few (8 rows and 8 heads, 2048 blocks, d 128: 4.3 us, of
// which the launch and the first loads are most), and the top-k of up to 4096 blocks keeps its
// keys in registers.

#include <algorithm>

#include "batch.h"
#include "dev_common.h"

namespace relaxkv {
namespace {

template <typename T> __device__ __forceinline__ void load8(const T* p, float* f);
template <> __device__ __forceinline__ void load8<uint16_t>(const uint16_t* p, float* f) {
    const u32x4 r = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(r[i] << 16);
        f[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
}
template <> __device__ __forceinline__ void load8<float>(const float* p, float* f) {
    const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = a[i];
        f[4 + i] = b[i];
    }
}

// One wave per block: D/8 lanes take a key's row, 512/D keys at a time.
template <typename T, int D>
__global__ __launch_bounds__(256) void block_means(const T* __restrict__ k, KvStrides ks,
                                                   int layer0, int n_heads, int Hkv, int nb, int T_c,
                                                   int block, T* __restrict__ means) {
    constexpr int LPK = D / 8, KPW = 64 / LPK;
    const int lane = threadIdx.x & 63, c = lane % LPK, r = lane / LPK;
    const long units = (long)n_heads * nb;                        // (layer, head, block)
    for (long unit = blockIdx.x * 4l + (threadIdx.x >> 6); unit < units; unit += gridDim.x * 4l) {
        const int lg = (int)(unit / nb), j = (int)(unit - (long)lg * nb);
        const int l = lg / Hkv, g = lg - l * Hkv;
        const int i0 = j * block, n = min(block, T_c - i0);
        const T* src = k + (layer0 + l) * ks.layer + g * ks.head + (int64_t)i0 * ks.token + c * 8;
        double acc[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.0;
#pragma unroll 4
        for (int i = r; i < n; i += KPW) {
            float f[8];
            load8<T>(src + i * ks.token, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += (double)f[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int o = LPK; o < 64; o <<= 1) acc[e] += __shfl_xor(acc[e], o, 64);
        if (r == 0) {
            T* dst = means + unit * D + c * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double m = acc[e] / n;
                if constexpr (sizeof(T) == 4) {
                    dst[e] = (float)m;
                } else {
                    // Rounded once: through float32 to odd (a truncated float32 whose last bit
                    // remembers what was cut off), from which the rounding to bf16 is that of m.
                    float x = (float)m;
                    uint32_t u = __float_as_uint(x);
                    if ((double)x != m && x == x) {
                        if (fabs((double)x) > fabs(m)) --u;
                        u |= 1;
                    }
                    dst[e] = (u & 0x7fffffffu) > 0x7f800000u ? (uint16_t)((u >> 16) | 0x40)
                                                             : f32_to_bf16_bits(__uint_as_float(u));
                }
            }
        }
    }
}

// 16 rows against 64 blocks of a KV head per workgroup, on the 64-bit matrix instruction (16x16x4):
// a wave takes 16 blocks, lane r + 16 k the elements [k d/4, (k + 1) d/4) of row r's summed queries
// and of block r's mean, so that step i multiplies element k d/4 + i for the four k.
// (58 rows and 8 heads, 3125 blocks, d 128: 16.8 us; with vector multiply-adds, whose queries
// come from LDS two at a time, 24.)
constexpr int kScoreRows = 16;
template <typename T, int D>
__global__ __launch_bounds__(256) void block_scores(const T* __restrict__ q,
                                                    const T* __restrict__ means,
                                                    const int32_t* __restrict__ counts, int n_rows,
                                                    int H, int Hkv, int G, int nb,
                                                    float* __restrict__ scores) {
    typedef double f64x4 __attribute__((ext_vector_type(4)));
    typedef double f64x2 __attribute__((ext_vector_type(2)));
    constexpr int NR = kScoreRows, KD = D / 4;
    __shared__ __attribute__((aligned(16))) double qs[NR][D + 2];     // (rows in different banks)
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, kk = lane >> 4;
    const int g = blockIdx.y, t0 = blockIdx.z * NR, b = (blockIdx.x * 4 + (tid >> 6)) * 16 + r;
    const T* m = means + ((size_t)g * nb + min(b, nb - 1)) * D + kk * KD;
    float mf[KD];
#pragma unroll
    for (int i = 0; i < KD; i += 8) load8<T>(m + i, mf + i);
    const int rows = min(counts[0], n_rows);
    if (t0 >= rows) return;
    // The summed group queries: 8 elements of one row per thread, the heads' loads in flight
    // together.
    for (int x = tid; x < NR * D / 8; x += 256) {
        const int t = x / (D / 8), c = (x - t * (D / 8)) * 8;
        double s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = 0.0;
        if (t0 + t < rows) {
            const T* p = q + ((size_t)(t0 + t) * H + g * G) * D + c;
            for (int h0 = 0; h0 < G; h0 += 4) {
                float f[4][8];
#pragma unroll
                for (int h = 0; h < 4; ++h) load8<T>(p + min(h0 + h, G - 1) * D, f[h]);
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] += h0 + h < G ? (double)f[h][e] : 0.0;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) qs[t][c + e] = s[e];
    }
    __syncthreads();
    f64x4 acc = {0.0, 0.0, 0.0, 0.0}, acc1 = acc;
#pragma unroll
    for (int i = 0; i < KD; i += 2) {
        const f64x2 a = *(const f64x2*)&qs[r][kk * KD + i];
        acc = __builtin_amdgcn_mfma_f64_16x16x4f64(a[0], (double)mf[i], acc, 0, 0, 0);
        acc1 = __builtin_amdgcn_mfma_f64_16x16x4f64(a[1], (double)mf[i + 1], acc1, 0, 0, 0);
    }
    acc += acc1;
#pragma unroll
    for (int v = 0; v < 4; ++v) {                        // (row kk + 4 v, block r)
        const int t = t0 + kk + 4 * v;
        if (b < nb && t < rows) scores[((size_t)t * Hkv + g) * nb + b] = (float)acc[v];
    }
}

// Ascending with the score; -0 as +0; NaN below every number.
__device__ __forceinline__ uint32_t score_key(float f) {
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
    if (u == 0x80000000u) u = 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Inclusive prefix sum over the wave's lanes.
__device__ __forceinline__ int wave_scan_dpp(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);     // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, true);     // row_bcast:15, 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, true);
    return x;
}

// The k largest of a row's keys, by a workgroup of W waves: wave w holds the E * 64 blocks from
// w * E * 64, block e * 64 + lane of them in register e.  The k-th largest key is found 8 bits at
// a time from a histogram in LDS of the keys that share the bits found so far, in four copies
// (scores share few exponents, and an atomic takes a turn per lane of the same address); the
// next digit's histogram is cleared while this one is summed.  Blocks past the row's end hold
// key 0; a NaN's key 0 lies at a lower block, and k is at most the row's length, so none of
// them is ever taken.
// (2048 blocks, 64 rows of KV heads, k 32: 5.2 us with 8 waves, 5.8 with 4; 500 blocks 4.7 with 4
// waves, 6.5 with one; two bits at a time by counting keys in every wave 11.4, one wave per row and
// one bit at a time by ballots 42.)
template <int W>
struct TopkLds {
    int hist[2][4][256];
    int wsum[4], found[2];
    uint32_t part[W];
};

template <int W, int E, int NT = W * 64>   // (NT: threads of the workgroup)
__device__ __forceinline__ void topk_keys(TopkLds<W>& sm, const uint32_t (&key)[E], int k, int32_t* out) {
    constexpr int COPIES = 4;
    constexpr int SW = W < 4 ? W : 4, BPT = 256 / (SW * 64);   // waves that sum, bins per thread
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i0 = w * (E * 64) + lane;
    for (int i = tid; i < COPIES * 256; i += NT) sm.hist[0][0][i] = 0;
    __syncthreads();
    uint32_t t = 0;
    int need = k;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int shift = 24 - 8 * d, cur = d & 1;
        int (*h)[256] = sm.hist[cur];
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (w < W && (d == 0 || key[e] >> (shift + 8) == t >> (shift + 8)))
                atomicAdd(&h[lane & (COPIES - 1)][key[e] >> shift & 255], 1);
        __syncthreads();
        if (d < 3)
            for (int i = tid; i < COPIES * 256; i += NT) sm.hist[cur ^ 1][0][i] = 0;
        // Thread i sums the bins from 255 - i * BPT downwards.
        int c[BPT], sum = 0, incl = 0;
        if (w < SW) {
#pragma unroll
            for (int j = 0; j < BPT; ++j) {
                const int bin = 255 - tid * BPT - j;
                c[j] = h[0][bin] + h[1][bin] + h[2][bin] + h[3][bin];
                sum += c[j];
            }
            incl = wave_scan_dpp(sum);
            if (SW > 1 && lane == 63) sm.wsum[w] = incl;
        }
        if (SW > 1) __syncthreads();
        if (w < SW) {
            int before = incl - sum;
            if (SW > 1)
#pragma unroll
                for (int x = 0; x < SW; ++x) before += x < w ? sm.wsum[x] : 0;
#pragma unroll
            for (int j = 0; j < BPT; ++j) {
                if (before < need && before + c[j] >= need) {
                    sm.found[0] = 255 - tid * BPT - j;
                    sm.found[1] = before;
                }
                before += c[j];
            }
        }
        __syncthreads();
        t |= (uint32_t)sm.found[0] << shift;
        need -= sm.found[1];
    }
    // Every key above t, and of those equal to it the first `need`; in block order.
    int gt0 = 0, eq0 = 0;
    uint64_t mg[E], me[E];
    uint32_t own = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        mg[e] = __ballot(key[e] > t);
        me[e] = __ballot(key[e] == t);
        own += (uint32_t)__popcll(mg[e]) | (uint32_t)__popcll(me[e]) << 16;
    }
    if constexpr (W > 1) {
        if (w < W && lane == 0) sm.part[w] = own;
        __syncthreads();
#pragma unroll
        for (int x = 0; x < W; ++x) {
            const uint32_t p = x < w ? sm.part[x] : 0u;
            gt0 += p & 0xffff;
            eq0 += p >> 16;
        }
    }
    if (w >= W) return;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int gt = gt0 + lanes_below(mg[e]), eq = eq0 + lanes_below(me[e]);
        if (key[e] > t || (key[e] == t && eq < need)) out[gt + min(eq, need)] = i0 + e * 64;
        gt0 += __popcll(mg[e]);
        eq0 += __popcll(me[e]);
    }
}

// One workgroup per (row, KV head) over scores in memory.  The heads are the grid's second dimension:
// 2^22 units of 1024 threads are more than one dimension holds.
template <int W, int E>
__global__ __launch_bounds__(W * 64) void block_topk_reg(const float* __restrict__ scores, int nb,
                                                         int k, const int32_t* __restrict__ counts,
                                                         int n_rows, int Hkv,
                                                         int32_t* __restrict__ out) {
    __shared__ TopkLds<W> sm;
    const long unit = (long)blockIdx.x * Hkv + blockIdx.y;
    const int i0 = (threadIdx.x >> 6) * (E * 64) + (threadIdx.x & 63);
    const float* s = scores + unit * nb;                 // (within the workspace for every unit)
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = i0 + e * 64 < nb ? s[i0 + e * 64] : 0.f;
    if (unit >= (long)min(counts[0], n_rows) * Hkv) return;
    uint32_t key[E];
#pragma unroll
    for (int e = 0; e < E; ++e) key[e] = i0 + e * 64 < nb ? score_key(x[e]) : 0u;
    topk_keys<W, E>(sm, key, k, out + unit * k);
}

// Scores and top-k of one (row, KV head) in one workgroup: for steps of few rows, which are
// bound by the latency of a launch and not by a CU's 64-bit products.  Four lanes per block, each a
// quarter of the head dimension.  Per call, replayed, one launch and two (8 units, rows times KV
// heads, to 256):
//   d 64    250 blocks 5.4-6.1 us, 7.3-8.1;   1000 blocks 7.4-8.4, 7.6-8.5
//   d 128   250 blocks 5.9-6.6, 8.0-8.8;      500 blocks (in two passes) 8.2-13.7, 8.1-9.1
// (float32 and bf16; the means of a second pass at d 128 went through scratch memory): one launch for
// up to a block per thread at d 64 and one pass at d 128, and for one round of workgroups.
constexpr int kFusedThreads = 1024;
constexpr long kFusedUnits = 256;
inline int fused_blocks(const relaxkv_problem& p) {
    return p.d == 64 ? kFusedThreads : kFusedThreads / 4;
}
template <typename T, int D>
__global__ __launch_bounds__(kFusedThreads) void block_select_rows(const T* __restrict__ q,
                                                            const T* __restrict__ means, int nb, int k,
                                                            const int32_t* __restrict__ counts,
                                                            int n_rows, int H, int Hkv, int G,
                                                            int32_t* __restrict__ out) {
    constexpr int NT = kFusedThreads, NC = D / 32, BLK = NT / 4;   // chunks of a lane, blocks at a time
    constexpr int W = NT / 64;                           // (one block per thread in the top-k: nb <= NT)
    __shared__ TopkLds<W> sm;
    __shared__ float score[NT];
    __shared__ __attribute__((aligned(16))) double qs[D];
    const int tid = threadIdx.x, part = tid & 3;
    const int t = blockIdx.x / Hkv, g = blockIdx.x - t * Hkv;
    if (t >= min(counts[0], n_rows)) return;
    const T* m = means + (size_t)g * nb * D + part * 8;
    float mf[NC][8];
    auto load = [&](int b) {
#pragma unroll
        for (int i = 0; i < NC; ++i) load8<T>(m + (size_t)min(b, nb - 1) * D + i * 32, mf[i]);
    };
    load(tid >> 2);
    for (int c = tid; c < D; c += NT) {
        const T* p = q + ((size_t)t * H + g * G) * D + c;
        double s = 0.0;
#pragma unroll 4
        for (int h = 0; h < G; ++h) {
            if constexpr (sizeof(T) == 2) s += (double)bf16_bits_to_f32(p[h * D]);
            else s += (double)p[h * D];
        }
        qs[c] = s;
    }
    __syncthreads();
    for (int b0 = 0; b0 < (D == 64 ? nb : 1); b0 += BLK) {     // (d 128: nb <= BLK)
        const int b = b0 + (tid >> 2);
        double s = 0.0, s1 = 0.0;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            asm volatile("" ::: "memory");               // (the queries are read again, not kept)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                s = fma(qs[part * 8 + i * 32 + e], (double)mf[i][e], s);
                s1 = fma(qs[part * 8 + i * 32 + e + 1], (double)mf[i][e + 1], s1);
            }
        }
        if (D == 64 && b0 + BLK < nb) load(b + BLK);
        s += s1;
        s += __shfl_xor(s, 1, 64);
        s += __shfl_xor(s, 2, 64);
        if (part == 0 && b < nb) score[b] = (float)s;
    }
    __syncthreads();
    const uint32_t key[1] = {tid < nb ? score_key(score[min(tid, nb - 1)]) : 0u};
    topk_keys<W, 1>(sm, key, k, out + (size_t)blockIdx.x * k);
}

// Rows of any length: one workgroup per (row, KV head) reads its scores once per 8-bit
// digit and once for the compaction.
__global__ __launch_bounds__(256) void block_topk_long(const float* __restrict__ scores, int nb,
                                                       int k, const int32_t* __restrict__ counts,
                                                       int n_rows, int Hkv,
                                                       int32_t* __restrict__ out) {
    __shared__ int hist[256], scratch[4];
    __shared__ int digit_sh, above_sh;
    const long unit = (long)blockIdx.x * Hkv + blockIdx.y;
    const int tid = threadIdx.x;
    if (unit >= (long)min(counts[0], n_rows) * Hkv) return;
    const float* s = scores + unit * nb;
    uint32_t t = 0, mask = 0;
    int need = k;
    for (int shift = 24; shift >= 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < nb; i += 256) {
            const uint32_t key = score_key(s[i]);
            if ((key & mask) == t) atomicAdd(&hist[(key >> shift) & 255], 1);
        }
        __syncthreads();
        int total;
        const int h = hist[255 - tid];
        const int before = block_exclusive_scan<256>(h, scratch, total);
        if (before < need && before + h >= need) {
            digit_sh = 255 - tid;
            above_sh = before;
        }
        __syncthreads();
        t |= (uint32_t)digit_sh << shift;
        mask |= 255u << shift;
        need -= above_sh;
        __syncthreads();
    }
    int gt0 = 0, eq0 = 0;
    for (int i0 = 0; i0 < nb; i0 += 256) {
        const int i = i0 + tid;
        const uint32_t key = i < nb ? score_key(s[i]) : 0u;
        const bool g = i < nb && key > t, e = i < nb && key == t;
        int total;
        const int sc = block_exclusive_scan<256>((g ? 1 : 0) | (e ? 1 << 16 : 0), scratch, total);
        const int gt = gt0 + (sc & 0xffff), eq = eq0 + (sc >> 16);
        if (g || (e && eq < need)) out[unit * k + gt + min(eq, need)] = i;
        gt0 += total & 0xffff;
        eq0 += total >> 16;
    }
}

template <typename T, int D>
void launch_means(const relaxkv_problem& p, int layer0, int n_layers, const void* k, int block,
                  void* means, hipStream_t st) {
    const int nb = block_count(p, block), heads = n_layers * p.H_kv;
    const long units = (long)heads * nb;
    hipLaunchKernelGGL((block_means<T, D>), dim3((unsigned)std::min((units + 3) / 4, 1l << 22)), dim3(256), 0,
                       st, (const T*)k, kv_strides(p), layer0, heads, p.H_kv, nb, p.T_c, block,
                       (T*)means);
}

template <typename T, int D>
void launch_scores(const relaxkv_problem& p, const relaxkv_batch& b, int block, const void* means,
                   const void* q, float* scores, hipStream_t st) {
    const int nb = block_count(p, block);
    hipLaunchKernelGGL((block_scores<T, D>),
                       dim3((nb + 63) / 64, p.H_kv, (b.n_rows + kScoreRows - 1) / kScoreRows),
                       dim3(256), 0, st, (const T*)q, (const T*)means, b.counts, b.n_rows, p.H,
                       p.H_kv, p.H / p.H_kv, nb, scores);
}

}  // namespace

size_t block_select_bytes(const relaxkv_problem& p, const relaxkv_batch& b, int block) {
    return ((size_t)b.n_rows * p.H_kv * block_count(p, block) * 4 + 255) / 256 * 256;
}

hipError_t launch_block_means(const relaxkv_problem& p, int layer0, int n_layers,
                              const void* k_cache, int block, void* means, hipStream_t st) {
    if (p.dtype == RELAXKV_DTYPE_BF16) {
        if (p.d == 128) launch_means<uint16_t, 128>(p, layer0, n_layers, k_cache, block, means, st);
        else launch_means<uint16_t, 64>(p, layer0, n_layers, k_cache, block, means, st);
    } else {
        if (p.d == 128) launch_means<float, 128>(p, layer0, n_layers, k_cache, block, means, st);
        else launch_means<float, 64>(p, layer0, n_layers, k_cache, block, means, st);
    }
    return hipGetLastError();
}

hipError_t launch_block_select(const relaxkv_problem& p, const relaxkv_batch& b, int block,
                               const void* means, const void* q, int n_sel, int32_t* blocks,
                               float* scores, hipStream_t st) {
    const int nb = block_count(p, block);
    const long units = (long)b.n_rows * p.H_kv;
    if (nb <= fused_blocks(p) && units <= kFusedUnits) {
        auto go = [&](auto kernel, auto q_t) {
            typedef decltype(q_t) T;
            hipLaunchKernelGGL(kernel, dim3((unsigned)units), dim3(kFusedThreads), 0, st, (const T*)q,
                               (const T*)means, nb, n_sel, b.counts, b.n_rows, p.H, p.H_kv,
                               p.H / p.H_kv, blocks);
        };
        auto go_t = [&](auto q_t) {
            typedef decltype(q_t) T;
            if (p.d == 128) go(block_select_rows<T, 128>, q_t);
            else go(block_select_rows<T, 64>, q_t);
        };
        if (p.dtype == RELAXKV_DTYPE_BF16) go_t(uint16_t{});
        else go_t(float{});
        return hipGetLastError();
    }
    if (p.dtype == RELAXKV_DTYPE_BF16) {
        if (p.d == 128) launch_scores<uint16_t, 128>(p, b, block, means, q, scores, st);
        else launch_scores<uint16_t, 64>(p, b, block, means, q, scores, st);
    } else {
        if (p.d == 128) launch_scores<float, 128>(p, b, block, means, q, scores, st);
        else launch_scores<float, 64>(p, b, block, means, q, scores, st);
    }
    auto go = [&](auto kernel, int waves) {
        hipLaunchKernelGGL(kernel, dim3(b.n_rows, p.H_kv), dim3(waves * 64), 0, st, scores, nb, n_sel,
                           b.counts, b.n_rows, p.H_kv, blocks);
    };
    if (nb <= 512) go(block_topk_reg<4, 2>, 4);
    else if (nb <= 1024) go(block_topk_reg<8, 2>, 8);
    else if (nb <= 2048) go(block_topk_reg<8, 4>, 8);
    else if (nb <= 4096) go(block_topk_reg<16, 4>, 16);
    else go(block_topk_long, 4);
    return hipGetLastError();
}

}  // namespace relaxkv
