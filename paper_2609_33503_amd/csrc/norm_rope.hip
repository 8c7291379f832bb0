// Norms of queries and keys per head with the position rotation in the same pass, values
// copied: the rows that the attention calls take as "already rotated".
//
// One head x of a row at position P (w absent: no norm):
//   y_i = x_i / sqrt(mean_j x_j^2 + eps) * w_i;
//   (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = P f_i,
// for the pairs (a, b) = (i, i + rot/2), or (2i, 2i+1) interleaved, i < rot/2; the rest of
// the head is not rotated.  Everything is float32 and rounded once to the output type.
//
// Memory bound: each row is read and written once.  A group of d/16 lanes takes a head of a
// row; a lane holds the two 8-element chunks whose elements pair up (chunk c and c + rot/16,
// or neighbours when interleaved), so the rotation needs no exchange and the norm three (two
// at d 64).  The pair's 8 angles are those of 8 consecutive frequencies either way: the
// workgroup computes the angles of its rows once, into LDS, for all heads.
// Angles: P f_i is exact in 64 bits (f_i is float32) and is reduced to an eighth of a turn
// there, so positions of millions lose nothing; sine and cosine are their Taylor sums up to
// a^9 and a^10, whose remainders are below 2e-9 for |a| <= pi/4.
// 16411 rows of 40 query and 8 key/value heads, d 128, from a fused projection: 82 us, 5.7 TB/s (float32
// 168, 5.6).  Fewer rows: the launch and its dependent loads (2.9 us for 4 rows), then the copy rate
// (3001 float32 rows of 12 and 3 heads, d 64: 8.9 us; twice as many 15.0, 4.6 TB/s of what is added).

#include <algorithm>

#include "batch.h"
#include "dev_common.h"

namespace relaxkv {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeRows = 4;           // rows per workgroup at most

struct RopeArgs {
    const char *q, *k, *v;             // input rows (null: none)
    char *q_out, *k_out, *v_out;
    const char *qw, *kw;               // norm weights (null: no norm)
    const float* freq;
    const int32_t* pos;                // position of each row
    const int32_t* seq;                // batch: the request of each row (null: dense rows)
    const int32_t* counts;             // batch: rows of the step
    int64_t q_st, k_st, v_st;          // input row strides (elements)
    SuffixStrides ss;
    int n, H, Hkv, T, rot, inter;
    float eps;
};

template <typename T> struct Chunk;    // 8 consecutive elements as float
template <> struct Chunk<uint16_t> {
    u32x4 r;
    __device__ __forceinline__ void load(const uint16_t* p) { r = *(const u32x4*)p; }
    __device__ __forceinline__ void store(uint16_t* p) const { *(u32x4*)p = r; }
    __device__ __forceinline__ void get(float* f) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(r[i] << 16);
            f[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            const bf16x2 b = {(__bf16)f[2 * i], (__bf16)f[2 * i + 1]};
            r[i] = __builtin_bit_cast(uint32_t, b);
        }
    }
};
template <> struct Chunk<float> {
    f32x4 r[2];
    __device__ __forceinline__ void load(const float* p) {
        r[0] = *(const f32x4*)p;
        r[1] = *(const f32x4*)(p + 4);
    }
    __device__ __forceinline__ void store(float* p) const {
        *(f32x4*)p = r[0];
        *(f32x4*)(p + 4) = r[1];
    }
    __device__ __forceinline__ void get(float* f) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = r[i >> 2][i & 3];
    }
    __device__ __forceinline__ void set(const float* f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i >> 2][i & 3] = f[i];
    }
};

// cos and sin of pos * freq (NaN for a frequency that is not finite).
__device__ __forceinline__ void rotation(int pos, float freq, float& c, float& s) {
    const double quarters = (double)pos * (double)freq * 0.63661977236758134308;   // * 2 / pi
    const double n = __builtin_rint(quarters);
    const float a = (float)((quarters - n) * 1.57079632679489661923);              // |a| <= pi/4
    const float z = a * a;
    float sp = fmaf(z, 1.f / 362880, -1.f / 5040), cp = fmaf(z, -1.f / 3628800, 1.f / 40320);
    sp = fmaf(z, sp, 1.f / 120);
    cp = fmaf(z, cp, -1.f / 720);
    sp = fmaf(z, sp, -1.f / 6);
    cp = fmaf(z, cp, 1.f / 24);
    sp = fmaf(z * a, sp, a);
    cp = fmaf(z, cp, -0.5f);
    cp = fmaf(z, cp, 1.f);
    const int q = (int)(n - 4.0 * __builtin_floor(n * 0.25)) & 3;
    const float x = (q & 1) ? sp : cp, y = (q & 1) ? cp : sp;
    c = (q == 1 || q == 2) ? -x : x;
    s = q >= 2 ? -y : y;
}

template <typename T, int D>
__global__ __launch_bounds__(kRopeThreads) void norm_rope(RopeArgs a, int rows_per_wg) {
    constexpr int LPH = D / 16;                     // lanes per head
    constexpr int GROUPS = kRopeThreads / LPH;
    __shared__ float cs[kRopeRows][D / 2], sn[kRopeRows][D / 2];
    __shared__ float wt[2][D];
    const int tid = threadIdx.x;
    const int row0 = blockIdx.x * rows_per_wg;
    const int n = a.counts ? min(a.n, a.counts[0]) : a.n;
    if (row0 >= n) return;
    const int nr = min(rows_per_wg, n - row0);
    const int half = a.rot / 2;
    for (int i = tid; i < nr * half; i += kRopeThreads) {
        const int r = i / half, f = i - r * half;
        rotation(a.pos[row0 + r], a.freq[f], cs[r][f], sn[r][f]);
    }
    for (int i = tid; i < 2 * D; i += kRopeThreads) {
        const T* w = (const T*)(i < D ? a.qw : a.kw);
        float x = 1.f;
        if (w) {
            if constexpr (sizeof(T) == 2) x = bf16_bits_to_f32(w[i & (D - 1)]);
            else x = w[i & (D - 1)];
        }
        wt[i / D][i & (D - 1)] = x;
    }
    __syncthreads();
    const int grp = tid / LPH, j = tid % LPH;
    // The lane's two chunks: a pair to rotate (j below rot/16), or two to pass on.
    const int hc = a.rot / 16;
    const bool turn = j < hc;
    const int ca = a.inter ? 2 * j : turn ? j : 2 * j;
    const int cb = a.inter || !turn ? ca + 1 : j + hc;
    const int nq = a.q ? a.H : 0, nk = a.k ? a.Hkv : 0, nv = a.v ? a.Hkv : 0;
    const int heads = nq + nk + nv;
    for (int u = grp; u < nr * heads; u += GROUPS) {
        const int rl = u / heads, h = u - rl * heads, row = row0 + rl;
        const int kind = h < nq ? 0 : h < nq + nk ? 1 : 2;
        const int hh = kind == 0 ? h : kind == 1 ? h - nq : h - nq - nk;
        const T* src = kind == 0 ? (const T*)a.q + row * a.q_st
                     : kind == 1 ? (const T*)a.k + row * a.k_st : (const T*)a.v + row * a.v_st;
        src += hh * D;
        Chunk<T> A, B;
        A.load(src + ca * 8);
        B.load(src + cb * 8);
        T* dst;
        if (kind == 0) {
            dst = (T*)a.q_out + ((size_t)row * a.H + hh) * D;
        } else {
            dst = (T*)(kind == 1 ? a.k_out : a.v_out);
            if (a.seq)
                dst += a.seq[row] * a.ss.seq + hh * a.ss.head + (a.pos[row] - a.T) * a.ss.token;
            else
                dst += ((size_t)row * a.Hkv + hh) * D;
        }
        if (kind < 2) {
            float x[8], y[8];
            A.get(x);
            B.get(y);
            const bool norm = kind == 0 ? a.qw != nullptr : a.kw != nullptr;
            if (norm) {
                float q = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) q = fmaf(x[i], x[i], fmaf(y[i], y[i], q));
#pragma unroll
                for (int o = LPH / 2; o > 0; o >>= 1) q += __shfl_xor(q, o, 64);
                const float sc = 1.0f / sqrtf(q * (1.0f / D) + a.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] = x[i] * sc * wt[kind][ca * 8 + i];
                    y[i] = y[i] * sc * wt[kind][cb * 8 + i];
                }
            }
            if (turn) {
                const float* c = &cs[rl][j * 8];
                const float* s = &sn[rl][j * 8];
                if (a.inter) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float* e = i < 4 ? &x[2 * i] : &y[2 * i - 8];
                        const float p = e[0], r = e[1];
                        e[0] = p * c[i] - r * s[i];
                        e[1] = r * c[i] + p * s[i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float p = x[i], r = y[i];
                        x[i] = p * c[i] - r * s[i];
                        y[i] = r * c[i] + p * s[i];
                    }
                }
            }
            if (norm || turn) {
                A.set(x);
                B.set(y);
            }
        }
        A.store(dst + ca * 8);
        B.store(dst + cb * 8);
    }
}

template <typename T, int D>
void launch(const RopeArgs& a, hipStream_t st) {
    // As many rows per workgroup as give each group of lanes a head (16411 rows of 12 heads, d 64:
    // 11.2 us, 19.2 with one row; of 56 heads, d 128: 83.5 with one, 93.9 with four), but one
    // until that fills the chip four times over (1024 rows of 18 float32 heads, d 128: 5.2, 8.1
    // with four).
    const int heads = (a.q ? a.H : 0) + (a.k ? a.Hkv : 0) + (a.v ? a.Hkv : 0);
    constexpr int GROUPS = kRopeThreads / (D / 16);
    int rows = a.n > 1024 ? std::min(kRopeRows, (GROUPS + heads - 1) / heads) : 1;
    // A launch dimension holds fewer than 2^32 threads.
    static_assert(RELAXKV_MAX_FRESH_ROWS / kRopeRows * (int64_t)kRopeThreads < (int64_t)1 << 32, "every call fits");
    while ((int64_t)((a.n + rows - 1) / rows) * kRopeThreads >= (int64_t)1 << 32) ++rows;
    hipLaunchKernelGGL((norm_rope<T, D>), dim3((a.n + rows - 1) / rows), dim3(kRopeThreads), 0, st,
                       a, rows);
}

}  // namespace

hipError_t launch_norm_rope(const relaxkv_problem& p, const relaxkv_rope& r,
                            const relaxkv_rows& in, const int32_t* positions,
                            const relaxkv_batch* b, void* q_out, void* k_out, void* v_out,
                            SuffixStrides ss, hipStream_t st) {
    RopeArgs a;
    a.q = (const char*)in.q;
    a.k = (const char*)in.k;
    a.v = (const char*)in.v;
    a.q_out = (char*)q_out;
    a.k_out = (char*)k_out;
    a.v_out = (char*)v_out;
    a.qw = (const char*)r.q_weight;
    a.kw = (const char*)r.k_weight;
    a.freq = r.inv_freq;
    a.pos = b ? b->row_pos : positions;
    a.seq = b ? b->row_seq : nullptr;
    a.counts = b ? b->counts : nullptr;
    a.q_st = in.q_stride ? in.q_stride : (int64_t)p.H * p.d;
    a.k_st = in.k_stride ? in.k_stride : (int64_t)p.H_kv * p.d;
    a.v_st = in.v_stride ? in.v_stride : (int64_t)p.H_kv * p.d;
    a.ss = ss;
    a.n = in.n_rows;
    a.H = p.H;
    a.Hkv = p.H_kv;
    a.T = p.T_c;
    a.rot = r.rot;
    a.inter = r.interleaved;
    a.eps = r.eps;
    if (p.dtype == RELAXKV_DTYPE_BF16) {
        if (p.d == 128) launch<uint16_t, 128>(a, st);
        else launch<uint16_t, 64>(a, st);
    } else {
        if (p.d == 128) launch<float, 128>(a, st);
        else launch<float, 64>(a, st);
    }
    return hipGetLastError();
}

}  // namespace relaxkv
