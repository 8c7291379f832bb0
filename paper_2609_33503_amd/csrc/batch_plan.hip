// Row maps of one step of a batch, from the requests' lengths.
//
//   row_off[b] = sum_{c < b} new_c;  row i of request b: row_seq = b, row_pos = T_c + past_b + i;
// rows behind the last hold -1; and the row tiles of the attention's suffix part.
//
// One launch, bound by latency (reads 8 bytes per request, writes 8 per row): every workgroup
// sums all lengths itself (the totals before its 64 requests, and whether any length is bad,
// which empties the whole plan), scans its own requests in LDS, and its threads take its rows
// one each, finding their request by binary search in that scan, so that one request of
// many rows is spread over the workgroup as many requests of one row are.
// 61 rows of 64 requests 5.6 us per call back to back, 27376 rows of 1500 requests 6.7 us.

#include "batch.h"
#include "dev_common.h"

namespace relaxkv {
namespace {

constexpr int kPlanThreads = 256;
constexpr int kPlanSeqs = 64;          // requests per workgroup

// The last entry of the ascending off[0 .. kPlanSeqs] that is <= x (x < off[kPlanSeqs]).
__device__ __forceinline__ int owner(const int* off, int x) {
    int lo = 0;
#pragma unroll
    for (int h = kPlanSeqs / 2; h > 0; h >>= 1)
        if (off[lo + h] <= x) lo += h;
    return lo;
}

__global__ __launch_bounds__(kPlanThreads) void batch_plan_rows(
    const int32_t* __restrict__ past_len, const int32_t* __restrict__ new_len, int n_seq,
    int n_rows, int max_suffix, int T, int G, int Hkv, int tile_rows, int32_t* __restrict__ row_off,
    int32_t* __restrict__ row_seq, int32_t* __restrict__ row_pos, BatchTile* __restrict__ tiles,
    int32_t* __restrict__ counts) {
    __shared__ long sums[4][6];
    __shared__ int off[kPlanSeqs + 1], toff[kPlanSeqs + 1], past_s[kPlanSeqs];
    const int tid = threadIdx.x, first = blockIdx.x * kPlanSeqs;
    // A length is bad below 0, past the suffix room, or past the rows of the step.
    auto lengths = [&](int b, int& n, int& p) {
        n = new_len[b];
        p = past_len[b];
        const bool ok = n >= 0 && p >= 0 && n <= n_rows && n <= max_suffix && p <= max_suffix - n;
        if (!ok) n = p = 0;
        return ok;
    };
    auto tiles_of = [&](int n) { return (n * G + tile_rows - 1) / tile_rows; };
    long total = 0, before = 0, tbefore = 0, ttotal = 0, bad = 0;
    int longest = 0;
    for (int b = tid; b < n_seq; b += kPlanThreads) {
        int n, p;
        if (!lengths(b, n, p)) bad = 1;
        const int t = tiles_of(n);
        total += n;
        ttotal += t;
        if (n) longest = max(longest, p + n);
        if (b < first) {
            before += n;
            tbefore += t;
        }
    }
    long part[6] = {total, ttotal, before, tbefore, bad, longest};
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < 6; ++i) {
            const long other = __shfl_xor(part[i], o, 64);
            part[i] = i < 5 ? part[i] + other : max(part[i], other);
        }
    if ((tid & 63) == 0)
#pragma unroll
        for (int i = 0; i < 6; ++i) sums[tid >> 6][i] = part[i];
    __syncthreads();
    auto sum = [&](int i) { return sums[0][i] + sums[1][i] + sums[2][i] + sums[3][i]; };
    total = sum(0);
    bad = sum(4) + (total > n_rows);
    if (bad) total = 0;
    ttotal = bad ? 0 : sum(1);
    before = bad ? 0 : sum(2);
    tbefore = bad ? 0 : sum(3);
    longest = bad ? 0 : (int)max(max(sums[0][5], sums[1][5]), max(sums[2][5], sums[3][5]));
    if (tid < kPlanSeqs) {                       // wave 0: one request per lane
        const int b = first + tid;
        int n = 0, p = 0;
        if (b < n_seq && !bad) lengths(b, n, p);
        const int t = tiles_of(n);
        const int ni = wave_inclusive_scan(n), ti = wave_inclusive_scan(t);
        off[tid + 1] = ni;
        toff[tid + 1] = ti;
        past_s[tid] = p;
        if (tid == 0) off[0] = toff[0] = 0;
        if (b < n_seq) row_off[b] = (int)before + ni - n;
        if (b == n_seq - 1) {
            row_off[n_seq] = (int)total;
            counts[0] = (int)total;
            counts[1] = (int)ttotal;
            counts[2] = longest;
            counts[3] = bad ? RELAXKV_BATCH_ERR_LENGTHS : 0;
        }
    }
    if (blockIdx.x == 0 && tid == kPlanThreads - 1)      // (beside wave 0's scan)
        *(BatchSplit*)(counts + kBatchSplitAt) = batch_split((int)total, (int)ttotal, longest, T, G, Hkv);
    __syncthreads();
    const int rows = off[kPlanSeqs], nt = toff[kPlanSeqs];
    for (int r = tid; r < rows; r += kPlanThreads) {
        const int j = owner(off, r);
        row_seq[before + r] = first + j;
        row_pos[before + r] = T + past_s[j] + r - off[j];
    }
    for (int x = tid; x < nt; x += kPlanThreads) {
        const int j = owner(toff, x);
        BatchTile t;
        t.seq = first + j;
        t.row_begin = (int)before + off[j];
        t.n_new = off[j + 1] - off[j];
        t.past = past_s[j];
        t.row0 = (x - toff[j]) * tile_rows;
        t.pad[0] = t.pad[1] = t.pad[2] = 0;
        tiles[tbefore + x] = t;
    }
    for (long r = total + (long)blockIdx.x * kPlanThreads + tid; r < n_rows;
         r += (long)gridDim.x * kPlanThreads)
        row_seq[r] = row_pos[r] = -1;
}

}  // namespace

hipError_t launch_batch_plan(const relaxkv_problem& p, const relaxkv_batch& b,
                             const int32_t* past_len, const int32_t* new_len, hipStream_t st) {
    hipLaunchKernelGGL(batch_plan_rows, dim3((b.n_seq + kPlanSeqs - 1) / kPlanSeqs),
                       dim3(kPlanThreads), 0, st, past_len, new_len, b.n_seq, b.n_rows,
                       b.max_suffix, p.T_c, p.H / p.H_kv, p.H_kv, batch_tile_rows(p), b.row_off, b.row_seq,
                       b.row_pos, (BatchTile*)b.tiles, b.counts);
    return hipGetLastError();
}

}  // namespace relaxkv
