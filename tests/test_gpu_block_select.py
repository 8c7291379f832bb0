"""Row maps, key block means and block selection: integers equal to the oracle's, means equal
to the float64 mean rounded once."""

import numpy as np
import pytest
import torch

from batch_harness import Step, f64
from oracle import batch_oracle as bo
from paper_2609_33503_amd import relaxkv

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def request(T, H=8, H_kv=2, d=128, dtype=BF, L=1, spare=0, seed=0, token_major=False):
    g = torch.Generator().manual_seed(seed)
    if token_major:
        k = torch.randn(L, T + spare, H_kv, d, generator=g).to(dtype).cuda().transpose(1, 2)[:, :, :T]
    else:
        k = torch.randn(L, H_kv, T + spare, d, generator=g).to(dtype).cuda()[:, :, :T]
    return relaxkv.Request(torch.zeros(L, 1, H, d, dtype=dtype, device="cuda"), k, k, 0.15), k


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,d,H_kv,L,block,kw", [
    (1, 64, 1, 1, 16, {}), (16, 128, 2, 1, 16, {}), (17, 128, 2, 2, 16, {}), (127, 64, 3, 1, 128, {}),
    (1003, 64, 2, 2, 32, dict(spare=21)), (700, 128, 4, 3, 64, dict(token_major=True)),
    (513, 128, 1, 1, 128, {})])
def test_means(gpu_lib, T, d, H_kv, L, block, kw, dtype):
    req, k = request(T, H_kv=H_kv, H=H_kv, d=d, L=L, dtype=dtype, **kw)
    nb = req.block_count(block)
    rounded = bo.round_bf16 if dtype == BF else lambda x: x.astype(np.float32)
    allm = torch.zeros(L, H_kv, nb, d, dtype=dtype, device="cuda")
    req.block_means(None, k, block, allm)
    for l in range(L):
        want = rounded(bo.block_means(f64(k[l]), block))
        assert np.array_equal(f64(allm[l]), want.astype(np.float64)), l
        one = torch.zeros(1, H_kv, nb, d, dtype=dtype, device="cuda")
        req.block_means(l, k, block, one)
        assert torch.equal(one[0], allm[l])


def test_means_not_finite(gpu_lib):
    """NaN and Inf reach their own block and element alone; the largest values do not overflow."""
    req, k = request(64, H=1, H_kv=1, d=64)
    top = torch.finfo(BF).max
    k[0, 0, :16] = top
    k[0, 0, 17, 3] = float("nan")
    k[0, 0, 40, 5] = float("-inf")
    m = torch.zeros(1, 1, 4, 64, dtype=BF, device="cuda")
    req.block_means(0, k, 16, m)
    m = f64(m)[0, 0]
    assert np.all(m[0] == top)
    assert np.isnan(m[1, 3]) and np.isfinite(np.delete(m[1], 3)).all()
    assert np.isneginf(m[2, 5]) and np.isfinite(np.delete(m[2], 5)).all() and np.isfinite(m[3]).all()


def select(req, new, means, q, block, sel, room=64, extra=0):
    n = sum(new)
    batch = req.alloc_batch(len(new), n + extra, room)
    z = torch.zeros(len(new), dtype=torch.int32, device="cuda")
    req.plan_batch(batch, z, torch.tensor(new, dtype=torch.int32, device="cuda"))
    out = torch.full((n + extra, req.H_kv, sel), -7, dtype=torch.int32, device="cuda")
    req.block_select(batch, block, means, q, out, req.alloc_block_workspace(batch, block, sel))
    got = out.cpu().numpy()
    assert np.all(got[n:] == -7)
    return got[:n]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,H,H_kv,d,block,sel,new,extra", [
    (1, 1, 1, 64, 16, 1, [1], 0), (100, 8, 2, 128, 16, 7, [1, 1, 2], 0),
    (100, 8, 2, 128, 16, 1, [1], 3), (64 * 64, 10, 2, 128, 64, 63, [1, 5], 1),
    (64 * 64 + 1, 10, 2, 64, 64, 65, [9], 0), (16 * 1024, 4, 4, 64, 16, 37, [1, 1, 17], 0),
    (16 * 1025, 24, 2, 64, 16, 100, [3], 0), (16 * 4096, 4, 1, 64, 16, 2048, [2], 0),
    (16 * 4097, 4, 1, 64, 16, 33, [2], 0), (16 * 20000, 2, 1, 64, 16, 1000, [2, 1], 1)])
def test_select(gpu_lib, T, H, H_kv, d, block, sel, new, extra, dtype):
    req, _ = request(T, H=H, H_kv=H_kv, d=d, dtype=dtype)
    g = torch.Generator().manual_seed(T + sel)
    n, nb = sum(new), req.block_count(block)
    means = torch.randn(H_kv, nb, d, generator=g).to(dtype).cuda()
    q = torch.randn(n + extra, H, d, generator=g).to(dtype).cuda()
    got = select(req, new, means, q, block, sel, extra=extra)
    assert np.array_equal(got, bo.block_select(f64(q)[:n], f64(means), sel))


@pytest.mark.parametrize("nb", [40, 300, 2000, 5000])
def test_select_ties_and_odd_scores(gpu_lib, nb):
    """Few distinct scores, signed zeros, infinities and NaN: ties go to the lower block, a NaN
    is below every number."""
    req, _ = request(nb * 16, H=2, H_kv=1, d=64)
    r = np.random.default_rng(nb)
    means = torch.zeros(1, nb, 64, dtype=BF)
    means[0, :, 0] = torch.from_numpy(r.choice([-2.0, -0.0, 0.0, 1.0, 3.0], nb)).to(BF)
    means[0, 5, 0], means[0, 7, 0], means[0, 11, 0] = float("nan"), float("inf"), float("-inf")
    q = torch.zeros(1, 2, 64, dtype=BF)
    q[:, :, 0] = 0.5
    for sel in (1, 2, 17, nb - 2, nb):
        if sel > 2048:
            continue
        got = select(req, [1], means.cuda(), q.cuda(), 16, sel)
        s = means[0, :, 0].double().numpy() + 0.0
        key = np.where(np.isnan(s), -np.inf, s)
        # -inf is a number: above the NaN
        order = np.lexsort((np.arange(nb), np.isnan(s), -key))
        assert np.array_equal(got[0, 0], np.sort(order[:sel])), sel


def test_select_one_of_many_rows_alike(gpu_lib):
    """A row's list does not depend on the rows beside it."""
    req, _ = request(4000, H=6, H_kv=3, d=128)
    g = torch.Generator().manual_seed(4)
    means = torch.randn(3, 63, 128, generator=g).to(BF).cuda()
    q = torch.randn(21, 6, 128, generator=g).to(BF).cuda()
    got = select(req, [21], means, q, 64, 9)
    for t in (0, 7, 8, 20):
        assert np.array_equal(select(req, [1], means, q[t:t + 1].contiguous(), 64, 9)[0], got[t])


# ------------------------------------------------------------------ row maps

def plan(req, past, new, n_rows, room):
    b = req.alloc_batch(len(past), n_rows, room)
    b.buf.fill_(99)
    req.plan_batch(b, *(torch.tensor(v, dtype=torch.int32, device="cuda") for v in (past, new)))
    return b


@pytest.mark.parametrize("past,new,n_rows", [
    ([0], [1], 1), ([0], [0], 0), ([5], [0], 3), ([0, 3, 9], [2, 0, 5], 7), ([1] * 64, [1] * 64, 64),
    ([2] * 65, [1] * 65, 70), ([0] * 200, [3] * 200, 600), ([0], [3000], 3001),
    (list(range(700)), [i % 5 for i in range(700)], 1500), ([7] * 5000, [1] * 5000, 5003),
    ([0] * 65536, [1, 0] * 32768, 32768)])
@pytest.mark.parametrize("H,H_kv,dtype", [(8, 2, BF), (40, 8, F32), (200, 1, BF)])
def test_plan(gpu_lib, past, new, n_rows, H, H_kv, dtype):
    req, _ = request(100, H=H, H_kv=H_kv, d=64, dtype=dtype)
    if n_rows * H > 1 << 22:                              # more row heads than a batch takes
        with pytest.raises(ValueError):
            req.alloc_batch(len(past), n_rows, 4000)
        return
    b = plan(req, past, new, n_rows, 4000)
    off, seq, pos = bo.batch_plan(past, new, 100)
    n, tile, G = len(seq), 128 if dtype == BF else 16, H // H_kv
    assert np.array_equal(b.row_off.cpu().numpy(), off)
    for got, want in ((b.row_seq, seq), (b.row_pos, pos)):
        got = got.cpu().numpy()
        assert np.array_equal(got[:n], want) and np.all(got[n:] == -1)
    tiles = [(s, off[s], k, past[s], r) for s, k in enumerate(new) for r in range(0, k * G, tile)]
    longest = max([p + k for p, k in zip(past, new) if k], default=0)
    assert b.counts_to_host() == [n, len(tiles), longest, 0]
    at = b.s.tiles - b.buf.data_ptr()
    rec = b.buf[at:at + 32 * len(tiles)].view(torch.int32).view(-1, 8).cpu().numpy()
    assert np.array_equal(rec[:, :5], np.array(tiles, dtype=np.int64).reshape(-1, 5))


@pytest.mark.parametrize("past,new", [
    ([-1, 0], [1, 1]), ([0, 0], [1, -1]), ([50, 0], [1, 1]), ([0, 51], [1, 0]), ([0, 0], [6, 5]),
    ([0, 0], [11, 0]), ([2 ** 31 - 1, 0], [1, 1]), ([0, 0], [2 ** 31 - 1, 2 ** 31 - 1]),
    ([-2 ** 31, 0], [1, 1]), ([0] * 99 + [51], [0] * 100)])
def test_plan_bad_lengths(gpu_lib, past, new):
    """One bad length anywhere, or more rows than there is room for, empties the plan."""
    req, _ = request(100)
    b = plan(req, past, new, 10, 50)
    assert b.counts_to_host(check=False) == [0, 0, 0, relaxkv.BATCH_ERR_LENGTHS]
    assert torch.all(b.row_off == 0) and torch.all(b.row_seq == -1) and torch.all(b.row_pos == -1)
    with pytest.raises(relaxkv.RelaxKVError):
        b.counts_to_host()
    # and a good step afterwards clears the word
    ok = [0] * len(past)
    req.plan_batch(b, *(torch.tensor(v, dtype=torch.int32, device="cuda") for v in (ok, ok)))
    assert b.counts_to_host() == [0, 0, 0, 0]


def test_refusals(gpu_lib):
    req, k = request(100)
    b = req.alloc_batch(2, 4, 50)
    z = torch.zeros(2, dtype=torch.int32, device="cuda")
    for args in ((b, z.long(), z), (b, z, z[:1]), (b, z.cpu(), z), (None, z, z)):
        with pytest.raises(ValueError):
            req.plan_batch(*args)
    for args in ((0, 1, 1), (1, -1, 1), (1, 1, 0), (1 << 17, 1, 1), (1, 1 << 17, 1)):
        with pytest.raises(ValueError):
            req.alloc_batch(*args)
    req.plan_batch(b, z, z)
    m = torch.zeros(1, 2, 7, 128, dtype=BF, device="cuda")
    req.block_means(0, k, 16, m)
    for args in ((1, k, 16, m), (-1, k, 16, m), (0, k, 0, m), (0, k, 32, m), (0, k.float(), 16, m),
                 (0, k, 16, m.float()), (0, k, 16, m[0])):
        with pytest.raises(ValueError):
            req.block_means(*args)
    with pytest.raises(relaxkv.RelaxKVError):
        req.block_means(0, k, 15, m)
    q = torch.zeros(4, 8, 128, dtype=BF, device="cuda")
    out = torch.zeros(4, 2, 3, dtype=torch.int32, device="cuda")
    ws = req.alloc_block_workspace(b, 16, 3)
    req.block_select(b, 16, m[0], q, out, ws)
    for args in ((b, 16, m, q, out, ws), (b, 16, m[0], q[:3], out, ws), (b, 32, m[0], q, out, ws),
                 (b, 16, m[0], q, out.long(), ws), (b, 16, m[0], q, out[:3], ws), (b, 16, m[0], q, out, None)):
        with pytest.raises(ValueError):
            req.block_select(*args)
    with pytest.raises(relaxkv.RelaxKVError):
        req.block_select(b, 16, m[0], q, out, ws[:16])
    with pytest.raises(relaxkv.RelaxKVError):
        req.block_select(b, 16, m[0], q, torch.zeros(4, 2, 8, dtype=torch.int32, device="cuda"), ws)
    torch.cuda.synchronize()
