"""Batched serving calls at the ends of their range: steps whose splits fill their launches, values
of any size next to one another; against the float64 oracle."""

import numpy as np
import pytest
import torch

from batch_harness import HALF, Step, attn_tol, f64
from oracle import batch_oracle as bo
from paper_2609_33503_amd import relaxkv

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("T,H,H_kv,d,past,new", [
    (4096, 64, 8, 64, [0], [112]),                # 448 context items of four splits, a suffix item per tile
    (2830, 24, 2, 128, [5] * 15 + [0], [7] * 15 + [85]),
    (5000, 20, 2, 64, [1, 9, 0], [80, 90, 70]),
])
def test_every_split_of_a_step_is_run(gpu_lib, T, H, H_kv, d, past, new):
    """float32 steps of 286 to 448 context items, in a workspace that holds NaN: a split that no
    workgroup takes would show.  A batch with more room gives the same bits."""
    room = max(p + n for p, n in zip(past, new))
    s, more = (Step(past=past, new=new, T=T, H=H, H_kv=H_kv, d=d, dtype=F32, seed=21, room=room + r, extra_rows=e)
               for r, e in ((0, 0), (300, 700)))
    for x in (s, more):
        ws = x.req.alloc_shared_workspace(x.batch)
        ws.view(torch.float32).fill_(float("nan"))
        x.shared(ws)
    s.check(s.reference())
    assert torch.equal(s.out, more.out[:s.n]) and torch.equal(s.lse, more.lse[:s.n])


def _needs(gb):
    torch.cuda.empty_cache()                         # (what earlier tests' tensors still hold)
    if torch.cuda.mem_get_info()[0] < gb << 30:
        pytest.skip(f"needs {gb} GB of device memory")


def _run(s, block):
    lists = None
    if block:
        nb = -(-s.T // block)
        lists = torch.arange(nb, dtype=torch.int32, device="cuda").expand(s.q.shape[0], s.H_kv, nb).contiguous()
        s.blocks(block, lists)
    else:
        s.shared()
    return s.reference(lists, block)


@pytest.mark.parametrize("block", [0, 64])
@pytest.mark.parametrize("kw", [
    dict(past=[0, 5, 200], new=[1, 1, 1], T=700),
    dict(past=[30], new=[1], T=9000, d=64),
    dict(past=[3, 40], new=[40, 1], T=300, H=12, H_kv=2),
    dict(past=[2] * 6, new=[9] * 6, T=2000, H=16, H_kv=4, d=64),
], ids=["decode", "splits", "wide", "chunks"])
@pytest.mark.parametrize("exps", [(0, -20), (0, -18, -26), (0, -30), (20, 0, -60), (60, -60)])
def test_channels_of_any_size(gpu_lib, exps, kw, block):
    """Value channels scaled by powers of two next to one another: a channel's output is that of
    the unscaled channel times its power, so its bound is too.  Elements more than 2^28 below a
    row's largest may be rounded to bf16 once more in each partial row: 2^-8 of each, with weights
    that sum to one at most 2^-8 sum_j p_j |V_j| <= 2^-8 (spread + |O|)."""
    s = Step(seed=31, **kw)
    c = 2.0 ** torch.tensor(exps, dtype=torch.float64)[torch.arange(s.d) % len(exps)]
    for t in (s.vc, s.vs):
        t.copy_((t.double() * c.cuda()).to(t.dtype))
    O, lse, spread = _run(s, block)
    c = c.numpy()
    tol = attn_tol(O / c, spread / c)
    if max(exps) - min(exps) > 20:
        tol = tol + 1.01 * HALF[BF] * (spread + np.abs(O)) / c
    assert np.abs(f64(s.lse)[:s.n] - lse).max() <= 5e-4
    bad = np.abs(f64(s.out)[:s.n] / c - O / c) / tol
    assert bad.max() <= 1.0, (bad.max(), np.unravel_index(bad.argmax(), bad.shape))


@pytest.mark.parametrize("block", [0, 16])
@pytest.mark.parametrize("exp", [-110, -118, -127, -130])
def test_values_near_the_types_smallest(gpu_lib, exp, block):
    """Values down to bf16's subnormal ones: within the bound of their size and float32's smallest
    normal number, never infinite."""
    s = Step(past=[0, 2], new=[1, 1], T=3, seed=32)
    for t in (s.vc, s.vs):
        t.copy_((t.double() * 2.0 ** exp).to(t.dtype))
    O, lse, spread = _run(s, block)
    c = 2.0 ** exp
    err = np.abs(f64(s.out)[:s.n] - O)
    assert np.all(err <= attn_tol(O / c, spread / c) * c + 2.0 ** -126)


def test_largest_values(gpu_lib):
    """Values near bf16's largest, few enough that their unnormalised sum is a float32 number, next
    to ordinary and tiny ones."""
    s = Step(past=[0], new=[1], T=2, seed=33)
    c = 2.0 ** torch.tensor([120.0, 0.0, -100.0], dtype=torch.float64)[torch.arange(s.d) % 3]
    for t in (s.vc, s.vs):
        t.copy_((t.double() * c.cuda()).to(t.dtype))
    O, lse, spread = _run(s, 0)
    c = c.numpy()
    tol = attn_tol(O / c, spread / c) + 1.01 * HALF[BF] * (spread + np.abs(O)) / c
    assert np.all(np.abs(f64(s.out)[:s.n] - O) / c <= tol)


def test_more_rows_than_a_row_per_workgroup_holds(gpu_lib):
    """fresh_rows in place over more than 2^24 rows of 64 heads: rows at both ends and around 2^24
    come out as in a call of their own, the others (zeros) as they were."""
    n, H, d = (1 << 24) + 5, 64, 64
    _needs(150)
    req = relaxkv.Request(torch.zeros(1, 1, H, d, dtype=BF, device="cuda"), *torch.zeros(2, 1, H, 64, d, dtype=BF, device="cuda"), 0.5)
    rope = relaxkv.Rope(torch.linspace(1, 0.01, 32, device="cuda"))
    at = torch.tensor([0, 1, 1 << 23, (1 << 24) - 1, 1 << 24, n - 2, n - 1], device="cuda")
    x, pos = torch.zeros(n, H, d, dtype=BF, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    x[at] = torch.randn(len(at), H, d, device="cuda", generator=torch.Generator("cuda").manual_seed(5)).to(BF)
    pos[at] = at.int() + 3
    few, want = x[at], torch.empty(len(at), H, d, dtype=BF, device="cuda")
    req.fresh_rows(rope, pos[at], None, few, None, None, want, None)
    assert not torch.equal(few, want)
    req.fresh_rows(rope, pos, None, x, None, None, x, None)
    assert torch.equal(x[at], want)
    x[at] = 0
    assert not any(bool(x[i:i + (1 << 20)].any()) for i in range(0, n, 1 << 20))


def test_selection_of_the_largest_step(gpu_lib):
    """block_select with the most rows and heads of a step, and 2049 blocks: against float64 scores of
    some rows."""
    n, H, d, block, sel = 65536, 64, 64, 16, 5
    nb = 2049
    _needs(60)
    g = torch.Generator("cuda").manual_seed(7)
    kc = torch.zeros(1, H, nb * block, d, dtype=BF, device="cuda")
    req = relaxkv.Request(torch.zeros(1, 1, H, d, dtype=BF, device="cuda"), kc, kc, 0.5)
    b = req.alloc_batch(n, n, 1)
    z = torch.zeros(n, dtype=torch.int32, device="cuda")
    req.plan_batch(b, z, z + 1)
    q = torch.randn(n, H, d, device="cuda", generator=g).to(BF)
    means = torch.randn(H, nb, d, device="cuda", generator=g).to(BF)
    lists = torch.full((n, H, sel), -7, dtype=torch.int32, device="cuda")
    ws = torch.empty(req._lib.relaxkv_block_select_workspace_bytes(req._ref, b.ref, block), dtype=torch.uint8,
                     device="cuda")
    req.block_select(b, block, means, q, lists, ws)
    assert not bool((lists == -7).any())
    at = [0, 1, 40000, n - 2, n - 1]
    assert np.array_equal(lists[at].cpu().numpy(), bo.block_select(f64(q[at]), f64(means), sel))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_calls_before_the_first_plan(gpu_lib, dtype):
    """A zeroed batch buffer is a step without rows: every call leaves its outputs as they were."""
    s = Step(past=[5, 1], new=[2, 1], T=200, dtype=dtype)
    s.batch = s.req.alloc_batch(2, 3, s.room)
    k, q_rot = torch.zeros(3, 2, 128, dtype=dtype, device="cuda"), torch.full_like(s.q, 7.0)
    ks, vs = s.ks.clone(), s.vs.clone()
    s.req.batch_rows(relaxkv.Rope(), s.batch, s.q, k, k, q_rot, s.ks, s.vs)
    lists = torch.full((3, 2, 4), -7, dtype=torch.int32, device="cuda")
    means = torch.zeros(2, 4, 128, dtype=dtype, device="cuda")
    s.req.block_select(s.batch, 64, means, s.q, lists, s.req.alloc_block_workspace(s.batch, 64, 4))
    s.shared()
    s.blocks(64, lists)
    assert s.batch.counts_to_host() == [0, 0, 0, 0]
    for t, v in ((q_rot, 7), (s.out, 7), (s.lse, 7), (lists, -7)):
        assert bool((t == v).all())
    assert torch.equal(ks.nan_to_num(9), s.ks.nan_to_num(9)) and torch.equal(vs.nan_to_num(9), s.vs.nan_to_num(9))
