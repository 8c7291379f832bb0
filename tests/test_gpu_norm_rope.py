"""Norm and rotation of projected rows against the float64 oracle: both pairings, partial
rotations, far and negative positions, slices of a fused projection, in place; and a batch's
rows into its suffix caches."""

import numpy as np
import pytest
import torch

from batch_harness import HALF, Step, f64
from oracle import batch_oracle as bo
from paper_2609_33503_amd import relaxkv

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def close(got, ref, dtype, what):
    """Half a step of the output type, and 2^-20 of the head's largest value: the float32
    operations before it (norm, two products, a sum, sine and cosine within 2^-24) are each off by
    at most 2^-23 of a value no larger than that, fewer than eight of them in a row."""
    ref = np.asarray(ref)
    tol = HALF[dtype] * np.abs(ref) + 2.0 ** -20 * np.abs(ref).max(-1, keepdims=True) + 1e-30
    err = np.abs(f64(got) - ref) / tol
    assert err.max(initial=0.0) <= 1.0, f"{what}: {err.max():.2f} of the bound"


def request(H, H_kv, d, dtype, T=64):
    z = torch.zeros(1, H_kv, T, d, dtype=dtype, device="cuda")
    return relaxkv.Request(torch.zeros(1, 1, H, d, dtype=dtype, device="cuda"), z, z, 0.2)


def rope(d, rot, dtype, norm, inter, theta=1e4, seed=1, eps=1e-6):
    g = torch.Generator().manual_seed(seed)
    f = theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(dtype).cuda() for _ in range(2)]
    return relaxkv.Rope(f.float().cuda() if rot else None, w[0] if norm else None,
                        w[1] if norm else None, eps, inter)


def oracle_rows(x, pos, r, w, inter):
    return bo.norm_rope(f64(x), pos, None if r.inv_freq is None else f64(r.inv_freq),
                        None if w is None else f64(w), r_eps(r), inter)


def r_eps(r):
    return float(np.float32(r.s.eps))


CASES = [
    # n, H, H_kv, d, rot, norm, interleaved, fused
    (1, 1, 1, 64, 64, True, False, False), (1, 40, 8, 128, 128, True, False, True),
    (7, 8, 2, 128, 128, True, True, True), (33, 12, 3, 128, 32, False, False, False),
    (33, 12, 3, 64, 16, True, True, True), (300, 14, 2, 128, 96, True, False, True),
    (5, 4, 4, 64, 48, False, True, False), (9, 8, 8, 128, 0, True, False, False),
    (3, 8, 8, 64, 0, False, False, True), (1027, 4, 1, 64, 64, True, False, True),
    (1500, 3, 1, 128, 64, True, True, False),
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,H,H_kv,d,rot,norm,inter,fused", CASES)
def test_fresh_rows(gpu_lib, n, H, H_kv, d, rot, norm, inter, fused, dtype):
    g = torch.Generator().manual_seed(n + rot)
    x = torch.randn(n, (H + 2 * H_kv) * d + (16 if fused else 0), generator=g).to(dtype).cuda()
    parts = [t.view(n, -1, d) if not fused else t.unflatten(1, (-1, d))
             for t in x[:, :(H + 2 * H_kv) * d].split([H * d, H_kv * d, H_kv * d], 1)]
    if not fused:
        parts = [t.contiguous() for t in parts]
    pos = torch.randint(-(1 << 22), 1 << 22, (n,), generator=g)
    req, r = request(H, H_kv, d, dtype), rope(d, rot, dtype, norm, inter)
    outs = [torch.full((n, h, d), 7.0, dtype=dtype, device="cuda") for h in (H, H_kv, H_kv)]
    req.fresh_rows(r, pos.int().cuda(), *parts, *outs)
    close(outs[0], oracle_rows(parts[0], pos, r, r.q_weight, inter), dtype, "q")
    close(outs[1], oracle_rows(parts[1], pos, r, r.k_weight, inter), dtype, "k")
    assert torch.equal(outs[2], parts[2])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_parts_and_in_place(gpu_lib, dtype):
    """Any of the three may be left out; a dense input may be its own output."""
    n, H, H_kv, d = 50, 6, 2, 128
    g = torch.Generator().manual_seed(9)
    q, k = (torch.randn(n, h, d, generator=g).to(dtype).cuda() for h in (H, H_kv))
    pos = torch.arange(n, dtype=torch.int32).cuda()
    req, r = request(H, H_kv, d, dtype), rope(d, 128, dtype, True, False)
    q2, k2 = torch.empty_like(q), torch.empty_like(k)
    req.fresh_rows(r, pos, q, k, None, q2, k2, None)
    only = torch.empty_like(k)
    req.fresh_rows(r, pos, None, k, None, None, only, None)
    assert torch.equal(only, k2)
    req.fresh_rows(r, pos, q, None, None, q, None, None)
    assert torch.equal(q, q2)
    req.fresh_rows(r, pos, None, None, k, None, None, only)
    assert torch.equal(only, k)
    req.fresh_rows(r, pos[:0], q[:0], k[:0], None, q2[:0], k2[:0], None)


def test_small_and_large_values(gpu_lib):
    """Rows of zeros (eps alone under the root), of tiny values, and of values whose mean
    square is large."""
    n, d = 4, 64
    x = torch.zeros(n, 1, d)
    x[1], x[2], x[3] = 1e-20, 3e15, torch.linspace(-5, 5, d)
    x = x.cuda()
    req, r = request(1, 1, d, F32), rope(d, 64, F32, True, False, eps=1e-5)
    out = torch.empty_like(x)
    pos = torch.tensor([0, 1, 2, 3], dtype=torch.int32).cuda()
    req.fresh_rows(r, pos, x, None, None, out, None, None)
    close(out, oracle_rows(x, pos.cpu(), r, r.q_weight, False), F32, "values")
    assert torch.all(out[0] == 0)


@pytest.mark.parametrize("layout", ["bhsd", "bshd", "hbsd"])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_batch_rows(gpu_lib, dtype, layout):
    """Queries to dense rows, keys and values to their suffix tokens; every other suffix
    token and the rows behind the last stay as they were."""
    s = Step(past=[0, 12, 5, 7], new=[3, 1, 0, 9], T=100, H=10, H_kv=2, dtype=dtype, extra_rows=4,
             layout=layout)
    n, N, d = s.n, s.q.shape[0], s.d
    g = torch.Generator().manual_seed(3)
    x = torch.randn(N, 14 * d, generator=g).to(dtype).cuda()
    x[n:] = float("nan")
    q, k, v = (t.unflatten(1, (-1, d)) for t in x.split([10 * d, 2 * d, 2 * d], 1))
    r = rope(d, 128, dtype, True, False, theta=1e6)
    ks0, vs0 = s.ks.clone(), s.vs.clone()
    out = torch.full((N, 10, d), 7.0, dtype=dtype, device="cuda")
    s.req.batch_rows(r, s.batch, q, k, v, out, s.ks, s.vs)
    close(out[:n], oracle_rows(q[:n], s.pos, r, r.q_weight, False), dtype, "q")
    assert torch.all(out[n:] == 7.0)
    kr = oracle_rows(k[:n], s.pos, r, r.k_weight, False)
    for i in range(n):
        b, t = int(s.seq[i]), int(s.pos[i]) - s.T
        close(s.ks[b, :, t], kr[i], dtype, f"k row {i}")
        assert torch.equal(s.vs[b, :, t], v[i])
        s.ks[b, :, t], s.vs[b, :, t] = ks0[b, :, t], vs0[b, :, t]
    for a, b in ((s.ks, ks0), (s.vs, vs0)):
        assert torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0))


def test_binding_refusals(gpu_lib):
    n, H, H_kv, d = 4, 4, 2, 64
    req, r = request(H, H_kv, d, BF), rope(d, 64, BF, True, False)
    q, k = (torch.zeros(n, h, d, dtype=BF, device="cuda") for h in (H, H_kv))
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    good = dict(rope=r, positions=pos, q=q, k=k, v=k, q_out=q.clone(), k_out=k.clone(), v_out=k.clone())
    req.fresh_rows(**good)
    for bad in (dict(positions=pos.long()), dict(positions=pos[:3]), dict(positions=pos.cpu()),
                dict(q=q.float()), dict(q=q.transpose(0, 1)), dict(q=q[:, :, ::2]), dict(q_out=None),
                dict(k=None), dict(k_out=k[:, :1]), dict(rope=None),
                dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)),
                dict(rope=rope(d, 64, F32, True, False)), dict(rope=rope(128, 64, BF, True, False))):
        with pytest.raises(ValueError):
            req.fresh_rows(**{**good, **bad})
    for rot in (8, 24, 80):
        with pytest.raises(relaxkv.RelaxKVError):
            req.fresh_rows(**{**good, "rope": rope(d, rot, BF, True, False)})
    torch.cuda.synchronize()


def test_expanded_rows_are_refused(gpu_lib):
    """One row repeated by a stride of 0, which in the descriptor selects dense rows."""
    req, r = request(4, 2, 64, BF), rope(64, 64, BF, True, False)
    q = torch.zeros(1, 4, 64, dtype=BF, device="cuda").expand(5, 4, 64)
    pos = torch.zeros(5, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        req.fresh_rows(r, pos, q, None, None, torch.zeros(5, 4, 64, dtype=BF, device="cuda"), None, None)
    one = torch.ones(1, 4, 64, dtype=BF, device="cuda")
    req.fresh_rows(r, pos[:1], one.expand(1, 4, 64), None, None, one, None, None)
    torch.cuda.synchronize()
