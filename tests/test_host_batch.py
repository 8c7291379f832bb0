"""Host-side checks of the batched serving calls (no GPU): sizes, carving, every refusal.
No call here reaches a kernel: each is refused, or has no rows."""

import ctypes
import types

import numpy as np
import pytest
import torch

import oracle
from oracle import batch_oracle as bo

BASE = 0x7f0000000000                                # never dereferenced


def _problem(rk, **kw):
    b = dict(L=2, T_c=1000, n_query=4, H=8, H_kv=2, d=128, dtype=rk.DTYPE_BF16)
    b.update(kw)
    return rk.Problem(b["L"], b["T_c"], b["n_query"], b["H"], b["H_kv"], b["d"], b["dtype"], 0.0,
                      0.15, 0x1000, 0x2000, 0x3000, None, 0, 0, 0)


def _batch(rk, p, n_seq=3, n_rows=10, max_suffix=50):
    s = rk.CBatch()
    lib = rk.load()
    n = lib.relaxkv_batch_bytes(ctypes.byref(p), n_seq, n_rows, max_suffix)
    assert n > 0 and n % 256 == 0
    assert lib.relaxkv_batch_bind(ctypes.byref(p), n_seq, n_rows, max_suffix, BASE, n,
                                  ctypes.byref(s)) == 0
    return s


@pytest.mark.parametrize("n_seq,n_rows,max_suffix,ok", [
    (1, 0, 1, True), (1, 1, 1, True), (65536, 65536, 1 << 22, True), (0, 1, 1, False),
    (65537, 1, 1, False), (1, -1, 1, False), (1, 65537, 1, False), (1, 1, 0, False),
    (1, 1, (1 << 22) + 1, False)])
def test_batch_sizes(rk, n_seq, n_rows, max_suffix, ok):
    lib, p = rk.load(), _problem(rk)
    n = lib.relaxkv_batch_bytes(ctypes.byref(p), n_seq, n_rows, max_suffix)
    assert (n > 0) == ok
    s = rk.CBatch()
    st = lib.relaxkv_batch_bind(ctypes.byref(p), n_seq, n_rows, max_suffix, BASE, n or 1 << 40,
                                ctypes.byref(s))
    assert st == (0 if ok else rk.EINVAL)


def test_batch_rows_times_heads(rk):
    lib = rk.load()
    for H, rows, ok in ((64, 65536, True), (128, 65536, False), (128, 32768, True)):
        p = _problem(rk, H=H, H_kv=8)
        assert (lib.relaxkv_batch_bytes(ctypes.byref(p), 4, rows, 8) > 0) == ok


@pytest.mark.parametrize("dtype,tile", [(1, 128), (0, 16)])
def test_batch_bind_carves(rk, dtype, tile):
    p = _problem(rk, dtype=dtype)
    s = _batch(rk, p, 700, 900, 33)
    assert (s.n_seq, s.n_rows, s.max_suffix) == (700, 900, 33)
    assert (s.T_c, s.H, s.H_kv, s.d, s.dtype) == (1000, 8, 2, 128, dtype)
    assert s.tile_cap == 900 * 4 // tile + 700
    lib = rk.load()
    n = lib.relaxkv_batch_bytes(ctypes.byref(p), 700, 900, 33)
    at = sorted([(s.counts, 256), (s.row_off, 4 * 701), (s.row_seq, 3600), (s.row_pos, 3600),
                 (s.tiles, 32 * s.tile_cap)])
    for (a, size), (b, _) in zip(at, at[1:] + [(BASE + n, 0)]):
        assert a % 256 == 0 and a >= BASE and b - a >= size
    for buf, size, want in ((BASE, n - 1, rk.ENOSPACE), (BASE + 16, n, rk.EINVAL), (None, n, rk.EINVAL)):
        assert lib.relaxkv_batch_bind(ctypes.byref(p), 700, 900, 33, buf, size, ctypes.byref(s)) == want


def test_tile_cap_bounds_every_step(rk):
    """The tiles of any step of n_rows rows and n_seq requests fit the carved ones."""
    rng = np.random.default_rng(1)
    for dtype, tile in ((1, 128), (0, 16)):
        for H, H_kv in ((8, 2), (7, 1), (40, 8), (384, 1)):
            p = _problem(rk, dtype=dtype, H=H, H_kv=H_kv)
            for _ in range(50):
                n_seq, n_rows = int(rng.integers(1, 40)), int(rng.integers(1, 200))
                s = _batch(rk, p, n_seq, n_rows, 1000)
                cut = np.sort(rng.integers(0, n_rows + 1, n_seq - 1))
                new = np.diff(np.concatenate([[0], cut, [n_rows]]))
                assert sum(-(-int(n) * (H // H_kv) // tile) for n in new) <= s.tile_cap


def _args(rk, prob, bat, /, **kw):
    """Good arguments of every call, by name; kw replaces some."""
    a = dict(p=ctypes.byref(prob), b=ctypes.byref(bat), layer=0, kc=0x2000, vc=0x3000, q=0x4000,
             suf=rk.CSuffix(0x5000, 0x6000, 0, 0, 0), out=0x7000, lse=None, ws=0x8000,
             wsb=1 << 40, block=64, blocks=0x9000, sel=4, means=0xa000,
             rope=rk.CRope(0xb000, None, None, 1e-6, 64, 0),
             rows=rk.CRows(0x4000, 0x4000, 0x4000, 0, 0, 0, bat.n_rows), past=0xc000, new=0xd000,
             pos=0xe000, qo=0xf000, ko=0xf000, vo=0xf000)
    a.update(kw)
    for k in ("suf", "rope", "rows"):
        if a[k] is not None:
            a[k] = ctypes.byref(a[k])
    return a


def _call(rk, name, a):
    lib = rk.load()
    f = getattr(lib, "relaxkv_" + name)
    names = {"batch_plan": "p b past new", "batch_rows": "p rope b rows qo suf",
             "fresh_rows": "p rope rows pos qo ko vo", "block_means": "p layer kc block means",
             "shared_attn": "p b layer kc vc q suf out lse ws wsb",
             "block_select": "p b block means q sel blocks ws wsb",
             "block_attn": "p b layer kc vc block blocks sel q suf out lse ws wsb"}[name]
    return f(*(a[n] for n in names.split()), None)


EINVAL, ENOSPACE, EUNSUPPORTED = -1, -2, -3
ATTN = ["shared_attn", "block_attn"]
REFUSED = [
    (ATTN, dict(layer=-1), EINVAL), (ATTN, dict(layer=2), EINVAL), (ATTN, dict(kc=None), EINVAL),
    (ATTN, dict(vc=None), EINVAL), (ATTN, dict(q=None), EINVAL), (ATTN, dict(out=None), EINVAL),
    (ATTN, dict(ws=None), EINVAL), (ATTN, dict(wsb=16), ENOSPACE), (ATTN, dict(suf=None), EINVAL),
    (ATTN, dict(kc=0x2008), EUNSUPPORTED), (ATTN, dict(out=0x7004), EUNSUPPORTED),
    (ATTN, dict(q=0x4002), EUNSUPPORTED), (ATTN, dict(ws=0x8008), EUNSUPPORTED),
    (["batch_plan"], dict(past=None), EINVAL), (["batch_plan"], dict(new=None), EINVAL),
    (["batch_plan", "shared_attn", "block_select"], dict(b=None), EINVAL),
    (["batch_plan", "batch_rows", "fresh_rows", "block_means"], dict(p=None), EINVAL),
    (["block_attn"], dict(blocks=None), EINVAL), (["block_attn", "block_select"], dict(sel=0), EINVAL),
    (["block_attn", "block_select"], dict(sel=17), EINVAL),
    (["block_attn", "block_select", "block_means"], dict(block=48), EINVAL),
    (["block_attn", "block_select", "block_means"], dict(block=8), EINVAL),
    (["block_means"], dict(layer=-2), EINVAL), (["block_means"], dict(layer=2), EINVAL),
    (["block_means"], dict(kc=None), EINVAL), (["block_means", "block_select"], dict(means=None), EINVAL),
    (["block_means", "block_select"], dict(means=0xa004), EUNSUPPORTED),
    (["block_select"], dict(ws=None), EINVAL), (["block_select"], dict(wsb=100), ENOSPACE),
    (["block_select"], dict(q=None), EINVAL), (["block_select"], dict(blocks=None), EINVAL),
    (["fresh_rows"], dict(pos=None), EINVAL), (["fresh_rows"], dict(qo=None), EINVAL),
    (["fresh_rows"], dict(ko=None), EINVAL), (["fresh_rows"], dict(vo=0xf008), EUNSUPPORTED),
    (["batch_rows"], dict(qo=None), EINVAL), (["batch_rows"], dict(suf=None), EINVAL),
    (["fresh_rows", "batch_rows"], dict(rope=None), EINVAL),
    (["fresh_rows", "batch_rows"], dict(rows=None), EINVAL),
]


@pytest.mark.parametrize("names,kw,status", REFUSED)
def test_refusals(rk, names, kw, status):
    p = _problem(rk)
    b = _batch(rk, p)
    for name in names:
        assert _call(rk, name, _args(rk, p, b, **kw)) == status, name


@pytest.mark.parametrize("f,status", [
    ((0xb000, None, None, 1e-6, 24, 0), EUNSUPPORTED), ((0xb000, None, None, 1e-6, 144, 0), EINVAL),
    ((0xb000, None, None, 1e-6, -16, 0), EINVAL), ((None, None, None, 1e-6, 16, 0), EINVAL),
    ((0xb000, None, None, -1.0, 16, 0), EINVAL), ((0xb000, None, None, float("nan"), 16, 0), EINVAL),
    ((0xb000, None, None, float("inf"), 16, 0), EINVAL), ((0xb000, None, None, 1e-6, 16, 2), EINVAL)])
def test_rope_refusals(rk, f, status):
    p = _problem(rk)
    b = _batch(rk, p)
    for name in ("fresh_rows", "batch_rows"):
        assert _call(rk, name, _args(rk, p, b, rope=rk.CRope(*f))) == status


@pytest.mark.parametrize("r,status", [
    ((0x4000, None, None, 1016, 0, 0, 10), EINVAL), ((0x4000, None, None, 1028, 0, 0, 10), EUNSUPPORTED),
    ((0x4004, None, None, 0, 0, 0, 10), EUNSUPPORTED), ((0x4000, None, None, -1024, 0, 0, 10), EINVAL),
    ((0x4000, None, None, 0, 0, 0, -1), EINVAL), ((0x4000, None, None, 1 << 41, 0, 0, 10), EUNSUPPORTED)])
def test_row_refusals(rk, r, status):
    p = _problem(rk)
    b = _batch(rk, p)
    for name in ("fresh_rows", "batch_rows"):
        a = _args(rk, p, b, rows=rk.CRows(*r), ko=None, vo=None)
        assert _call(rk, name, a) == status
    assert _call(rk, "batch_rows", _args(rk, p, b, rows=rk.CRows(0x4000, None, None, 0, 0, 0, 9))) == EINVAL


@pytest.mark.parametrize("s,status", [
    ((0x5000, None, 0, 0, 0), EINVAL), ((0x5004, 0x6000, 0, 0, 0), EUNSUPPORTED),
    ((0x5000, 0x6000, 0, 0, 64), EINVAL),                       # rows overlap
    ((0x5000, 0x6000, 0, 49 * 128, 128), EINVAL),               # heads overlap
    ((0x5000, 0x6000, 128, 0, 0), EINVAL),                      # requests overlap
    ((0x5000, 0x6000, -1, 0, 0), EINVAL), ((0x5000, 0x6000, 0, 0, 132), EUNSUPPORTED),
    ((0x5000, 0x6000, 0, 0, 1 << 24), EUNSUPPORTED), ((0x5000, 0x6000, 1 << 48, 0, 0), EUNSUPPORTED),
    ((0x5000, 0x6000, 0, 1 << 62, 0), EUNSUPPORTED)])
def test_suffix_refusals(rk, s, status):
    p = _problem(rk)
    b = _batch(rk, p)
    for name in ("batch_rows", "shared_attn", "block_attn"):
        assert _call(rk, name, _args(rk, p, b, suf=rk.CSuffix(*s))) == status


@pytest.mark.parametrize("field,value", [("T_c", 999), ("H", 16), ("H_kv", 4), ("d", 64),
                                         ("dtype", 0), ("tile_cap", 99), ("n_rows", -1),
                                         ("n_seq", 0), ("max_suffix", 0), ("row_seq", None),
                                         ("tiles", BASE + 4), ("counts", None)])
def test_batch_of_another_shape(rk, field, value):
    p = _problem(rk)
    for name in ("batch_plan", "batch_rows", "shared_attn", "block_select", "block_attn"):
        b = _batch(rk, p)
        setattr(b, field, value)
        assert _call(rk, name, _args(rk, p, b)) == rk.EINVAL, name
    lib = rk.load()
    assert lib.relaxkv_shared_attn_workspace_bytes(ctypes.byref(p), ctypes.byref(b)) == 0


def test_no_rows_is_no_work(rk):
    p = _problem(rk)
    b = _batch(rk, p, n_rows=0)
    for name in ("batch_rows", "shared_attn", "block_select", "block_attn"):
        a = _args(rk, p, b, q=None, out=None, blocks=None, ws=None, wsb=0,
                  rows=rk.CRows(None, None, None, 0, 0, 0, 0), qo=None)
        assert _call(rk, name, a) == 0, name
    assert _call(rk, "fresh_rows", _args(rk, p, b, pos=None)) == 0


def test_workspace_sizes(rk):
    """Partial rows of d fp16 values and 16 bytes: 128 for each of the 768 workgroups and of
    the (row chunk, KV head) pairs, and as many suffix rows as there are rows, 768 * 128 at
    least; listed blocks the latter twice."""
    lib = rk.load()
    al = lambda x: (x + 255) // 256 * 256                     # noqa: E731
    p = _problem(rk, T_c=32768, H=40, H_kv=8)
    for n_rows in (1, 64, 4000):
        b = _batch(rk, p, 64, n_rows, 600)
        rows = max(768 * 128, n_rows * 40)
        chunks = -(-n_rows * 5 // 128)
        for ctx, got in (((768 + chunks * 8) * 128, lib.relaxkv_shared_attn_workspace_bytes(
                              ctypes.byref(p), ctypes.byref(b))),
                         (rows, lib.relaxkv_block_attn_workspace_bytes(
                              ctypes.byref(p), ctypes.byref(b), 64, 9))):
            assert got == al((ctx + rows) * 256) + al((ctx + rows) * 16)
    b = _batch(rk, p, 64, 64, 600)
    assert lib.relaxkv_block_select_workspace_bytes(ctypes.byref(p), ctypes.byref(b), 64) == \
        al(64 * 8 * 512 * 4)
    assert lib.relaxkv_block_select_workspace_bytes(ctypes.byref(p), ctypes.byref(b), 40) == 0
    assert lib.relaxkv_block_attn_workspace_bytes(ctypes.byref(p), ctypes.byref(b), 64, 513) == 0
    assert lib.relaxkv_block_attn_workspace_bytes(ctypes.byref(p), ctypes.byref(b), 64, 512) > 0
    # float32: workgroups of 16 rows, d values and a log-sum-exp each: listed 512; shared context
    # 256 and three times 512, or the rows if more, and twice
    p = _problem(rk, dtype=0)
    for n_rows in (1, 3000):
        b = _batch(rk, p, n_rows=n_rows)
        assert lib.relaxkv_shared_attn_workspace_bytes(ctypes.byref(p), ctypes.byref(b)) == \
            2 * max((256 + 3 * 512) * 16, n_rows * 8) * (128 * 4 + 4)
        assert lib.relaxkv_block_attn_workspace_bytes(ctypes.byref(p), ctypes.byref(b), 64, 3) == \
            512 * 16 * (128 * 4 + 4)
    b = _batch(rk, p, n_rows=0)
    assert lib.relaxkv_shared_attn_workspace_bytes(ctypes.byref(p), ctypes.byref(b)) == 0


def test_too_many_selected_blocks(rk):
    p = _problem(rk, T_c=1 << 16)
    b = _batch(rk, p)
    a = _args(rk, p, b, block=16, sel=rk.MAX_SELECTED_BLOCKS + 1)
    assert _call(rk, "block_select", a) == rk.EUNSUPPORTED
    assert _call(rk, "block_attn", a) == rk.EUNSUPPORTED


def test_rope_object_refusals(rk):
    for f in (torch.zeros(4, dtype=torch.float64), torch.zeros(4, 2), torch.zeros(8)[::2], [1.0]):
        with pytest.raises(ValueError):
            rk.Rope(f)
    with pytest.raises(ValueError):
        rk.Rope(torch.zeros(8), q_weight=[1.0])


def test_expanded_tensors_are_refused(rk):
    """A stride of 0 selects the dense layout in the descriptors."""
    for dim in range(3):
        shape = [2, 3, 4, 64]
        t = torch.zeros(shape)
        assert rk._cache_strides(t) == (768, 256, 64)
        with pytest.raises(ValueError):
            rk._cache_strides(t.narrow(dim, 0, 1).expand(shape))
    assert rk._cache_strides(torch.zeros(1, 3, 1, 64)) == (0, 64, 0)
    req = types.SimpleNamespace(dtype=torch.float32, device=torch.device("cpu"), _index=-1, d=64)
    rows = lambda t, n: rk.Request._projected(req, t, "q", 4, n)        # noqa: E731
    fused = torch.zeros(5, 12, 64)
    assert rows(fused[:, 4:8], 5) == 768 and rows(fused[:1, 4:8], 1) == 0 and rows(None, 5) == 0
    with pytest.raises(ValueError):
        rows(fused[:1, :4].expand(5, 4, 64), 5)
    assert rows(fused[:1, :4].expand(1, 4, 64), 1) == 0


def test_too_many_fresh_rows(rk):
    p = _problem(rk)
    b = _batch(rk, p)
    a = _args(rk, p, b, rows=rk.CRows(0x4000, None, None, 0, 0, 0, (1 << 25) + 1), ko=None, vo=None)
    assert _call(rk, "fresh_rows", a) == EUNSUPPORTED


# ------------------------------------------------------------------ pins of the oracle

def test_oracle_one_request_is_the_query_side():
    """One request with no past is the query-side completion's oracle."""
    r = np.random.default_rng(2)
    q, kc, vc = r.normal(size=(5, 4, 16)), r.normal(size=(2, 30, 16)), r.normal(size=(2, 30, 16))
    kq, vq = r.normal(size=(5, 2, 16)), r.normal(size=(5, 2, 16))
    off, seq, pos = bo.batch_plan([0], [5], 30)
    O, lse, _ = bo.batch_attn(q, seq, pos, kc, vc, kq.transpose(1, 0, 2)[None], vq.transpose(1, 0, 2)[None])
    O_ref, lse_ref = oracle.query_attn(q, kc, vc, kq, vq)
    assert np.allclose(O, O_ref, atol=1e-12) and np.allclose(lse, lse_ref, atol=1e-12)
    nb = -(-30 // 16)
    blocks = np.broadcast_to(np.arange(nb), (5, 2, nb))
    Ob, lseb, _ = bo.batch_attn(q, seq, pos, kc, vc, kq.transpose(1, 0, 2)[None],
                                vq.transpose(1, 0, 2)[None], blocks=blocks, block=16)
    assert np.allclose(Ob, O, atol=1e-12) and np.allclose(lseb, lse, atol=1e-12)


@pytest.mark.parametrize("inter", [False, True])
def test_oracle_rotation_identities(inter):
    """Rotated products depend on the distance alone; a rotation and its inverse cancel; a
    quarter turn maps (a, b) to (-b, a)."""
    r = np.random.default_rng(3)
    f = 0.3 ** np.arange(4)
    q, k = r.normal(size=(1, 1, 10)), r.normal(size=(1, 1, 10))
    dot = lambda i, j: float((bo.norm_rope(q, [i], f, interleaved=inter)          # noqa: E731
                              * bo.norm_rope(k, [j], f, interleaved=inter)).sum())
    assert np.isclose(dot(7, 3), dot(104, 100)) and not np.isclose(dot(7, 3), dot(7, 4))
    assert np.allclose(bo.norm_rope(bo.norm_rope(q, [9], f), [-9], f), q)
    x = np.arange(2.0).reshape(1, 1, 2) + 1
    assert np.allclose(bo.norm_rope(x, [1], [np.pi / 2], interleaved=inter), [[[-2.0, 1.0]]])
    y = bo.norm_rope(q, [0], None, weight=np.full(10, 2.0), eps=0.0)
    assert np.isclose((y ** 2).mean(), 4.0)


def test_oracle_plan_select_and_rounding():
    off, seq, pos = bo.batch_plan([3, 0, 5], [2, 0, 1], 10)
    assert off.tolist() == [0, 2, 2, 3] and seq.tolist() == [0, 0, 2] and pos.tolist() == [13, 14, 15]
    means = np.array([[[1.0], [3.0], [3.0], [np.nan], [2.0]]])
    assert bo.block_select(np.ones((1, 2, 1)), means, 2).tolist() == [[[1, 2]]]
    assert bo.block_select(np.ones((1, 2, 1)), means, 5).tolist() == [[[0, 1, 2, 3, 4]]]
    assert bo.block_means(np.arange(5.0).reshape(1, 5, 1), 2)[0, :, 0].tolist() == [0.5, 2.5, 4.0]
    assert bo.round_bf16([1 + 2.0 ** -8, 1 + 2.0 ** -8 + 2.0 ** -40, -3.0, 0.0]).tolist() == \
        [1.0, 1 + 2.0 ** -7, -3.0, 0.0]
