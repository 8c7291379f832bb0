"""Attention of a batch over a shared context and own suffixes, and over listed blocks,
against the float64 oracle: lengths from one token, ragged splits and tiles, strides, heads,
rows and cache entries that must be neither read nor written (NaN), refusals."""

import numpy as np
import pytest
import torch

from batch_harness import Step, attn_tol, f64
from paper_2609_33503_amd import relaxkv

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

SHARED = {
    "one": dict(past=[0], new=[1], T=1, H=1, H_kv=1, d=64),
    "one-128": dict(past=[0], new=[1], T=1),
    "decode": dict(past=[0, 5, 63, 64, 200], new=[1, 1, 1, 1, 1], T=700),
    "paused": dict(past=[4, 0, 9], new=[1, 0, 2], T=333, extra_rows=3),
    "mixed": dict(past=[0, 31, 100, 0], new=[70, 1, 33, 5], T=515, H=10, H_kv=2, spare=9),
    "wide-group": dict(past=[3, 7], new=[2, 3], T=130, H=48, H_kv=1, d=64),
    "group-200": dict(past=[3], new=[2], T=100, H=200, H_kv=1, d=64),
    "mha": dict(past=[70, 2], new=[1, 9], T=257, H=3, H_kv=3),
    "token-major": dict(past=[10, 20, 64], new=[3, 1, 1], T=300, layout="bshd", extra_rows=1),
    "head-major": dict(past=[10, 20], new=[1, 1], T=300, layout="hbsd"),
    "suffix-splits": dict(past=[900, 255, 256, 0], new=[1, 1, 1, 4], T=64),
    "long-room": dict(past=[1, 0], new=[1, 40], T=90, room=5000),
    "chunks": dict(past=[0] * 40, new=[2] * 40, T=300, H=14, H_kv=2),
    "scale": dict(past=[4, 8], new=[2, 2], T=150, scale=0.5),
    "sharp": dict(past=[40, 8], new=[2, 30], T=400, sharp=12.0),
}


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("name", list(SHARED))
def test_shared(gpu_lib, name, dtype):
    s = Step(dtype=dtype, **SHARED[name])
    s.shared()
    torch.cuda.synchronize()
    s.check(s.reference(), name)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,H,H_kv,d,past,new", [
    (20011, 4, 1, 64, [17], [1]),             # few rows over a long context: many key splits
    (9000, 3, 3, 128, [400], [2]),            # the last split ends in the suffix, causally
    (2560, 8, 8, 64, [256 * 3 - 1, 5], [2, 1]),   # a row that sees nothing of the last split
    (5000, 16, 2, 128, [3] * 30, [1] * 30),   # two chunks of rows, several splits each
    (700, 16, 2, 128, [0] * 90, [3] * 90),    # chunks cut anywhere
    (96, 32, 8, 64, [0, 1], [400, 300]),      # many chunks over a short context
])
def test_shared_splits(gpu_lib, T, H, H_kv, d, past, new, dtype):
    if dtype == F32 and sum(new) > 100:
        new = [max(1, n // 5) for n in new]
    s = Step(past=past, new=new, T=T, H=H, H_kv=H_kv, d=d, dtype=dtype, seed=3)
    s.shared()
    s.check(s.reference())


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_room_does_not_change_the_bits(gpu_lib, dtype):
    """The same step in a batch with room for many more rows, requests and tokens."""
    a, b = (Step(past=[40, 3, 60], new=[1, 20, 1], T=900, dtype=dtype, seed=8, extra_rows=e, room=r)
            for e, r in ((0, 70), (900, 3000)))
    for s in (a, b):
        s.ks[:, :, 63:], s.vs[:, :, 63:] = 0, 0
    b.ks[:, :, :63], b.vs[:, :, :63] = a.ks[:, :, :63], a.vs[:, :, :63]
    b.kc.copy_(a.kc), b.vc.copy_(a.vc), b.q[:22].copy_(a.q)
    for s in (a, b):
        s.shared()
    assert torch.equal(a.out, b.out[:22]) and torch.equal(a.lse, b.lse[:22])
    lists = torch.arange(9, dtype=torch.int32, device="cuda").expand(922, 2, 9).contiguous()
    a.blocks(64, lists[:22])
    b.blocks(64, lists)
    assert torch.equal(a.out, b.out[:22]) and torch.equal(a.lse, b.lse[:22])


def test_shared_one_key_is_exact(gpu_lib):
    """A row's output over one visible key per part is between its values; with equal values it
    is that value exactly."""
    s = Step(past=[0, 0], new=[1, 1], T=130, seed=4)
    s.vc.copy_(s.vc[:, :, :1].expand_as(s.vc))
    s.vs.copy_(s.vc[:, :, :1].expand(1, 2, 1, 128).expand_as(s.vs))
    s.shared()
    want = s.vc[0, :, 0].repeat_interleave(4, 0)
    assert torch.equal(s.out[0], want) and torch.equal(s.out[1], want)


def _lists(rng, n, H_kv, nb, m, junk=True):
    """Distinct blocks in any order, some entries no block, now and then one twice."""
    out = np.full((n, H_kv, m), -1, dtype=np.int32)
    for t in range(n):
        for g in range(H_kv):
            k = int(rng.integers(0, min(m, nb) + 1))
            out[t, g, :k] = rng.permutation(nb)[:k]
            if junk and m > k:
                out[t, g, k:] = rng.choice([-1, nb, 1 << 30, -(1 << 31)], m - k)
            if junk and k > 1 and rng.random() < 0.3:
                out[t, g, 0] = out[t, g, 1]
            rng.shuffle(out[t, g])
    return out


BLOCKS = {
    "one": (dict(past=[0], new=[1], T=1, H=1, H_kv=1, d=64), 16, 1),
    "decode": (dict(past=[0, 5, 63, 200], new=[1, 1, 1, 1], T=1000), 64, 9),
    "tail": (dict(past=[3, 1], new=[2, 1], T=64 * 5 + 7, extra_rows=2, spare=57), 64, 6),
    "small-blocks": (dict(past=[3, 90], new=[5, 1], T=771, H=24, H_kv=2, d=64), 16, 30),
    "block-128": (dict(past=[0, 0], new=[1, 40], T=900, H=10, H_kv=2), 128, 5),
    "splits": (dict(past=[9], new=[1], T=9000, H=2, H_kv=1), 32, 200),
    "group-200": (dict(past=[3], new=[2], T=100, H=200, H_kv=1, d=64), 16, 7),
    "many": (dict(past=[1], new=[1], T=2048 * 16 + 5, H=2, H_kv=1, d=64), 16, 2048),
}


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("name", list(BLOCKS))
def test_blocks(gpu_lib, name, dtype):
    kw, block, m = BLOCKS[name]
    s = Step(dtype=dtype, **kw)
    nb = -(-s.T // block)
    lists = _lists(np.random.default_rng(5), s.q.shape[0], s.H_kv, nb, min(m, nb))
    lists = torch.from_numpy(lists).cuda()
    s.blocks(block, lists)
    torch.cuda.synchronize()
    s.check(s.reference(lists, block), name)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_blocks_empty_lists(gpu_lib, dtype):
    """No listed block at all: the row sees its own suffix alone, whatever the cache holds."""
    s = Step(past=[0, 70], new=[1, 2], T=200, dtype=dtype)
    s.kc.fill_(float("nan"))
    s.vc.fill_(float("nan"))
    lists = torch.full((3, 2, 4), -1, dtype=torch.int32, device="cuda")
    s.blocks(64, lists)
    s.check(s.reference(lists, 64))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_all_blocks_is_the_whole_context(gpu_lib, dtype):
    s = Step(past=[5, 30], new=[2, 3], T=777, dtype=dtype)
    lists = torch.arange(13, dtype=torch.int32, device="cuda").expand(5, 2, 13).contiguous()
    s.blocks(64, lists)
    s.check(s.reference())


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_unlisted_blocks_and_other_requests_do_not_reach(gpu_lib, dtype):
    """NaN and Inf in blocks that no row lists, and in the suffix of a request, reach no row of
    another request that does not see them."""
    s = Step(past=[20, 40, 9], new=[1, 1, 1], T=640, dtype=dtype)
    lists = torch.tensor([1, 4, 7], dtype=torch.int32, device="cuda").expand(3, 2, 3).contiguous()
    ref = s.reference(lists, 64)
    for i in (0, 2, 3, 5, 6, 8, 9):
        s.vc[:, :, i * 64:(i + 1) * 64] = float("inf")
        s.kc[:, :, i * 64:(i + 1) * 64] = float("nan")
    s.vs[1] = float("nan")
    s.blocks(64, lists)
    out, lse = f64(s.out), f64(s.lse)
    assert np.isnan(out[1]).all()
    s.out[1], s.lse[1] = torch.from_numpy(ref[0][1]).to(s.out), torch.from_numpy(ref[1][1]).to(s.lse)
    s.check(ref)


@pytest.mark.parametrize("low", [float("-inf"), torch.finfo(BF).min, -1e30])
def test_lowest_keys(gpu_lib, low):
    """Logits of -inf or near the type's lowest value (a key whose first element is that, under
    a query of one): such keys weigh nothing, no row turns NaN."""
    s = Step(past=[30, 2], new=[1, 2], T=300, seed=6)
    s.q[..., 0] = 1.0
    s.kc[:, :, 64:192, 0] = low                       # two whole tiles, and the first key
    s.kc[:, :, 0, 0] = low
    ref = s.reference()
    s.shared()
    s.check(ref)


@pytest.mark.parametrize("low", [float("-inf"), torch.finfo(F32).min, -1e30])
def test_lowest_keys_f32(gpu_lib, low):
    """The same in float32, in more splits than have another key, and among listed blocks."""
    s = Step(past=[30, 2], new=[1, 2], T=1000, seed=6, dtype=F32)
    s.q[..., 0] = 1.0
    s.kc[:, :, 64:900, 0] = low
    s.kc[:, :, 0, 0] = low
    ref = s.reference()
    s.shared()
    s.check(ref)
    lists = torch.arange(16, dtype=torch.int32, device="cuda").expand(3, 2, 16).contiguous()
    s.blocks(64, lists)
    s.check(s.reference(lists, 64))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,block", [(640, None), (640, 64), (20, None), (9000, None)])
def test_not_finite_reaches_the_rows_that_see_it(gpu_lib, T, block, dtype):
    """A NaN in a query or a key that a row sees, or a logit of +inf: its output and its
    log-sum-exp are NaN, also where none of its logits is a number, and only its own."""
    s = Step(past=[20, 3, 9], new=[1, 3, 1], T=T, seed=9, dtype=dtype)
    s.q[4, :, 1] = 1.0
    lists = None
    if block:
        lists = torch.arange(T // block, dtype=torch.int32, device="cuda").expand(5, 2, -1).contiguous()
    O, lse, spread = s.reference(lists, block)
    s.q[0, 2, 5] = float("nan")
    s.ks[1, :, 4, 7] = float("nan")                   # the second new token of request 1
    s.ks[2, 0, 9, 1] = float("inf")
    bad = np.zeros((5, 8), bool)
    bad[0, 2] = bad[2:4] = bad[4, :4] = True
    if block:
        s.blocks(block, lists)
    else:
        s.shared()
    assert np.array_equal(np.isnan(f64(s.lse)), bad)
    assert np.array_equal(np.isnan(f64(s.out)), np.broadcast_to(bad[..., None], O.shape))
    at = torch.from_numpy(bad).cuda()
    s.out[at], s.lse[at] = torch.from_numpy(O[bad]).to(s.out), torch.from_numpy(lse[bad]).to(s.lse)
    s.check((O, lse, spread))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_largest_step(gpu_lib, dtype):
    """The most rows, heads and requests of a step: one new token each over one context key
    and its own, softmax of two logits."""
    n, H, d = 65536, 64, 64
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *sh: torch.randn(*sh, device="cuda", generator=g).to(dtype)    # noqa: E731
    kc, vc, ks, vs = rnd(1, H, 1, d), rnd(1, H, 1, d), rnd(n, H, 1, d), rnd(n, H, 1, d)
    q = rnd(n, H, d)
    req = relaxkv.Request(torch.zeros(1, 1, H, d, dtype=dtype, device="cuda"), kc, vc, 0.5)
    b = req.alloc_batch(n, n, 1)
    z = torch.zeros(n, dtype=torch.int32, device="cuda")
    req.plan_batch(b, z, z + 1)
    assert b.counts_to_host() == [n, n, 1, 0]
    out = torch.empty_like(q)
    lists = torch.zeros(n, H, 1, dtype=torch.int32, device="cuda")
    for blocks in (False, True):
        out.zero_()
        if blocks:
            ws = req.alloc_block_workspace(b, 16, 1)
            req.block_attn(b, 0, kc, vc, 16, lists, q, ks, vs, out, None, ws)
        else:
            ws = req.alloc_shared_workspace(b)
            req.shared_attn(b, 0, kc, vc, q, ks, vs, out, None, ws)
        del ws
        for i in range(0, n, 8192):
            Q, K, V = (t[i:i + 8192].double().reshape(-1, H, d) for t in (q, ks, vs))
            K0, V0 = kc[0, :, 0].double(), vc[0, :, 0].double()
            p = torch.sigmoid(((Q * K).sum(-1) - (Q * K0).sum(-1)) * d ** -0.5)[..., None]
            O = p * V + (1 - p) * V0
            spread = p * (V - O).abs() + (1 - p) * (V0 - O).abs()
            err = (out[i:i + 8192].double() - O).abs()
            if dtype == BF:                           # attn_tol
                tol = 1.01 * 2.0 ** -8 * (1 + 2.0 ** -3) * (spread + O.abs()) + 1e-4 * spread + 1e-6
            else:
                tol = torch.full_like(O, 1e-5 * float(O.abs().max()))
            assert bool((err <= tol).all())


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,H_kv,past,new,T", [
    (160, 1, [3, 70], [2, 1], 300),           # a group's second chunk of 32 heads
    (129, 1, [3], [1], 100),                  # of one head
    (8, 2, [5] * 33, [1] * 33, 700),          # 132 rows: a last chunk of 4
    (8, 2, [5] * 33, [1] * 33, 8000),
    (8, 2, [0] * 7, [7] * 7, 100),            # 196 rows: of 68
    (10, 10, [2, 9, 0], [1, 1, 17], 520),     # heads that do not divide over the XCDs
    (65, 1, [30], [1], 64), (64, 1, [30], [1], 65),     # around the rows that 16-row waves hold
])
def test_chunk_borders(gpu_lib, H, H_kv, past, new, T, d, dtype):
    s = Step(past=past, new=new, T=T, H=H, H_kv=H_kv, d=d, dtype=dtype, seed=12, room=max(
        p + n for p, n in zip(past, new)))
    s.shared()
    s.check(s.reference(), "shared")
    nb = -(-T // 32)
    lists = torch.from_numpy(_lists(np.random.default_rng(1), s.n, H_kv, nb, min(nb, 11))).cuda()
    s.out.fill_(7.0), s.lse.fill_(7.0)
    s.blocks(32, lists)
    s.check(s.reference(lists, 32), "blocks")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_smallest_and_largest_scales(gpu_lib, dtype):
    """Under a tiny scale all keys weigh the same; under a huge one the largest logit alone counts:
    the next one is further below it than a float32 logit is rounded."""
    for scale in (1e-30, 1e-37):
        s = Step(past=[30, 2], new=[1, 2], T=300, seed=6, dtype=dtype, scale=scale)
        s.shared()
        s.check(s.reference())
    for scale in (1e5, 1e30):
        for T in (300, 5000):
            s = Step(past=[30, 2], new=[1, 2], T=T, seed=6, dtype=dtype, scale=scale)
            s.shared()
            q, k, v = f64(s.q), f64(s.kc[0]), f64(s.vc[0])
            seen = 0
            for t in range(s.n):
                own = slice(0, int(s.pos[t]) - T + 1)
                for h in range(s.H):
                    g = h // (s.H // s.H_kv)
                    K, V = (np.concatenate((c[g], f64(x[s.seq[t], g, own]))) for c, x in ((k, s.ks), (v, s.vs)))
                    x = K @ q[t, h]
                    i, j = np.argsort(-x)[:2]
                    # Each logit is off by 130 roundings of 2^-24 of the sum of its products' sizes;
                    # where the two are closer than that, either may win.
                    err = 2 * 130 * 2.0 ** -24 * (np.abs(K[[i, j]]) @ np.abs(q[t, h])).max()
                    if (x[i] - x[j] - err) * scale < 30:
                        continue
                    seen += 1
                    got = f64(s.out[t, h])
                    assert np.all(np.abs(got - V[i]) <= 1e-6 + 2.0 ** -20 * np.abs(V).max()), (scale, T, t, h)
                    assert abs(float(s.lse[t, h]) - x[i] * scale) <= err * scale + 1
            assert seen >= s.n * s.H // 2


def test_bit_identical_runs_and_streams(gpu_lib):
    """Same bits on every run, on another stream and with a used workspace."""
    s = Step(past=[100, 3, 60], new=[1, 20, 1], T=3000, H=16, H_kv=4)
    ws = s.req.alloc_shared_workspace(s.batch)
    s.shared(ws)
    a, l = s.out.clone(), s.lse.clone()
    ws.fill_(255)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.out.zero_()
        s.shared(ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, s.out) and torch.equal(l, s.lse)
    s.req.shared_attn(s.batch, 0, s.kc, s.vc, s.q, s.ks, s.vs, s.out, None, ws)
    assert torch.equal(a, s.out)


def test_layers(gpu_lib):
    """The layer's slab of the cache is the one read."""
    s = Step(past=[5], new=[2], T=200, L=3, spare=4)
    for l in (2, 0, 1):
        s.shared(layer=l)
        s.check(s.reference(layer=l), f"layer {l}")
    lists = torch.tensor([0, 3], dtype=torch.int32, device="cuda").expand(2, 2, 2).contiguous()
    s.blocks(64, lists, layer=1)
    s.check(s.reference(lists, 64, layer=1))


def test_bad_lengths_leave_everything(gpu_lib):
    """A plan of bad lengths has no rows: outputs stay as they were."""
    s = Step(past=[5, 1], new=[2, 1], T=200)
    s.past_d[1] = -1
    s.req.plan_batch(s.batch, s.past_d, s.new_d)
    s.shared()
    lists = torch.zeros(3, 2, 1, dtype=torch.int32, device="cuda")
    s.blocks(64, lists)
    torch.cuda.synchronize()
    assert torch.all(s.out == 7.0) and torch.all(s.lse == 7.0)
    with pytest.raises(relaxkv.RelaxKVError):
        s.batch.counts_to_host()
    assert s.batch.counts_to_host(check=False) == [0, 0, 0, relaxkv.BATCH_ERR_LENGTHS]


def test_binding_refusals(gpu_lib):
    s = Step(past=[5, 1], new=[2, 1], T=200)
    ws = s.req.alloc_shared_workspace(s.batch)
    good = dict(batch=s.batch, layer=0, k_cache=s.kc, v_cache=s.vc, q=s.q, k_suffix=s.ks,
                v_suffix=s.vs, out=s.out, lse_out=s.lse, ws=ws)
    s.req.shared_attn(**good)
    other = Step(past=[5, 1], new=[2, 1], T=201)
    for bad in (dict(q=s.q[:2]), dict(q=s.q.float()), dict(q=s.q.cpu()), dict(out=s.out[:, :4]),
                dict(lse_out=s.lse.double()), dict(k_suffix=s.ks[:1]), dict(v_suffix=s.vs.float()),
                dict(k_suffix=s.ks.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(batch=other.batch), dict(batch=None), dict(k_cache=other.kc), dict(ws=ws.cpu())):
        with pytest.raises(ValueError):
            s.req.shared_attn(**{**good, **bad})
    for bad in (dict(ws=ws[:64]), dict(ws=None), dict(layer=1), dict(layer=-1)):
        with pytest.raises(relaxkv.RelaxKVError):
            s.req.shared_attn(**{**good, **bad})
    lists = torch.zeros(3, 2, 2, dtype=torch.int32, device="cuda")
    wsb = s.req.alloc_block_workspace(s.batch, 64, 2)
    blk = dict(good, block=64, blocks=lists, ws=wsb)
    s.req.block_attn(**blk)
    for bad in (dict(blocks=lists[:2]), dict(blocks=lists.long()), dict(blocks=lists[0])):
        with pytest.raises(ValueError):
            s.req.block_attn(**{**blk, **bad})
    for bad in (dict(block=48), dict(blocks=torch.zeros(3, 2, 5, dtype=torch.int32, device="cuda"))):
        with pytest.raises(relaxkv.RelaxKVError):
            s.req.block_attn(**{**blk, **bad})
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_output_in_place_of_the_queries(gpu_lib, dtype):
    for kw in (SHARED["mixed"], SHARED["suffix-splits"], SHARED["one"]):
        s = Step(dtype=dtype, **kw)
        s.shared()
        want, x = s.out.clone(), s.q.clone()
        ws = s.req.alloc_shared_workspace(s.batch)
        s.req.shared_attn(s.batch, 0, s.kc, s.vc, x, s.ks, s.vs, x, None, ws)
        assert torch.equal(x[:s.n], want[:s.n])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_offsets_past_32_bits(gpu_lib, dtype):
    """The last layer and head of a cache of more than 2^32 elements, and suffixes 2^31 elements apart,
    written by batch_rows: against a short cache of the same keys."""
    L, H, T, d = 6, 16, 1 << 19, 128
    if torch.cuda.mem_get_info()[0] < 110 << 30:
        pytest.skip("needs 110 GB of device memory")
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *sh: torch.randn(*sh, device="cuda", generator=g).to(dtype)    # noqa: E731
    far, n, block, m = 1 << 31, 3, 64, 20
    kc, vc = (torch.zeros(L, H, T, d, dtype=dtype, device="cuda") for _ in range(2))
    kc[-1, :, -m * block:], vc[-1, :, -m * block:] = rnd(H, m * block, d), rnd(H, m * block, d)
    buf = [torch.zeros(far * (n - 1) + H * 2 * d, dtype=dtype, device="cuda") for _ in range(2)]
    ks, vs = (b.as_strided((n, H, 2, d), (far, 2 * d, d, 1)) for b in buf)
    req = relaxkv.Request(torch.zeros(L, 1, H, d, dtype=dtype, device="cuda"), kc, vc, 0.5)
    b = req.alloc_batch(n, n, 2)
    z = torch.zeros(n, dtype=torch.int32, device="cuda")
    req.plan_batch(b, z, z + 1)
    q, k, v = rnd(n, H, d), rnd(n, H, d), rnd(n, H, d)
    qr, out = torch.empty_like(q), torch.empty_like(q)
    req.batch_rows(relaxkv.Rope(), b, q, k, v, qr, ks, vs)
    assert torch.equal(qr, q) and torch.equal(ks[:, :, 0], k) and torch.equal(vs[:, :, 0], v)
    nb = T // block
    lists = torch.arange(nb - m, nb, dtype=torch.int32, device="cuda").expand(n, H, m).contiguous()
    req.block_attn(b, L - 1, kc, vc, block, lists, q, ks, vs, out, None, req.alloc_block_workspace(b, block, m))
    sk, sv = (t[-1:, :, -m * block:].contiguous() for t in (kc, vc))
    short = relaxkv.Request(torch.zeros(1, 1, H, d, dtype=dtype, device="cuda"), sk, sv, 0.5)
    c = short.alloc_batch(n, n, 2)
    short.plan_batch(c, z, z + 1)
    want, dense = torch.empty_like(q), [t.contiguous() for t in (ks, vs)]
    short.block_attn(c, 0, sk, sv, block, lists - (nb - m), q, *dense, want, None,
                     short.alloc_block_workspace(c, block, m))
    assert torch.equal(out, want) and bool(want.any(-1).all())
    # All of the cache: the other keys are 0, and so are their values.
    lse = torch.empty(n, H, device="cuda")
    req.shared_attn(b, L - 1, kc, vc, q, ks, vs, out, lse, req.alloc_shared_workspace(b))
    zeros = T - m * block
    K, V = (torch.cat((t[0].double().expand(n, -1, -1, -1), o[:, :, None].double()), 2)
            for t, o in ((sk, k), (sv, v)))
    x = (K * q[:, :, None].double()).sum(-1) * d ** -0.5
    z = x.exp().sum(-1) + zeros
    p = (x.exp() / z[..., None])[..., None]
    O = (p * V).sum(2)
    spread = (p * (V - O[:, :, None]).abs()).sum(2) + (zeros / z)[..., None] * O.abs()
    O, spread = f64(O), f64(spread)
    tol = attn_tol(O, spread) if dtype == BF else 1e-5 * np.abs(O).max()
    assert np.all(np.abs(f64(out) - O) <= tol)
    assert np.abs(f64(lse) - f64(z.log())).max() <= 5e-4
    mean = torch.empty(L, H, nb, d, dtype=dtype, device="cuda")
    req.block_means(None, kc, block, mean)
    one = torch.empty(1, H, m, d, dtype=dtype, device="cuda")
    short.block_means(0, sk, block, one)
    assert torch.equal(mean[-1, :, -m:], one[0]) and not mean[:-1].any() and not mean[-1, :, :-m].any()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_steps_without_rows(gpu_lib, dtype):
    """A batch with no room for rows, and a step in which every request rests: nothing is
    written."""
    for new, extra in (([0, 0], 0), ([0, 0], 5)):
        s = Step(past=[7, 0], new=new, T=100, dtype=dtype, extra_rows=extra, room=9)
        assert s.batch.counts_to_host() == [0, 0, 0, 0]
        assert s.batch.row_off.tolist() == [0, 0, 0] and s.batch.row_seq.tolist() == [-1] * extra
        n = s.q.shape[0]
        k = torch.zeros(n, 2, 128, dtype=dtype, device="cuda")
        ks, vs, q_rot = s.ks.clone(), s.vs.clone(), torch.full_like(s.q, 7.0)
        s.req.batch_rows(relaxkv.Rope(), s.batch, s.q, k, k, q_rot, s.ks, s.vs)
        s.shared()
        lists = torch.full((n, 2, 3), -7, dtype=torch.int32, device="cuda")
        means = torch.zeros(2, 7, 128, dtype=dtype, device="cuda")
        ws = s.req.alloc_block_workspace(s.batch, 16, 3)
        s.req.block_select(s.batch, 16, means, s.q, lists, ws)
        s.blocks(16, lists)
        assert torch.equal(ks.nan_to_num(9), s.ks.nan_to_num(9)) and torch.equal(vs.nan_to_num(9), s.vs.nan_to_num(9))
        for t, v in ((q_rot, 7), (s.out, 7), (s.lse, 7), (lists, -7)):
            assert bool((t == v).all())


def test_expanded_suffix_is_refused(gpu_lib):
    """A stride of 0 (an expanded tensor) selects the dense layout in the descriptor, so it must
    not get there."""
    s = Step(past=[5, 1], new=[2, 1], T=200)
    ws = s.req.alloc_shared_workspace(s.batch)
    for dim in range(3):
        k = s.ks.narrow(dim, 0, 1).expand(s.ks.shape)
        with pytest.raises(ValueError):
            s.req.shared_attn(s.batch, 0, s.kc, s.vc, s.q, k, k, s.out, s.lse, ws)
        with pytest.raises(ValueError):
            s.req.batch_rows(relaxkv.Rope(), s.batch, None, None, None, None, k, k)
    torch.cuda.synchronize()
