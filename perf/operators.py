"""Performance cases of the batched serving operators: what a program runs between a
model's projections and its attention output when many requests share one context cache.

Kinds of case (one operator pass each):
  plan     row maps of a step (request and position of every row) from the requests' lengths
  rows     norms of queries and keys per head with the position rotation, values copied: into
           dense fresh rows ("fresh"), or into a batch's suffix caches ("batch")
  shared   attention of a batch's rows over the shared context cache and, causally, their own
           request's suffix
  means    key block means of the context cache
  blocks   per row and KV head: the context blocks that a score by block means selects, then the
           attention over those blocks and the request's own suffix

``own`` False computes a case in plain torch operations, True through the binding.
"""

import functools
import math
import random

import torch

own = False

SHIFT = 8.0                # what the shared query direction adds to a relevant key's logit
EPS = 1e-6


def listed():
    def case(name, kind, **kw):
        c = dict(name=name, kind=kind, B=1, T=1024, H=32, Hkv=8, d=128, dtype="bf16", past=0, new=1,
                 spare=0, L=1, rot=128, norm=True, inter=False, theta=1e6, n=0, block=64, sel=0,
                 far=0)
        c.update(kw)
        return c

    return [
        # A decode step of 64 requests over an 8K context: one row each, latency alone.
        case("plan-decode-64", "plan", B=64, T=8192, past=700),
        # A mixed step of many requests: some decode, some bring a whole question.
        case("plan-mixed-1500", "plan", B=1500, T=32768, past=2000, new=60),
        # The new tokens of 16 decoding requests into their suffix caches.
        case("rows-decode-16", "rows", B=16, T=8192, past=500),
        # A middle layer's active targets of a 32K repair: half of the context's rows.
        case("rows-targets-32k", "rows", n=16411, T=32768, H=40),
        # float32, partial interleaved rotation without norms, positions up to the longest
        # context the library takes.
        case("rows-f32-far", "rows", n=3001, T=4096, H=12, Hkv=3, d=64, dtype="f32", rot=32,
             norm=False, inter=True, theta=1e4, far=1 << 22),
        # The smallest workload of the repository, shared by four requests.
        case("shared-f32-1k", "shared", B=4, T=1024, H=4, Hkv=2, d=64, dtype="f32", past=20, new=3),
        # 64 sampled continuations of one 32K document, a token each.
        case("shared-decode-32k", "shared", B=64, T=32768, H=40, past=600),
        # Questions of ragged lengths, some already decoding, on a ragged 8K context.
        case("shared-mixed-8k", "shared", B=20, T=8011, past=120, new=96, spare=181),
        # The key block means of a repaired 16K cache, every layer.
        case("means-16k", "means", L=40, T=16384, H=40),
        # A ragged float32 cache allocated for more tokens, a partial last block.
        case("means-f32-1k", "means", L=2, T=1003, H=4, Hkv=2, d=64, dtype="f32", block=32, spare=21),
        # Eight requests decoding over a 128K context, 2K keys each.
        case("blocks-decode-128k", "blocks", B=8, T=131072, past=300, sel=32),
        # A ragged batch of short new runs at d 64, a wide GQA group, small blocks.
        case("blocks-mixed-16k", "blocks", B=33, T=16381, H=24, Hkv=2, d=64, past=90, new=9,
             block=32, sel=24),
    ]


HEADS = [(32, 8, 128), (40, 8, 128), (16, 4, 128), (12, 3, 128), (14, 2, 128), (32, 16, 128),
         (4, 4, 128), (24, 2, 64), (8, 2, 64), (16, 4, 64)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["plan", "rows", "rows", "shared", "shared", "shared", "means", "blocks",
                       "blocks", "blocks"])
    f32 = rng.random() < 0.25
    H, Hkv, d = rng.choice(HEADS)
    top = {"plan": 32768, "rows": 32768, "shared": 32768, "means": 16384, "blocks": 131072}[kind]
    if f32:
        top = min(top, 3000)
    T = _log_int(rng, 200, top)
    if rng.random() < 0.3:
        T = max(64, T // 64 * 64)
    B = _log_int(rng, 1, {"plan": 1500, "rows": 128}.get(kind, 64))
    decode = rng.random() < 0.5
    new = 1 if decode else _log_int(rng, 2, 60 if kind == "plan" else 24)
    block = rng.choice([16, 32, 64, 128])
    c = dict(kind=kind, B=B, T=T, H=H, Hkv=Hkv, d=d, dtype="f32" if f32 else "bf16",
             past=_log_int(rng, *((40, 2000) if kind == "plan" else (1, 200 if f32 else 600))), new=new,
             spare=rng.choice([0, 0, rng.randint(1, 700)]), L=1,
             rot=rng.choice([d, d, d // 2, d // 4]), norm=rng.random() < 0.6,
             inter=rng.random() < 0.3, theta=rng.choice([1e4, 5e5, 1e6]), n=0, block=block, sel=0,
             far=0)
    if kind == "rows" and rng.random() < 0.5:
        c["n"], c["far"] = _log_int(rng, 1, 3000 if f32 else 8000), rng.choice([0, 0, 1 << 22])
    if kind == "means":
        c["L"] = _log_int(rng, 1, 16)
    if kind == "blocks":
        c["sel"] = min(_log_int(rng, 2, 48), max(1, 2048 // block), -(-T // block))
    if kind in ("shared", "blocks"):
        # the plain form's logits of all rows stay below 2^31 bytes
        keys = T if kind == "shared" else c["sel"] * block * d // 4
        while (_count(c) + 8) * H * keys * 4 >= 1 << 31 or _count(c) * H * T > 1 << 27:
            c["B"], c["new"] = max(1, c["B"] // 2), max(1, c["new"] // 2)
            if c["B"] == 1 and c["new"] == 1:
                break
    return c


# ------------------------------------------------------------------ inputs

@functools.lru_cache(maxsize=256)
def _lens_of(B, past, new):
    """(past, new) lengths of the B requests: one fixed draw, so that shapes are a property
    of the case.  A decode step (new 1) has a paused request now and then (no row); a
    mixed step has decoding requests, requests of up to `new` rows and first tokens."""
    r = random.Random(B * 1000003 + past * 1009 + new)
    p, n = [], []
    for b in range(B):
        p.append(0 if r.random() < 0.05 else r.randint(max(1, past // 4), max(1, past)) if past else 0)
        if new == 1:
            n.append(0 if b and r.random() < 0.05 else 1)
        else:
            n.append(1 if r.random() < 0.4 else 0 if b and r.random() < 0.05 else r.randint(1, new))
    return tuple(p), tuple(n)


def _lens(c):
    return _lens_of(c["B"], c["past"], c["new"])


def _count(c):
    return sum(_lens(c)[1])


def _cap(c):
    """Rows allocated: a mixed step's buffers are a few rows larger than the step."""
    return _count(c) + (0 if c["new"] == 1 else 5)


def _room(c):
    """Suffix tokens allocated per request."""
    return c["past"] + c["new"] + 7


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _blocks(c):
    return -(-c["T"] // c["block"])


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(c, g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(_dtype(c))


def _cache(c, g):
    """[L][Hkv][T][d] as a view of an allocation with spare tokens."""
    full = torch.empty(c["L"], c["Hkv"], c["T"] + c["spare"], c["d"], device="cuda", dtype=_dtype(c))
    for l in range(c["L"]):
        full[l] = _randn(c, g, *full.shape[1:])
    return full[:, :, :c["T"]]


def _maps(c):
    """Request and position of every row, -1 behind the last."""
    past, new = _lens(c)
    seq = [b for b in range(c["B"]) for _ in range(new[b])]
    pos = [c["T"] + past[b] + i for b in range(c["B"]) for i in range(new[b])]
    pad = [-1] * (_cap(c) - len(seq))
    return [torch.tensor(v + pad, dtype=torch.int64, device="cuda") for v in (seq, pos)]


def _inputs(c, seed):
    """Every tensor the case's calls take, made from the seed alone."""
    g = _gen(seed)
    B, T, H, Hkv, d, kind = (c[k] for k in ("B", "T", "H", "Hkv", "d", "kind"))
    x = {}
    if kind == "plan":
        # the new rows in an order that the seed gives, after suffixes of any length
        order = torch.randperm(B, generator=g, device="cuda")
        x["past"] = torch.randint(0, c["past"] + 7, (B,), generator=g, device="cuda").int()
        x["new"] = torch.tensor(_lens(c)[1], dtype=torch.int32, device="cuda")[order]
        return x
    if kind == "means":
        x["k"] = _cache(c, g)
        return x
    if not (kind == "rows" and c["n"]):
        x["past"], x["new"] = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in _lens(c))
        x["seq"], x["pos"] = _maps(c)
        x["ks"], x["vs"] = (_randn(c, g, B, Hkv, _room(c), d) for _ in range(2))
    if kind == "rows":
        n = c["n"] or _cap(c)
        x["qkv"] = _randn(c, g, n, (H + 2 * Hkv) * d)        # one row of the fused projection
        x["qw"], x["kw"] = ((1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(_dtype(c))
                            for _ in range(2))
        x["freq"] = (c["theta"] ** (-torch.arange(0, c["rot"], 2, device="cuda",
                                                  dtype=torch.float64) / c["rot"])).float()
        if c["n"]:
            high = c["far"] or c["T"]
            x["pos"] = torch.randint(0, high, (n,), generator=g, device="cuda").sort().values.int()
        return x
    # Attention: the queries of a KV head share a direction, and 2% of the positions, in
    # spans of 64 as a retrieved passage lies, carry it in their keys.
    n = _cap(c)
    x["k"], x["v"] = _cache(c, g), _cache(c, g)
    u = torch.randn(Hkv, d, generator=g, device="cuda")
    x["q"] = (_randn(c, g, n, H, d).float() + u.repeat_interleave(H // Hkv, 0)).to(_dtype(c))
    spans = torch.randperm(-(-T // 64), generator=g, device="cuda")[:max(1, T // 64 // 50)]
    rel = (spans[:, None] * 64 + torch.arange(64, device="cuda")).flatten()
    rel = rel[rel < T]
    x["k"][0][:, rel] = (x["k"][0][:, rel].float() + SHIFT / math.sqrt(d) * u[:, None]).to(_dtype(c))
    if kind == "blocks":
        x["means"] = _plain_means(c, x["k"])
    return x


def prepare(case, seed):
    c = case
    x = _inputs(c, seed)
    s = dict(c=c, x=x)
    B, T, H, Hkv, d, kind = (c[k] for k in ("B", "T", "H", "Hkv", "d", "kind"))
    n = c["n"] or _cap(c)
    dt = _dtype(c)
    if kind == "means":
        s["means"] = torch.zeros(c["L"], Hkv, _blocks(c), d, device="cuda", dtype=dt)
    if kind == "rows":
        s["q"] = torch.zeros(n, H, d, device="cuda", dtype=dt)
        if c["n"]:
            s["kv"] = torch.zeros(2, n, Hkv, d, device="cuda", dtype=dt)
    if kind in ("shared", "blocks"):
        s["out"] = torch.zeros(n, H, d, device="cuda", dtype=dt)
        s["lse"] = torch.zeros(n, H, device="cuda")
    if kind == "blocks":
        s["list"] = torch.zeros(n, Hkv, c["sel"], device="cuda", dtype=torch.int32)
    if own:
        from paper_2609_33503_amd import relaxkv as rk
        # The request's descriptor (the context cache); kinds that never read it get a
        # one-layer view of the right shape.
        k = x.get("k")
        if k is None:
            k = torch.empty(1, Hkv, T, d, device="cuda", dtype=dt)
        req = rk.Request(torch.zeros(c["L"], 1, H, d, device="cuda", dtype=dt), k, x.get("v", k), 0.15)
        s["req"] = req
        if "past" in x:
            s["batch"] = req.alloc_batch(B, n, _room(c))
            req.plan_batch(s["batch"], x["past"], x["new"])
        if kind == "rows":
            s["rope"] = rk.Rope(x["freq"], x["qw"] if c["norm"] else None,
                                x["kw"] if c["norm"] else None, EPS, c["inter"])
        if kind == "shared":
            s["ws"] = req.alloc_shared_workspace(s["batch"])
        if kind == "blocks":
            s["ws"] = req.alloc_block_workspace(s["batch"], c["block"], c["sel"])
    return s


def _split(c, qkv):
    """The fused projection's queries, keys and values, as views."""
    H, Hkv, d = c["H"], c["Hkv"], c["d"]
    n = qkv.shape[0]
    q, k, v = qkv.split([H * d, Hkv * d, Hkv * d], 1)
    return q.view(n, H, d), k.view(n, Hkv, d), v.view(n, Hkv, d)


def run(state):
    s, c, x = state, state["c"], state["x"]
    kind = c["kind"]
    if own:
        req = s["req"]
        if kind == "plan":
            b = s["batch"]
            req.plan_batch(b, x["past"], x["new"])
            return {"row_off": b.row_off, "row_seq": b.row_seq, "row_pos": b.row_pos}
        if kind == "rows":
            q, k, v = _split(c, x["qkv"])
            if c["n"]:
                req.fresh_rows(s["rope"], x["pos"], q, k, v, s["q"], s["kv"][0], s["kv"][1])
                return {"q": s["q"], "k": s["kv"][0], "v": s["kv"][1]}
            req.batch_rows(s["rope"], s["batch"], q, k, v, s["q"], x["ks"], x["vs"])
            return {"q": s["q"], "k": x["ks"], "v": x["vs"]}
        if kind == "means":
            req.block_means(None, x["k"], c["block"], s["means"])
            return s["means"]
        if kind == "shared":
            req.shared_attn(s["batch"], 0, x["k"], x["v"], x["q"], x["ks"], x["vs"], s["out"],
                            s["lse"], s["ws"])
            return {"out": s["out"], "lse": s["lse"]}
        req.block_select(s["batch"], c["block"], x["means"][0], x["q"], s["list"], s["ws"])
        req.block_attn(s["batch"], 0, x["k"], x["v"], c["block"], s["list"], x["q"], x["ks"],
                       x["vs"], s["out"], s["lse"], s["ws"])
        return {"blocks": s["list"], "out": s["out"], "lse": s["lse"]}
    if kind == "plan":
        return _plain_plan(c, x)
    if kind == "rows":
        return _plain_rows(c, s, x)
    if kind == "means":
        s["means"].copy_(_plain_means(c, x["k"]))
        return s["means"]
    n = _count(c)
    if kind == "shared":
        s["out"][:n], s["lse"][:n] = _plain_shared(c, x)
        return {"out": s["out"], "lse": s["lse"]}
    s["list"][:n] = _plain_select(c, x)
    s["out"][:n], s["lse"][:n] = _plain_block_attn(c, x, s["list"][:n])
    return {"blocks": s["list"], "out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------ plain forms (32 bits)

def _plain_plan(c, x):
    past, new, cap = x["past"].long(), x["new"].long(), _cap(c)
    ends = torch.cumsum(new, 0)
    off = torch.cat([torch.zeros_like(ends[:1]), ends])
    rows = torch.arange(cap, device="cuda")
    seq = torch.searchsorted(ends, rows, right=True)
    real = rows < ends[-1]
    at = seq.clamp(max=c["B"] - 1)
    pos = c["T"] + past[at] + rows - off[at]
    none = torch.full_like(rows, -1)
    return {"row_off": off.int(), "row_seq": torch.where(real, seq, none).int(),
            "row_pos": torch.where(real, pos, none).int()}


def _plain_norm_rotate(c, h, w, pos, freq):
    """[n][heads][d] in 32 bits: RMS norm of each head (where norm is set), then the rotation."""
    h = h.float()
    if c["norm"]:
        h = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * w.float()
    angle = pos.double()[:, None] * freq.double()           # far positions: angles in 64 bits
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    r = h[..., :c["rot"]]
    if c["inter"]:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = r[..., :c["rot"] // 2], r[..., c["rot"] // 2:]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([r, h[..., c["rot"]:]], -1).to(_dtype(c))


def _plain_rows(c, s, x):
    q, k, v = _split(c, x["qkv"])
    n = c["n"] or _count(c)
    pos = x["pos"][:n]
    s["q"][:n] = _plain_norm_rotate(c, q[:n], x["qw"], pos, x["freq"])
    k = _plain_norm_rotate(c, k[:n], x["kw"], pos, x["freq"])
    if c["n"]:
        s["kv"][0], s["kv"][1] = k, v
        return {"q": s["q"], "k": s["kv"][0], "v": s["kv"][1]}
    x["ks"][x["seq"][:n], :, pos - c["T"]] = k
    x["vs"][x["seq"][:n], :, pos - c["T"]] = v[:n]
    return {"q": s["q"], "k": x["ks"], "v": x["vs"]}


def _plain_means(c, k):
    """[L][Hkv][blocks][d]: sums in 64 bits, whatever their order; rounded once."""
    L, Hkv, T, d = k.shape
    b, full = c["block"], T // c["block"]
    m = k[:, :, :full * b].reshape(L, Hkv, full, b, d).sum(3, dtype=torch.float64) / b
    if T > full * b:
        m = torch.cat([m, k[:, :, full * b:].sum(2, keepdim=True, dtype=torch.float64) / (T - full * b)], 2)
    return m.to(k.dtype)


def _grouped(c, q):
    """[Hkv][n * G][d] in 32 bits."""
    n, G = q.shape[0], c["H"] // c["Hkv"]
    return q.float().view(n, c["Hkv"], G, c["d"]).transpose(0, 1).reshape(c["Hkv"], n * G, c["d"])


def _plain_suffix(c, x, n):
    """Logits [Hkv][n * G][room] of each row over its own request's suffix, masked, and the
    request-wise index that takes its probabilities back ([B][new] rows)."""
    B, H, Hkv, d, M, S = c["B"], c["H"], c["Hkv"], c["d"], max(_lens(c)[1]), _room(c)
    G, seq = H // Hkv, x["seq"][:n]
    own_pos = x["pos"][:n] - c["T"]
    at = own_pos - x["past"].long()[seq]                    # the row's place in its request
    qp = torch.zeros(B, M, Hkv, G, d, device="cuda")
    qp[seq, at] = x["q"][:n].float().view(n, Hkv, G, d)
    qp = qp.permute(0, 2, 1, 3, 4).reshape(B, Hkv, M * G, d)
    s = torch.matmul(qp, x["ks"].float().transpose(2, 3).contiguous()) / math.sqrt(d)
    s = s.view(B, Hkv, M, G, S)[seq, :, at]                 # [n][Hkv][G][S]
    keys = torch.arange(S, device="cuda")
    s = s.masked_fill((keys[None] > own_pos[:, None])[:, None, None], -math.inf)
    return s, seq, at, M


def _plain_suffix_out(c, x, p, seq, at, M):
    """[n][Hkv][G][d]: probabilities p over the own suffix times its values."""
    B, Hkv, d, S = c["B"], c["Hkv"], c["d"], _room(c)
    G = c["H"] // Hkv
    pp = torch.zeros(B, M, Hkv, G, S, device="cuda")
    pp[seq, at] = p
    pp = pp.permute(0, 2, 1, 3, 4).reshape(B, Hkv, M * G, S)
    o = torch.matmul(pp, x["vs"].float())
    return o.view(B, Hkv, M, G, d)[seq, :, at]


def _plain_shared(c, x):
    n, H, Hkv, d = _count(c), c["H"], c["Hkv"], c["d"]
    G = H // Hkv
    k, v = x["k"][0].float(), x["v"][0].float()
    s1 = torch.matmul(_grouped(c, x["q"][:n]), k.transpose(1, 2).contiguous()) / math.sqrt(d)
    s2, seq, at, M = _plain_suffix(c, x, n)
    m1 = s1.amax(-1).view(Hkv, n, G).transpose(0, 1)
    m = torch.maximum(m1, s2.amax(-1))                      # [n][Hkv][G]
    p1 = torch.exp(s1 - m.transpose(0, 1).reshape(Hkv, n * G, 1))
    p2 = torch.exp(s2 - m[..., None])
    z = p1.sum(-1).view(Hkv, n, G).transpose(0, 1) + p2.sum(-1)
    o = torch.matmul(p1, v).view(Hkv, n, G, d).transpose(0, 1) + _plain_suffix_out(c, x, p2, seq, at, M)
    return (o / z[..., None]).reshape(n, H, d).to(_dtype(c)), (m + torch.log(z)).reshape(n, H)


def _plain_select(c, x):
    """[n][Hkv][sel]: the blocks whose mean key has the largest product with the sum of the
    group's queries, in 64 bits and rounded to 32 once; ties to the lower block; ascending."""
    n, Hkv, d = _count(c), c["Hkv"], c["d"]
    qs = x["q"][:n].double().view(n, Hkv, c["H"] // Hkv, d).sum(2).transpose(0, 1)
    sc = torch.matmul(qs.contiguous(), x["means"][0].double().transpose(1, 2).contiguous()).float()
    best = torch.sort(sc, dim=-1, descending=True, stable=True).indices[..., :c["sel"]]
    return torch.sort(best, dim=-1).values.transpose(0, 1).int()


def _plain_block_attn(c, x, blocks):
    n, H, Hkv, d, b = _count(c), c["H"], c["Hkv"], c["d"], c["block"]
    G = H // Hkv
    pos = (blocks.long()[..., None] * b + torch.arange(b, device="cuda")).flatten(2)    # [n][Hkv][keys]
    real = pos < c["T"]
    at_k = pos.clamp(max=c["T"] - 1).transpose(0, 1)
    heads = torch.arange(Hkv, device="cuda")[:, None, None]
    k, v = (x[t][0][heads, at_k].float().transpose(0, 1) for t in ("k", "v"))           # [n][Hkv][keys][d]
    q = x["q"][:n].float().view(n, Hkv, G, d)
    s1 = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d)
    s1 = s1.masked_fill(~real[:, :, None], -math.inf)
    s2, seq, at, M = _plain_suffix(c, x, n)
    m = torch.maximum(s1.amax(-1), s2.amax(-1))
    p1, p2 = torch.exp(s1 - m[..., None]), torch.exp(s2 - m[..., None])
    z = p1.sum(-1) + p2.sum(-1)
    o = torch.matmul(p1, v) + _plain_suffix_out(c, x, p2, seq, at, M)
    return (o / z[..., None]).reshape(n, H, d).to(_dtype(c)), (m + torch.log(z)).reshape(n, H)


# ------------------------------------------------------------ work

def work(case):
    c = case
    B, T, H, Hkv, d, kind = (c[k] for k in ("B", "T", "H", "Hkv", "d", "kind"))
    e = 4 if c["dtype"] == "f32" else 2
    past, new = _lens(c)
    n = _count(c)
    if kind == "plan":
        return dict(bytes=8 * B + 4 * (B + 1) + 8 * _cap(c), flops=0)
    if kind == "rows":
        n = c["n"] or n
        return dict(bytes=2 * n * (H + 2 * Hkv) * d * e + 4 * n + 2 * d * e + 2 * c["rot"],
                    flops=n * (H + Hkv) * (3 * c["rot"] + (4 * d if c["norm"] else 0)))
    if kind == "means":
        return dict(bytes=c["L"] * Hkv * d * e * (T + _blocks(c)), flops=c["L"] * Hkv * d * T)
    held = sum(p + k for p, k in zip(past, new) if k)       # suffix tokens that some row sees
    seen = sum(k * p + k * (k + 1) // 2 for p, k in zip(past, new))
    io = 2 * n * H * d * e + 4 * n * H + 2 * held * Hkv * d * e
    if kind == "shared":
        return dict(bytes=io + 2 * Hkv * T * d * e, flops=4 * H * d * (n * T + seen))
    # every row's list may be another: at most the whole cache once
    keys = min(T, n * c["sel"] * c["block"])
    return dict(bytes=io + 2 * Hkv * keys * d * e + Hkv * _blocks(c) * d * e + 4 * n * Hkv * c["sel"],
                flops=4 * H * d * (n * min(T, c["sel"] * c["block"]) + seen) + 2 * n * Hkv * d * _blocks(c))


# ------------------------------------------------------------ float64 reference

def _exact_rows(c, x):
    n = c["n"] or _count(c)
    H, Hkv, d, r = c["H"], c["Hkv"], c["d"], c["rot"]
    flat = x["qkv"].double()
    pos = x["pos"][:n].double()
    res = {}
    for name, heads, start, w in (("q", H, 0, x["qw"]), ("k", Hkv, H * d, x["kw"])):
        h = flat[:n, start:start + heads * d].reshape(n, heads, d)
        if c["norm"]:
            h = h / torch.sqrt((h ** 2).sum(-1, keepdim=True) / d + EPS) * w.double()
        y = h.clone()
        for i in range(r // 2):
            i0, i1 = (2 * i, 2 * i + 1) if c["inter"] else (i, i + r // 2)
            co, si = (f(pos * x["freq"][i].double())[:, None] for f in (torch.cos, torch.sin))
            y[:, :, i0] = h[:, :, i0] * co - h[:, :, i1] * si
            y[:, :, i1] = h[:, :, i0] * si + h[:, :, i1] * co
        res[name] = y
    res["v"] = flat[:n, (H + Hkv) * d:].reshape(n, Hkv, d)
    if c["n"]:
        return res
    q = torch.zeros(_cap(c), H, d, dtype=torch.float64, device="cuda")
    q[:n] = res["q"]
    ks, vs = x["ks"].double(), x["vs"].double()
    seq, pos = x["seq"].tolist(), x["pos"].tolist()
    for i in range(n):
        ks[seq[i], :, pos[i] - c["T"]], vs[seq[i], :, pos[i] - c["T"]] = res["k"][i], res["v"][i]
    return {"q": q, "k": ks, "v": vs}


def _exact_attn(c, x, lists=None):
    """Row by request and KV head in 64 bits: softmax over the concatenated keys."""
    n, H, Hkv, d, T = _cap(c), c["H"], c["Hkv"], c["d"], c["T"]
    G = H // Hkv
    out = torch.zeros(n, H, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(n, H, dtype=torch.float64, device="cuda")
    past, new = _lens(c)
    for g in range(Hkv):
        hs = slice(g * G, (g + 1) * G)
        K, V = x["k"][0, g].double(), x["v"][0, g].double()
        kt = K.t().contiguous()
        r = 0
        for b in range(c["B"]):
            Sk, Sv = x["ks"][b, g].double(), x["vs"][b, g].double()
            for lo in range(0, new[b], 8):
                m = min(8, new[b] - lo)
                rows = torch.arange(r + lo, r + lo + m, device="cuda")
                q = x["q"][r + lo:r + lo + m, hs].double().reshape(m * G, d)
                see = past[b] + lo + torch.arange(m, device="cuda") + 1
                top = past[b] + lo + m
                s = torch.cat([q @ kt, q @ Sk[:top].t()], 1).view(m, G, T + top) / math.sqrt(d)
                late = torch.arange(top, device="cuda")[None] >= see[:, None]
                s[:, :, T:].masked_fill_(late[:, None], -math.inf)
                if lists is not None:
                    keep = torch.zeros(m, _blocks(c), dtype=torch.bool, device="cuda")
                    keep.scatter_(1, lists[rows, g].long(), True)
                    s[:, :, :T].masked_fill_(~keep.repeat_interleave(c["block"], 1)[:, None, :T], -math.inf)
                z = torch.logsumexp(s, -1)
                p = torch.exp(s - z[..., None]).view(m * G, T + top)
                out[rows, hs] = (p[:, :T] @ V + p[:, T:] @ Sv[:top]).view(m, G, d)
                lse[rows, hs] = z
            r += new[b]
    return out, lse


def exact(case, seed):
    c = case
    x = _inputs(c, seed)
    kind = c["kind"]
    if kind == "plan":
        off, seq, pos = [0], [], []
        for b, (p, k) in enumerate(zip(x["past"].tolist(), x["new"].tolist())):
            off.append(off[-1] + k)
            seq += [b] * k
            pos += [c["T"] + p + i for i in range(k)]
        pad = [-1] * (_cap(c) - len(seq))
        return {"row_off": torch.tensor(off, dtype=torch.int32),
                "row_seq": torch.tensor(seq + pad, dtype=torch.int32),
                "row_pos": torch.tensor(pos + pad, dtype=torch.int32)}
    if kind == "rows":
        return _exact_rows(c, x)
    if kind == "means":
        m = torch.empty(c["L"], c["Hkv"], _blocks(c), c["d"], dtype=torch.float64, device="cuda")
        for l in range(c["L"]):
            for h, part in enumerate(x["k"][l].double()):
                m[l, h] = torch.stack([t.mean(0) for t in part.split(c["block"])])
        return m
    if kind == "shared":
        out, lse = _exact_attn(c, x)
        return {"out": out, "lse": lse}
    n, Hkv, d, G = _count(c), c["Hkv"], c["d"], c["H"] // c["Hkv"]
    lists = torch.zeros(_cap(c), Hkv, c["sel"], dtype=torch.int32, device="cuda")
    for g in range(Hkv):
        q = sum(x["q"][:n, g * G + j].double() for j in range(G))
        sc = (q @ x["means"][0, g].double().t()).float()
        for lo in range(0, n, 64):
            by = torch.argsort(-sc[lo:lo + 64], dim=1, stable=True)[:, :c["sel"]]
            lists[lo:min(n, lo + 64), g] = by.sort(1).values.int()
    out, lse = _exact_attn(c, x, lists)
    return {"blocks": lists, "out": out, "lse": lse}
