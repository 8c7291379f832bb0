"""A decoding loop over a repaired cache as a serving program runs it: plan, norm and rotation
into the suffix caches, shared attention on one layer and selected blocks on the other, several
steps with requests that start, rest and bring whole questions; against the float64 oracle
fed the projections alone, and recorded into a graph that later steps replay."""

import numpy as np
import pytest
import torch

from batch_harness import HALF, attn_tol, f64
from oracle import batch_oracle as bo
from paper_2609_33503_amd import relaxkv

pytestmark = pytest.mark.gpu

L, T, H, H_kv, d, B, ROOM, ROWS, BLOCK, SEL = 2, 500, 10, 2, 64, 4, 60, 24, 32, 5
STEPS = [[7, 0, 1, 12], [1, 3, 1, 0], [1, 1, 1, 1], [0, 1, 1, 5], [1, 1, 1, 1]]


class Server:
    def __init__(self, seed=0):
        g = torch.Generator().manual_seed(seed)
        bf = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()       # noqa: E731
        self.bf = bf
        self.kc, self.vc = bf(L, H_kv, T, d), bf(L, H_kv, T, d)
        self.req = relaxkv.Request(bf(L, 1, H, d), self.kc, self.vc, 0.2)
        self.batch = self.req.alloc_batch(B, ROWS, ROOM)
        self.ks, self.vs = torch.zeros(L, B, H_kv, ROOM, d).to(self.kc), torch.zeros(L, B, H_kv, ROOM, d).to(self.kc)
        f = (1e4 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().cuda()
        self.rope = relaxkv.Rope(f, 1 + 0.1 * bf(d), 1 + 0.1 * bf(d))
        self.past = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.new = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.qkv = torch.zeros(L, ROWS, (H + 2 * H_kv) * d, dtype=torch.bfloat16, device="cuda")
        self.q, self.out = (torch.zeros(L, ROWS, H, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.lse = torch.zeros(L, ROWS, H, device="cuda")
        self.means = torch.zeros(1, H_kv, self.req.block_count(BLOCK), d, dtype=torch.bfloat16, device="cuda")
        self.lists = torch.zeros(ROWS, H_kv, SEL, dtype=torch.int32, device="cuda")
        self.req.block_means(1, self.kc, BLOCK, self.means)
        self.ws = self.req.alloc_shared_workspace(self.batch)
        self.wsb = self.req.alloc_block_workspace(self.batch, BLOCK, SEL)

    def step(self):
        r = self.req
        r.plan_batch(self.batch, self.past, self.new)
        for l in range(L):
            q, k, v = (t.unflatten(1, (-1, d)) for t in
                       self.qkv[l].split([H * d, H_kv * d, H_kv * d], 1))
            r.batch_rows(self.rope, self.batch, q, k, v, self.q[l], self.ks[l], self.vs[l])
            if l == 0:
                r.shared_attn(self.batch, l, self.kc, self.vc, self.q[l], self.ks[l], self.vs[l],
                              self.out[l], self.lse[l], self.ws)
            else:
                r.block_select(self.batch, BLOCK, self.means[0], self.q[l], self.lists, self.wsb)
                r.block_attn(self.batch, l, self.kc, self.vc, BLOCK, self.lists, self.q[l],
                             self.ks[l], self.vs[l], self.out[l], self.lse[l], self.wsb)
        self.past += self.new

    def load(self, new, seed):
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        g = torch.Generator().manual_seed(seed)
        n = sum(new)
        self.qkv[:, :n] = torch.randn(L, n, self.qkv.shape[2], generator=g).to(torch.bfloat16)


def test_decoding_loop(gpu_lib):
    s = Server()
    ks, vs = (np.zeros((L, B, H_kv, ROOM, d)) for _ in range(2))
    past = [0] * B
    for i, new in enumerate(STEPS):
        s.load(new, 100 + i)
        s.step()
        n = sum(new)
        off, seq, pos = bo.batch_plan(past, new, T)
        x = f64(s.qkv)[:, :n]
        for l in range(L):
            w = [f64(t) for t in (s.rope.q_weight, s.rope.k_weight)]
            f, eps = f64(s.rope.inv_freq), float(np.float32(1e-6))
            q = bo.norm_rope(x[l][:, :H * d].reshape(n, H, d), pos, f, w[0], eps)
            k = bo.norm_rope(x[l][:, H * d:(H + H_kv) * d].reshape(n, H_kv, d), pos, f, w[1], eps)
            v = x[l][:, (H + H_kv) * d:].reshape(n, H_kv, d)
            tol = lambda y: HALF[torch.bfloat16] * np.abs(y) + 2.0 ** -20 * np.abs(y).max(-1, keepdims=True)  # noqa: E731,E501
            assert np.all(np.abs(f64(s.q[l])[:n] - q) <= tol(q))
            # the attention is held to the rows that it was given
            got_k = f64(s.ks[l])
            for r in range(n):
                b, t = seq[r], pos[r] - T
                assert np.all(np.abs(got_k[b, :, t] - k[r]) <= tol(k[r]))
                ks[l, b, :, t], vs[l, b, :, t] = got_k[b, :, t], v[r]
            assert np.array_equal(got_k, ks[l]) and np.array_equal(f64(s.vs[l]), vs[l])
            lists = None
            if l == 1:
                lists = bo.block_select(f64(s.q[l])[:n], f64(s.means[0]), SEL)
                assert np.array_equal(s.lists.cpu().numpy()[:n], lists)
            O, lse, spread = bo.batch_attn(f64(s.q[l])[:n], seq, pos, f64(s.kc[l]), f64(s.vc[l]),
                                           ks[l], vs[l], None, lists, BLOCK)
            assert np.all(np.abs(f64(s.out[l])[:n] - O) <= attn_tol(O, spread)), (i, l)
            assert np.all(np.abs(f64(s.lse[l])[:n] - lse) <= 5e-4), (i, l)
        past = [p + k for p, k in zip(past, new)]
        assert s.past.tolist() == past


def test_step_graph_replays_match_eager(gpu_lib):
    """One recorded step serves every later one: lengths, rows and caches are read on the
    device.  Eager work and synchronisations lie between the replays; two graphs that are
    replayed in turn share the workspaces."""
    eager, s = Server(), Server()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.load([0] * B, 0)
        s.step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.step()
        graphs.append(g)
    s.past.zero_()
    for i, new in enumerate(STEPS):
        eager.load(new, 100 + i)
        eager.step()
        s.load(new, 100 + i)
        s.out.fill_(float("nan"))
        eager.out[:, sum(new):] = 0
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        n = sum(new)
        for a, b in ((s.q, eager.q), (s.out, eager.out), (s.lse, eager.lse)):
            assert torch.equal(a[:, :n], b[:, :n]), i
        assert torch.isnan(s.out[:, n:]).all()
        assert torch.equal(s.lists[:n], eager.lists[:n]) and torch.equal(s.ks, eager.ks)
        assert torch.equal(s.vs, eager.vs) and torch.equal(s.past, eager.past)
        _ = (s.out.nan_to_num() * 2).sum().item()


def test_two_batches_at_once(gpu_lib):
    """Two steps of different batches on two streams, each with its own workspace."""
    a, b = Server(1), Server(2)
    for x, new in ((a, STEPS[0]), (b, STEPS[3])):
        x.load(new, 5)
        x.step()
    want = [(x.out.clone(), x.lse.clone()) for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for x in (a, b):
        x.past.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for x, st in ((a, streams[0]), (b, streams[1])):
            with torch.cuda.stream(st):
                x.out.zero_()
                x.step()
                x.past.zero_()
    torch.cuda.synchronize()
    for x, (o, l) in zip((a, b), want):
        assert torch.equal(x.out, o) and torch.equal(x.lse, l)
