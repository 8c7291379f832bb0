"""Inputs and comparisons of the batched serving tests (seeded, made on the CPU)."""

import numpy as np
import torch

from oracle import batch_oracle as bo
from paper_2609_33503_amd import relaxkv

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative


def attn_tol(O, spread, sharp=1.0):
    """Bound of a bf16 output's error, elementwise; spread = sum_j p_j |V_j - O|.
    - A probability is rounded to bf16, off by at most 2^-8 of itself; numerator and
      normaliser take the same rounded values, so O moves by at most 2^-8 spread.  (Two keys of
      equal weight rounded opposite ways reach it.)
    - O is rounded once: 2^-8 |O|.
    - The partial outputs of the key splits are rounded to fp16, half a step of 11 bits, 2^-11 of
      each: with weights that sum to one, at most 2^-11 sum_j p_j |V_j| <= 2^-11 (spread + |O|).
    - Float32 logits: 130 roundings (128 products, the scale, the maximum) of 2^-24 of a sum
      of |q_c k_c| / sqrt(d), about 0.64 d / sqrt(d) = 7.2 for normal q and k at d 128 and
      below 13 for all of them: 1e-4, times `sharp` where the queries are scaled by it.  Each p
      is off by that factor, O by that much of the spread.
    - 1% for the products of these, 1e-6 for what is near zero."""
    h = HALF[torch.bfloat16]
    return 1.01 * h * (1 + 2.0 ** -3) * (spread + np.abs(O)) + 1e-4 * sharp * spread + 1e-6


def f64(t):
    return t.detach().double().cpu().numpy()


class Step:
    """One step of a batch: context cache, suffix caches, rows and the bound batch.
    `room` suffix tokens per request; every suffix token past a request's length, every row
    behind the last and `spare` context rows past T hold NaN."""

    def __init__(self, past, new, T, H=8, H_kv=2, d=128, dtype=torch.bfloat16, room=None,
                 extra_rows=0, spare=0, layout="bhsd", scale=0.0, seed=0, L=1, sharp=1.0):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g)                   # noqa: E731
        self.past, self.new, self.T, self.H, self.H_kv, self.d = past, new, T, H, H_kv, d
        self.dtype, self.sharp, B = dtype, sharp, len(past)
        self.n = sum(new)
        N = self.n + extra_rows
        self.room = room or max(p + k for p, k in zip(past, new)) + 3
        dev = lambda t: t.to(dtype).cuda()                              # noqa: E731
        full = [torch.full((L, H_kv, T + spare, d), float("nan")) for _ in range(2)]
        for t in full:
            t[:, :, :T] = rnd(L, H_kv, T, d)
        self.kc, self.vc = (dev(t)[:, :, :T] for t in full)
        q = torch.full((N, H, d), float("nan"))
        q[:self.n] = rnd(self.n, H, d) * sharp
        self.q = dev(q)
        suf = [torch.full((B, H_kv, self.room, d), float("nan")) for _ in range(2)]
        for b in range(B):
            for t in suf:
                t[b, :, :past[b] + new[b]] = rnd(H_kv, past[b] + new[b], d)
        order = {"bhsd": (0, 1, 2, 3), "bshd": (0, 2, 1, 3), "hbsd": (1, 0, 2, 3)}[layout]
        back = np.argsort(order).tolist()
        self.ks, self.vs = (dev(t).permute(order).contiguous().permute(back) for t in suf)
        dummy = torch.zeros(L, 1, H, d, dtype=dtype, device="cuda")
        self.req = relaxkv.Request(dummy, self.kc, self.vc, 0.15, softmax_scale=scale)
        self.scale = scale or d ** -0.5
        self.batch = self.req.alloc_batch(B, N, self.room)
        self.past_d, self.new_d = (torch.tensor(v, dtype=torch.int32, device="cuda")
                                   for v in (past, new))
        self.req.plan_batch(self.batch, self.past_d, self.new_d)
        self.off, self.seq, self.pos = bo.batch_plan(past, new, T)
        self.out = torch.full((N, H, d), 7.0, dtype=dtype, device="cuda")
        self.lse = torch.full((N, H), 7.0, device="cuda")

    def shared(self, ws=None, layer=0):
        if ws is None:
            ws = self.req.alloc_shared_workspace(self.batch)
        self.req.shared_attn(self.batch, layer, self.kc, self.vc, self.q, self.ks, self.vs, self.out,
                             self.lse, ws)
        return self.out, self.lse

    def blocks(self, block, lists, ws=None, layer=0):
        if ws is None:
            ws = self.req.alloc_block_workspace(self.batch, block, lists.shape[2])
        self.req.block_attn(self.batch, layer, self.kc, self.vc, block, lists, self.q, self.ks,
                            self.vs, self.out, self.lse, ws)
        return self.out, self.lse

    def reference(self, lists=None, block=None, layer=0):
        return bo.batch_attn(f64(self.q)[:self.n], self.seq, self.pos, f64(self.kc[layer]),
                             f64(self.vc[layer]), f64(self.ks), f64(self.vs), self.scale,
                             None if lists is None else lists.cpu().numpy(), block)

    def check(self, ref, what=""):
        """bf16: attn_tol.  float32: 1e-5 of the largest output, the bound of the float32 core's
        other tests.  lse: float32 logits (1e-4, times `sharp`) and sums, 5e-4 at least."""
        O, lse, spread = ref
        n = self.n
        got, got_l = f64(self.out), f64(self.lse)
        assert np.all(got[n:] == 7.0) and np.all(got_l[n:] == 7.0), f"{what}: rows behind the last"
        got, got_l = got[:n], got_l[:n]
        assert np.array_equal(np.isneginf(got_l), np.isneginf(lse)), what
        fin = np.isfinite(lse)
        assert np.all(np.isfinite(got)), what
        if fin.any():
            assert np.max(np.abs(got_l[fin] - lse[fin])) <= max(5e-4, 1e-4 * self.sharp), what
        if self.dtype == torch.bfloat16:
            tol = attn_tol(O, spread, self.sharp)
        else:
            tol = 1e-5 * max(1e-30, np.abs(O).max()) * np.ones_like(O)
        bad = np.abs(got - O) / tol
        assert bad.max(initial=0.0) <= 1.0, f"{what}: {bad.max():.2f} of the bound at {np.unravel_index(bad.argmax(), bad.shape)}"
