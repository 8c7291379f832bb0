"""Batched serving calls at the ends of their range: steps whose splits fill their launches,
against the float64 oracle."""

import pytest
import torch

from batch_harness import Step

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("T,H,H_kv,d,past,new", [
    (4096, 64, 8, 64, [0], [112]),                # 448 context items of four splits, a suffix item per tile
    (2830, 24, 2, 128, [5] * 15 + [0], [7] * 15 + [85]),
    (5000, 20, 2, 64, [1, 9, 0], [80, 90, 70]),
])
def test_every_split_of_a_step_is_run(gpu_lib, T, H, H_kv, d, past, new):
    """float32 steps of 286 to 448 context items, in a workspace that holds NaN: a split that no
    workgroup takes would show."""
    s = Step(past=past, new=new, T=T, H=H, H_kv=H_kv, d=d, dtype=F32, seed=21,
             room=max(p + n for p, n in zip(past, new)))
    ws = s.req.alloc_shared_workspace(s.batch)
    ws.view(torch.float32).fill_(float("nan"))
    s.shared(ws)
    s.check(s.reference())
