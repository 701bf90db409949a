"""Gradients with few key heads and long sequences, whose tiles of keys are divided among CTAs and added up: against the
formulas, and the same every time."""

from __future__ import annotations

import pytest
import torch

from test_gpu_prompt import DT, dev, inputs, offs
from test_gpu_prompt_grad import check, gradient_of

pytestmark = pytest.mark.gpu

# rows, keys (None: the same), heads, key heads, dims
PARTS = [
    ([1000], None, 8, 1, 128), ([300, 5, 0, 700, 64], None, 12, 2, 64), ([1100], None, 5, 1, 72), ([900, 40], [1100, 700], 8, 1, 128),
    ([513], [130], 28, 4, 64), ([2100], None, 3, 3, 80), ([200, 200, 1, 1500], None, 6, 2, 8), ([640], None, 64, 1, 120),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", range(len(PARTS)))
def test_grad_of_few_key_heads(n, dtype):
    import paper_2605_29657_gb300 as occ
    rows, keys, H, Hkv, D = PARTS[n]
    q, k, v = inputs(rows, keys, H, Hkv, D, DT[dtype], n, gain=0.8, first=2, behind=1)
    dout = gradient_of(q, DT[dtype], n)
    off, koff = offs(rows, 2), None if keys is None else offs(keys, 2)
    got = check(q, k, v, dout, off, koff, where="causal")
    check(q, k, v, dout, off, koff, scale=0.2, causal=False, where="full")
    # a workspace for larger calls serves, whatever an earlier one left in it
    ws = occ.alloc_prompt_workspace(q.shape[0] + 5000, H, k.shape[0] + 5000, Hkv)
    ws[256:] = 0xff
    kw = dict(key_off=None if koff is None else dev(koff))
    out, lse = occ.occam_prompt_attend(q, k, v, dev(off), ws, **kw)
    for _ in range(3):
        new = occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, dev(off), ws, **kw)
        for i, (x, y) in enumerate(zip(new, got)):
            o = off if i == 0 or koff is None else koff
            assert torch.equal(x[o[0]:o[-1]], y[o[0]:o[-1]])
    assert occ.occam_get_status(ws) == 0
