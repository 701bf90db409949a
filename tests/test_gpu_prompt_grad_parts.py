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


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("off,koff", [([1000, 2000, 0, 1000], None), ([0, 700, 1 << 40, 700, 2000], None),
                                      ([1000, 2000, 0, 1000], [1100, 2200, 0, 1100]), ([0, 1000, 1000, 2000], [900, 1900, 0, 900])])
def test_grad_parts_beside_a_sequence_that_does_not_fit(off, koff, dtype):
    """Offsets that go back leave out their own sequence only: the others' divided gradients are those of a call without it."""
    import paper_2605_29657_gb300 as occ
    from paper_2605_29657_gb300 import _lib as L
    ko = off if koff is None else koff
    q, k, v = inputs([2000], [max(x for x in ko if x < 1 << 40)], 8, 1, 64, DT[dtype], 7, gain=0.8)
    dout, ws = gradient_of(q, DT[dtype], 7), occ.alloc_prompt_workspace(2000, 8, k.shape[0], 1)
    good = [i for i in range(len(off) - 1) if off[i] <= off[i + 1] <= 2000 and ko[i] <= ko[i + 1] <= k.shape[0]]
    assert 0 < len(good) < len(off) - 1
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    got, want = ([torch.full_like(x, 7.0) for x in (q, k, v)] for _ in range(2))
    kw = dict(out=out, lse=lse)
    occ.occam_prompt_attend(q, k, v, dev(off), ws, key_off=dev(ko), **kw)
    occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, dev(off), ws, key_off=dev(ko), dq=got[0], dk=got[1], dv=got[2])
    assert occ.occam_get_status(ws) == L.OCCAM_ERR_INVALID_ARG
    for i in good:
        a, b = dev([off[i], off[i + 1]]), dev([ko[i], ko[i + 1]])
        occ.occam_prompt_attend(q, k, v, a, ws, key_off=b, **kw)
        occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, a, ws, key_off=b, dq=want[0], dk=want[1], dv=want[2])
    assert occ.occam_get_status(ws) == 0
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_grad_of_many_rows_without_keys():
    """Nothing to divide."""
    q, k, v = inputs([3000], [0], 8, 1, 64, torch.bfloat16, 1)
    dq, dk, dv = check(q, k, v, gradient_of(q, torch.bfloat16), [0, 3000], [0, 0])
    assert not dq.any() and dk.shape[0] == dv.shape[0] == 0
