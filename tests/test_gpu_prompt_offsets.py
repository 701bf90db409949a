"""Offsets that go back and forth over the same rows: more work than the tensors have is refused on the device."""

from __future__ import annotations

import pytest
import torch

from test_gpu_prompt import dev, inputs
from test_gpu_prompt_grad import gradient_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
def test_offsets_back_and_forth_are_recorded(D):
    import paper_2605_29657_gb300 as occ
    from paper_2605_29657_gb300 import _lib as L
    n = 2048  # 8 blocks of 256 rows and 16 tiles of 128 keys a head; two sequences of them are more than 8 + 4 and 16 + 4 can hold
    q, k, v = inputs([n], None, 2, 2, D, torch.bfloat16)
    dout, whole, bad = gradient_of(q, torch.bfloat16), dev([0, n]), dev([0, n, 0, n, 0])
    ws = occ.alloc_prompt_workspace(n, 2)
    out, lse = occ.occam_prompt_attend(q, k, v, whole, ws)
    want = occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, whole, ws)
    to = torch.full_like(q, 7.0), torch.full_like(lse, 7.0)
    occ.occam_prompt_attend(q, k, v, bad, ws, out=to[0], lse=to[1])
    assert occ.occam_get_status(ws) == L.OCCAM_ERR_INVALID_ARG
    assert all(bool((x == 7.0).all()) for x in to)
    grads = [torch.full_like(x, 7.0) for x in (q, k, v)]
    occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, bad, ws, dq=grads[0], dk=grads[1], dv=grads[2])
    assert occ.occam_get_status(ws) == L.OCCAM_ERR_INVALID_ARG
    assert all(bool((x == 7.0).all()) for x in grads)
    # the workspace serves the next call
    again = occ.occam_prompt_attend(q, k, v, whole, ws)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    for x, y in zip(occ.occam_prompt_attend_grad(q, k, v, out, lse, dout, whole, ws), want):
        assert torch.equal(x, y)
    assert occ.occam_get_status(ws) == 0
