"""The gradient formulas that the prompt tests compare with, against differences of the attention itself (64 bits, CPU)."""

from __future__ import annotations

import pytest
import torch

import prompt_reference as P


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("off,koff", [([0, 5, 5, 12], None), ([1, 4, 9], [0, 7, 9])])
def test_formulas_against_differences(off, koff, causal):
    g = torch.Generator().manual_seed(1)
    rows, keys = off[-1] + 1, (koff or off)[-1]
    x = [torch.randn(s, generator=g, dtype=torch.float64).half() for s in ((rows, 4, 8), (keys, 2, 8), (keys, 2, 8))]
    dout = torch.randn((rows, 4, 8), generator=g, dtype=torch.float64).half()
    dout[:off[0]] = dout[off[-1]:] = 0
    grads = P.grad(*x, dout, off, koff, 0.3, causal)[:3]

    def loss(q, k, v):
        total = 0.0
        ko = koff or off
        for i in range(len(off) - 1):
            for h in range(4):
                Q, K, V = q[off[i]:off[i + 1], h], k[ko[i]:ko[i + 1], h // 2], v[ko[i]:ko[i + 1], h // 2]
                r, m = Q.shape[0], K.shape[0]
                if r == 0 or m == 0:
                    continue
                s = Q @ K.T * 0.3
                if causal:
                    s = s.masked_fill(~torch.ones((r, m), dtype=torch.bool).tril(m - r), -torch.inf)
                total = total + (torch.softmax(s, -1).nan_to_num(0.0) @ V * dout[off[i]:off[i + 1], h].double()).sum()
        return total

    step = 1e-5
    x = [y.double() for y in x]
    for n in range(3):
        d = torch.randn(x[n].shape, generator=g, dtype=torch.float64)
        hi, lo = ([y + s * d if i == n else y for i, y in enumerate(x)] for s in (step, -step))
        diff = (loss(*hi) - loss(*lo)) / (2 * step)
        assert abs(float(diff - (grads[n] * d).sum())) <= 1e-6 * float((grads[n] * d).abs().sum() + 1)
