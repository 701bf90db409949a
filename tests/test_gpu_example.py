"""The example that runs the rotary and cache operators together: its
attention calls against the plain implementation, its pages, its branches."""

from __future__ import annotations

import importlib.util
import os

import pytest
import torch

from tests import cache_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "prune_and_answer.py")
    spec = importlib.util.spec_from_file_location("prune_and_answer", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_second_question_on_a_pruned_branch(example):
    calls = []

    class Checked(example.Decoder):
        def attend(self, layer, q, seqs, row_off, max_rows):
            out = super().attend(layer, q, seqs, row_off, max_rows)
            off = row_off.tolist()
            n = off[-1]  # (the rows past the kept ones belong to no sequence)
            want, _, tol, _ = R.Cache(self.cache).attend(layer, q[:n], seqs.tolist(), off)
            u = R.UNIT[out.dtype]
            over = (out[:n].double().cpu() - want).abs() - (u * want.abs() + R.TINY[out.dtype] + (1 + u) * tol)
            calls.append(float(over.max()))
            return out

    r = example.run(images=3, steps=3, decoder_type=Checked)
    assert r["status"] == 0
    assert len(calls) == example.LAYERS * (1 + 2 * 3) and max(calls) <= 0, calls
    for rows, one, two in zip(r["rows"], *r["prefix"]):
        assert 0 < two <= one <= rows
    assert sum(r["prefix"][1]) < sum(r["prefix"][0]) < sum(r["rows"])
    c = r["cache"]
    assert not c.refs.any() and not c.length.any() and bool((c.table == -1).all())


def test_a_branch_that_keeps_all_answers_the_same(example):
    r = example.run(stricter=0)
    assert r["status"] == 0 and r["prefix"][0] == r["prefix"][1]
    assert r["answers"][0] == r["answers"][1]
    assert torch.equal(*r["logits"])
