"""Which device, stream and workspace a call of whole-prompt attention, its gradient, append with the rotation and attention over
shared pages goes to, without a GPU: as for the other cache calls."""

from __future__ import annotations

import pytest
import torch

from test_cache_devices_cpu import I32, I64, U8, cache, env  # noqa: F401  (env: the fixture)

B16, F32 = torch.bfloat16, torch.float32


@pytest.fixture
def calls(env, monkeypatch):  # noqa: F811
    from paper_2605_29657_gb300 import _cache, _prompt
    monkeypatch.setattr(_prompt, "library", _cache.library)
    return env


def tensors(device, other=None, where=None):
    shapes = dict(seqs=((2,), I32), group_off=((2,), I32), row_off=((3,), I64), key_off=((3,), I64), k=((4, 2, 64), B16), v=((4, 2, 64), B16),
                  q=((4, 4, 64), B16), out=((4, 4, 64), B16), lse=((4, 4), F32), dout=((4, 4, 64), B16), dq=((4, 4, 64), B16),
                  dk=((4, 2, 64), B16), dv=((4, 2, 64), B16), positions=((3, 4), I32), inv_freq=((32,), F32), axis=((32,), I32),
                  out_q=((4, 4, 64), B16), ws=((1 << 20,), U8))
    return {n: torch.empty(s, dtype=d, device=other if n == where else device) for n, (s, d) in shapes.items()}


CALLS = {
    "prompt_attend": (lambda o, c, t: o.occam_prompt_attend(t["q"], t["k"], t["v"], t["row_off"], t["ws"], key_off=t["key_off"], out=t["out"],
                                                            lse=t["lse"]), "k v row_off ws key_off out lse"),
    "prompt_attend_grad": (lambda o, c, t: o.occam_prompt_attend_grad(t["q"], t["k"], t["v"], t["out"], t["lse"], t["dout"], t["row_off"],
                                                                      t["ws"], key_off=t["key_off"], dq=t["dq"], dk=t["dk"], dv=t["dv"]),
                           "k v out lse dout row_off ws key_off dq dk dv"),
    "cache_append_rope": (lambda o, c, t: o.occam_cache_append_rope(c, 0, t["q"], t["k"], t["v"], t["seqs"], t["row_off"], t["positions"],
                                                                    t["inv_freq"], t["axis"], out_q=t["out_q"], ws=t["ws"]),
                          "q k v seqs row_off positions inv_freq axis out_q ws"),
    "cache_attend_shared": (lambda o, c, t: o.occam_cache_attend_shared(c, 0, t["q"], t["seqs"], t["row_off"], 2, t["group_off"], 4, t["ws"],
                                                                        out=t["out"], lse=t["lse"]), "q seqs row_off group_off ws out lse"),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_call_runs_on_the_device_of_its_tensors(calls, name):
    occ, reached = calls
    for n, device in enumerate(("cuda:0", "cuda:1")):
        CALLS[name][0](occ, cache(occ, device), tensors(device))
        assert reached[n:] == [("occam_" + name, n)]
    assert torch._C._cuda_getDevice() == 0


@pytest.mark.parametrize("name,where", [(n, w) for n, (_, ws) in CALLS.items() for w in ws.split()])
def test_a_tensor_of_another_device_is_refused(calls, name, where):
    occ, reached = calls
    for other in ("cuda:0", "cpu"):
        with pytest.raises(occ.OccamError):
            CALLS[name][0](occ, cache(occ, "cuda:1"), tensors("cuda:1", other, where))
    assert not reached


@pytest.mark.parametrize("name", CALLS)
def test_shapes_and_types_that_are_refused(calls, name):
    occ, reached = calls
    call, names = CALLS[name]
    for where in names.split():
        t = tensors("cuda:0")
        was = t[where]
        wrong = [torch.empty(was.shape, dtype=torch.float64, device="cuda:0"), None if where != "key_off" else 3]
        if where != "ws":  # (a workspace's size is the library's to check)
            wrong += [torch.empty((*was.shape, 2), dtype=was.dtype, device="cuda:0"),
                      torch.empty((*was.shape[:-1], 2 * was.shape[-1]), dtype=was.dtype, device="cuda:0")[..., ::2]]
        if where in ("out", "lse", "dq", "dk", "dv", "out_q", "q") or (where == "ws" and "cache" in name):
            del wrong[1]  # (new tensors then, or no queries, or the cache's own)
        for bad in wrong:
            t[where] = bad
            with pytest.raises(occ.OccamError):
                call(occ, cache(occ, "cuda:0"), t)
    assert not reached


def test_results_without_given_tensors_are_new_ones_like_the_inputs(calls):
    occ, reached = calls
    t, c = tensors("cuda:1"), cache(occ, "cuda:1")
    out, lse = occ.occam_prompt_attend(t["q"], t["k"], t["v"], t["row_off"], t["ws"])
    assert out.shape == t["q"].shape and out.dtype == B16 and lse.shape == (4, 4) and lse.dtype == F32 and out.device == t["q"].device
    got = occ.occam_prompt_attend_grad(t["q"], t["k"], t["v"], t["out"], t["lse"], t["dout"], t["row_off"], t["ws"])
    assert [x.shape for x in got] == [t["q"].shape, t["k"].shape, t["v"].shape] and all(x.device == t["q"].device for x in got)
    q = occ.occam_cache_append_rope(c, 0, t["q"], t["k"], t["v"], t["seqs"], t["row_off"], t["positions"], t["inv_freq"], t["axis"], ws=t["ws"])
    assert q.shape == t["q"].shape
    assert occ.occam_cache_append_rope(c, 0, None, t["k"], t["v"], t["seqs"], t["row_off"], t["positions"], t["inv_freq"], t["axis"],
                                       ws=t["ws"]) is None
    out, lse = occ.occam_cache_attend_shared(c, 0, t["q"], t["seqs"], t["row_off"], 2, t["group_off"], 4, t["ws"])
    assert out.shape == t["q"].shape and lse.shape == (4, 4)
    assert len(reached) == 5


def test_other_arguments_that_are_refused(calls):
    occ, reached = calls
    t, c = tensors("cuda:0"), cache(occ, "cuda:0")

    class Stream:
        device, cuda_stream = torch.device("cuda:1"), 7

    prompt = lambda **kw: occ.occam_prompt_attend(t["q"], t["k"], t["v"], t["row_off"], t["ws"], **kw)
    grad = lambda **kw: occ.occam_prompt_attend_grad(t["q"], t["k"], t["v"], t["out"], t["lse"], t["dout"], t["row_off"], t["ws"], **kw)
    enter = lambda **kw: occ.occam_cache_append_rope(c, 0, kw.pop("q", t["q"]), t["k"], t["v"], t["seqs"], t["row_off"], t["positions"],
                                                     t["inv_freq"], t["axis"], ws=t["ws"], **kw)
    shared = lambda most=4, rows=2, **kw: occ.occam_cache_attend_shared(c, 0, t["q"], t["seqs"], t["row_off"], rows, t["group_off"], most,
                                                                         t["ws"], **kw)
    for call in (prompt, grad, enter, shared):
        with pytest.raises(occ.OccamError):
            call(stream=Stream)
    for call, kw in ((prompt, dict(scale="x")), (grad, dict(scale="x")), (enter, dict(pairing="odd")), (enter, dict(q=None, out_q=t["out_q"])),
                     (shared, dict(scale="x")), (shared, dict(rows="x"))):
        with pytest.raises(occ.OccamError):
            call(**kw)
    with pytest.raises(occ.OccamError):
        occ.occam_prompt_attend(t["q"].cpu(), t["k"], t["v"], t["row_off"], t["ws"])
    assert not reached
