"""Which device, stream and workspace a call of the cache binding goes to, without a GPU: tensors of
two devices that hold no memory, and a library that records what reaches it."""

from __future__ import annotations

import contextlib

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

I32, I64, U8 = torch.int32, torch.int64, torch.uint8


@pytest.fixture
def env(monkeypatch):
    import paper_2605_29657_gb300 as occ
    from paper_2605_29657_gb300 import _cache

    reached, current = [], [0]

    class Library:
        def __getattr__(self, name):
            def call(*args):
                reached.append((name, current[0]))
                return 0
            call.__name__ = name
            return call

    @contextlib.contextmanager
    def device(index):
        was, current[0] = current[0], index
        yield
        current[0] = was

    monkeypatch.setattr(_cache, "library", lambda lib=Library(): lib)
    monkeypatch.setattr(_cache, "_ptr", lambda t: None if t is None else 4096)
    monkeypatch.setattr(torch.Tensor, "data_ptr", lambda t: 4096)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0)
    monkeypatch.setattr(torch.cuda, "device", device)
    with FakeTensorMode():
        yield occ, reached


def tensors(device, other=None, where=None):
    """A call's tensors by name, on `device`; the one named `where` on `other`."""
    shapes = dict(seqs=((2,), I32), counts=((2,), I32), dst=((2,), I32), row_off=((3,), I64), keep=((9,), U8), keep_off=((3,), I64),
                  k=((4, 2, 64), torch.bfloat16), v=((4, 2, 64), torch.bfloat16), q=((4, 4, 64), torch.bfloat16),
                  out=((4, 4, 64), torch.bfloat16), lse=((4, 4), torch.float32), positions=((3, 4), I32),
                  inv_freq=((32,), torch.float32), axis=((32,), I32), out_q=((4, 4, 64), torch.bfloat16),
                  out_k=((4, 2, 64), torch.bfloat16), ws=((1 << 20,), U8))
    return {n: torch.empty(s, dtype=d, device=other if n == where else device) for n, (s, d) in shapes.items()}


def cache(occ, device):
    c = occ.PagedCache.__new__(occ.PagedCache)
    c.device, c.heads, c.dim, c.layers = torch.device(device), 2, 64, 1
    c.at = c.device.index
    c._ref, c._ws = None, (256, 1 << 20)
    return c


CALLS = {
    "extend": (lambda o, c, t: o.occam_cache_extend(c, t["seqs"], t["counts"], ws=t["ws"]), "seqs counts ws"),
    "append": (lambda o, c, t: o.occam_cache_append(c, 0, t["k"], t["v"], t["seqs"], t["row_off"], ws=t["ws"]), "k v seqs row_off ws"),
    "attend": (lambda o, c, t: o.occam_cache_attend(c, 0, t["q"], t["seqs"], t["row_off"], 2, keep=t["keep"], keep_off=t["keep_off"],
                                                    out=t["out"], lse=t["lse"], ws=t["ws"]),
               "q seqs row_off keep keep_off out lse ws"),
    "fork": (lambda o, c, t: o.occam_cache_fork(c, t["seqs"], t["dst"], ws=t["ws"]), "seqs dst ws"),
    "compact": (lambda o, c, t: o.occam_cache_compact(c, t["seqs"], t["keep"], t["keep_off"], ws=t["ws"]), "seqs keep keep_off ws"),
    "release": (lambda o, c, t: o.occam_cache_release(c, t["seqs"], ws=t["ws"]), "seqs ws"),
    "get_status": (lambda o, c, t: c.status(ws=t["ws"]), "ws"),
    "rope": (lambda o, c, t: o.occam_rope(t["q"], t["k"], t["positions"], t["inv_freq"], t["axis"], out_q=t["out_q"], out_k=t["out_k"]),
             "k positions inv_freq axis out_q out_k"),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_call_runs_on_the_device_of_its_tensors(env, name):
    occ, reached = env
    for n, device in enumerate(("cuda:0", "cuda:1")):
        CALLS[name][0](occ, cache(occ, device), tensors(device))
        assert len(reached) == n + 1 and reached[n][0].endswith(name) and reached[n][1] == n
    assert torch._C._cuda_getDevice() == 0


@pytest.mark.parametrize("name,where", [(n, w) for n, (_, ws) in CALLS.items() for w in ws.split()])
def test_a_tensor_of_another_device_is_refused(env, name, where):
    occ, reached = env
    for other in ("cuda:0", "cpu"):
        with pytest.raises(occ.OccamError):
            CALLS[name][0](occ, cache(occ, "cuda:1"), tensors("cuda:1", other, where))
    assert not reached


def test_workspaces_and_streams_that_are_refused(env):
    occ, reached = env
    t, c = tensors("cuda:0"), cache(occ, "cuda:0")

    class Stream:
        device, cuda_stream = torch.device("cuda:1"), 7

    for ws in (t["counts"], torch.empty((256, 256), dtype=U8, device="cuda:0").T, 4096, t["k"]):
        with pytest.raises(occ.OccamError):
            occ.occam_cache_extend(c, t["seqs"], t["counts"], ws=ws)
    with pytest.raises(occ.OccamError):
        occ.occam_cache_extend(c, t["seqs"], t["counts"], stream=Stream)
    with pytest.raises(occ.OccamError):
        occ.occam_rope(t["q"], None, t["positions"], t["inv_freq"], t["axis"], stream=Stream)
    assert not reached
    Stream.device = torch.device("cuda:0")
    occ.occam_cache_extend(c, t["seqs"], t["counts"], stream=Stream)
    assert reached == [("occam_cache_extend", 0)]


def test_a_cache_over_tensors_of_two_devices_is_refused(env):
    occ, reached = env
    names = dict(k=((1, 4, 2, 16, 64), torch.float8_e4m3fn), v=((1, 4, 2, 16, 64), torch.float8_e4m3fn),
                 k_scale=((1, 4, 2), torch.float32), v_scale=((1, 4, 2), torch.float32), table=((3, 2), I32), length=((3,), I32),
                 refs=((4,), I32))
    for where in names:
        with pytest.raises(occ.OccamError):
            occ.PagedCache.wrap(**{n: torch.empty(s, dtype=d, device="cuda:1" if n == where else "cuda:0") for n, (s, d) in names.items()})
    assert not reached
