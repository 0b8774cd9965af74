"""Calls without a workspace: each has scratch of its own, whatever thread, stream or graph it runs on."""
import threading

import numpy as np
import pytest
import torch

from paper_1312_5853_amd import binding as hp

_empty = torch.empty


class _Library:
    """Stands in for the library: notes where a call's scratch lies, and lets `other` run before the first call returns."""

    def __init__(self, other):
        self.other, self.seen = other, []

    def bias_bwd_workspace_bytes(self, *a):
        return 4096

    fc_workspace_bytes = bias_bwd_workspace_bytes

    def _call(self, ws):
        self.seen.append(getattr(ws, "value", ws))
        if len(self.seen) == 1:
            self.other()
        return hp.OK

    def bias_bwd(self, *a):
        return self._call(a[-3])

    fc_bwd_filter = group_norm_act_bwd = distill_loss_fwd_bwd = bias_bwd


def _calls():
    dy, x = torch.zeros(2, 3, 4, 4), torch.zeros(2, 4, 3, 3)
    stat, lab = torch.zeros(2, 2), torch.zeros(2, dtype=torch.int64)
    return {"bias_bwd": lambda: hp.bias_bwd(dy), "fc_bwd_filter": lambda: hp.fc_bwd_filter(torch.zeros(2, 3), torch.zeros(2, 5)),
            "group_norm_act_bwd": lambda: hp.group_norm_act_bwd(x, x, stat, stat),
            "distill_loss_fwd_bwd": lambda: hp.distill_loss_fwd_bwd(torch.zeros(2, 9), labels=lab)}


@pytest.mark.parametrize("name", sorted(_calls()))
def test_calls_that_overlap_share_no_scratch(name, monkeypatch):
    """Another call, of any kind, between the moment a call has its scratch and the moment it has enqueued its work."""
    for other in _calls().values():
        lib = _Library(other)
        monkeypatch.setattr(hp, "lib", lambda lib=lib: lib)
        monkeypatch.setattr(hp, "_stream_handle", lambda stream: 0)
        monkeypatch.setattr(hp, "_current_stream", lambda *a: 0)
        monkeypatch.setattr(hp, "_on_gpu", lambda *a: None)
        monkeypatch.setattr(hp, "_norm_workspace_bytes", lambda *a: 4096)
        monkeypatch.setattr(hp, "_loss_workspace_bytes", lambda *a: 4096)
        monkeypatch.setattr(torch, "empty", lambda *a, **k: _empty(*a, **dict(k, device="cpu")))
        held = {}
        monkeypatch.setattr(hp, "_take_scratch", lambda n, stream: held.setdefault((t := _empty(n, dtype=torch.uint8)).data_ptr(), t).data_ptr())
        monkeypatch.setattr(hp, "_give_scratch", held.pop)
        _calls()[name]()
        first, second = lib.seen
        assert first and second and abs(first - second) >= 4096 and not held


def _norm_case(seed, N):
    """A backward pass in tiles: three launches that hand sums on through the scratch."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, dy = (torch.randn((N, 16, 160, 160), device="cuda", generator=g) for _ in range(2))
    _, mean, rstd = hp.group_norm_act_fwd(x, 2, ws=hp.Workspace())
    return lambda **kw: hp.group_norm_act_bwd(x, dy, mean, rstd, **kw)


def _loss_case(seed, N):
    """Loss and gradient of rows in parts."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn((N, 70001), device="cuda", generator=g)
    idx, val = torch.randint(0, 70001, (N, 20), device="cuda", generator=g), torch.randn((N, 20), device="cuda", generator=g)
    return lambda **kw: hp.distill_loss_fwd_bwd(z, top_idx=idx, top_val=val, temperature=2.0, **kw)


def _conv_case(seed, N):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, dy = (torch.randn((N, 64, 13, 13), device="cuda", generator=g) for _ in range(2))
    return lambda **kw: (hp.conv_bwd_filter(x, dy, 3, 3, 1, 1, **kw),)


CASES = [_norm_case, _loss_case, _conv_case]


@pytest.mark.gpu
@pytest.mark.parametrize("make", CASES)
@pytest.mark.parametrize("explicit", [False, True])
def test_two_streams_without_a_workspace(make, explicit):
    a, b = make(1, 6), make(2, 9)
    want = [f(ws=hp.Workspace()) for f in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for i, f in enumerate((a, b)):
            if explicit:
                got.append((i, f(stream=streams[i])))
            else:
                with torch.cuda.stream(streams[i]):
                    got.append((i, f()))
    torch.cuda.synchronize()
    for i, out in got:
        assert all(torch.equal(p, q) for p, q in zip(out, want[i]))


@pytest.mark.gpu
@pytest.mark.parametrize("make", CASES)
def test_two_threads_on_one_stream(make):
    calls = make(1, 6), make(2, 9)
    want = [f(ws=hp.Workspace()) for f in calls]
    torch.cuda.synchronize()
    got = [[], []]

    def work(i):
        for _ in range(20):
            got[i].append(calls[i]())

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(2):
        assert len(got[i]) == 20
        for out in got[i]:
            assert all(torch.equal(p, q) for p, q in zip(out, want[i]))


@pytest.mark.gpu
@pytest.mark.parametrize("make", CASES)
def test_a_graph_keeps_its_scratch(make):
    """A captured call without a workspace, larger calls and new tensors between its replays."""
    call, larger = make(1, 6), make(2, 40)
    want = call(ws=hp.Workspace())
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for _ in range(3):
        larger()
        fill = [torch.full((1 << 18,), float("nan"), device="cuda") for _ in range(20)]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))
        assert all(bool(torch.isnan(f).all()) for f in fill)
