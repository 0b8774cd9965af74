"""Layer norm, tensors in blocks and the passes on them as programs run them: on several streams and threads without a workspace,
in graphs, on long tensors, on the large tiles; run together."""
import threading

import numpy as np
import pytest
import torch

import oracle
from paper_1312_5853_amd import binding as hp

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _norm_case(seed, N):
    """A backward pass whose work-groups hand sums of columns on through the scratch."""
    g = _gen(seed)
    x, dy = (torch.randn((N * 200, 1000), device="cuda", generator=g) for _ in range(2))
    _, mean, rstd = hp.layer_norm_fwd(x)
    return lambda **kw: hp.layer_norm_bwd(x, dy, mean, rstd, **kw)


def _kept_norm_case(seed, N):
    g = _gen(seed)
    x, dy = (torch.randn((N * 200, 700), device="cuda", generator=g) for _ in range(2))
    _, mean, rstd = hp.layer_norm_fwd(x)
    q = hp.quantize_blocks(x, "e4m3")
    return lambda **kw: hp.layer_norm_bwd_kept(q, dy, mean, rstd, **kw)


def _grad_case(seed, N):
    """A sum in parts."""
    g = _gen(seed)
    q = hp.quantize_blocks(torch.randn((N * 300, 200), device="cuda", generator=g), "e4m3")
    dy = torch.randn((N * 300, 150), device="cuda", generator=g)
    return lambda **kw: (hp.fc_bwd_filter_kept(q, dy, **kw),)


def _few_case(seed, N):
    g = _gen(seed)
    w = hp.quantize_blocks(torch.randn((500, 1300), device="cuda", generator=g), "e2m1")
    x = torch.randn((N * 8, 1300), device="cuda", generator=g)
    return lambda **kw: (hp.fc_fwd_q4(x, w, **kw),)


def _tiles_case(seed, N):
    g = _gen(seed)
    w = hp.quantize_blocks(torch.randn((900, 600), device="cuda", generator=g), "e2m1")
    x = torch.randn((N * 300, 600), device="cuda", generator=g)
    return lambda **kw: (hp.fc_fwd_q4(x, w, **kw),)


CASES = [_norm_case, _kept_norm_case, _grad_case, _few_case, _tiles_case]


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


@pytest.mark.parametrize("make", CASES)
def test_a_graph_keeps_its_scratch(make):
    """A captured call without a workspace, larger calls and new tensors between its replays."""
    call, larger = make(1, 6), make(2, 20)
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


def test_two_graphs_with_a_workspace_each():
    """Both replayed in turn and over each other, on streams of their own."""
    a, b = _grad_case(1, 6), _tiles_case(2, 4)
    want = [f(ws=hp.Workspace())[0].clone() for f in (a, b)]
    graphs, outs, spaces = [], [], []
    for f in (a, b):
        ws = hp.Workspace()
        f(ws=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(f(ws=ws)[0])
        graphs.append(g)
        spaces.append(ws)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,I,O", [(1500, 1300, 700), (3500, 2100, 3600), (520, 2048, 1000), (33, 4500, 40)])
def test_forward_in_four_bits_in_tiles(N, I, O, dtype):
    """Sizes that the tiles of 128 and of 256 take, with an odd number of steps and ragged edges; and one of many steps for few
    samples.  Against exact products of the values held, summed in 64 bits."""
    g = _gen(N)
    x, w = torch.randn((N, I), device="cuda", generator=g).to(dtype), torch.randn((O, I), device="cuda", generator=g)
    bias = torch.randn((O,), device="cuda", generator=g)
    q = hp.quantize_blocks(w, "e2m1")
    xv, wv = hp.dequantize_blocks(hp.quantize_blocks(x, "e2m1")).double(), hp.dequantize_blocks(q).double()
    want, size = xv @ wv.t().contiguous() + bias.double(), xv.abs() @ wv.abs().t().contiguous() + bias.double().abs()
    got = hp.fc_fwd_q4(x, q, bias, out_bf16=dtype is torch.bfloat16)
    bound = 2 * U * (I + 64) * size
    if dtype is torch.bfloat16:                                      # rounded from a sum that is itself off
        bound = bound * (1 + 2.0 ** -8) + want.abs() * 2.0 ** -8
    assert ((got.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,I,O", [(1100, 3900, 4003), (1025, 4096, 4000), (300, 1100, 1003)])
def test_filter_gradient_in_tiles(N, I, O, dtype):
    """Sizes that the tiles of 256 take (and one for those of 128), rows that end inside a step, outputs that end inside a tile."""
    g = _gen(N)
    q = hp.quantize_blocks(torch.randn((N, I), device="cuda", generator=g), "e4m3")
    dy = torch.randn((N, O), device="cuda", generator=g).to(dtype)
    xv, d = hp.dequantize_blocks(q).double(), dy.double().t().contiguous()
    got = hp.fc_bwd_filter_kept(q, dy)
    n = N * (3 if dtype is torch.float32 else 1) + 64
    assert ((got.double() - d @ xv).abs() <= 2 * U * n * (d.abs() @ xv.abs())).all()


def test_rows_past_the_last_output_stay_out():
    """dy's last row has no next one: with 1003 outputs in tiles of 128 nothing is read past it, and NaN behind it stays there."""
    N, I, O = 192, 128, 1003
    buf = torch.full((N * O + 64,), float("nan"), device="cuda")
    dy = buf[:N * O].view(N, O)
    dy.fill_(1.0)
    q = hp.quantize_blocks(torch.ones((N, I), device="cuda"), "e4m3")
    assert (hp.fc_bwd_filter_kept(q, dy) == N).all()


def test_offsets_past_32_bits():
    """Rows beyond 2^31 values: as they are alone."""
    N, C = 140000, 16000                                             # 2.24e9 values
    x = torch.empty((N, C), dtype=torch.bfloat16, device="cuda")
    x[:-3].fill_(0.5)
    x[-3:] = torch.randn((3, C), device="cuda", generator=_gen(1)).bfloat16()
    q = hp.quantize_blocks(x, "e4m3")
    alone = hp.quantize_blocks(x[-3:], "e4m3")
    assert torch.equal(q.codes[-3:], alone.codes) and torch.equal(q.scales[-3:], alone.scales)
    y, mean, rstd = hp.layer_norm_fwd(x)
    few = hp.layer_norm_fwd(x[-3:])
    assert torch.equal(y[-3:], few[0]) and torch.equal(mean[-3:], few[1]) and torch.equal(rstd[-3:], few[2])
    back = hp.dequantize_blocks(q, x=y)
    assert torch.equal(back[-3:], hp.dequantize_blocks(alone, dtype=torch.bfloat16))
    dx, _, dbeta = hp.layer_norm_bwd_kept(q, x, mean, rstd, dx=y)
    assert torch.equal(dx[-3:], hp.layer_norm_bwd_kept(alone, x[-3:], few[1], few[2])[0])
    # N - 3 halves and three more: exact in 64 bits, rounded at the end
    want = (N - 3) * 0.5 + x[-3:].double().sum(0)
    assert ((dbeta.double() - want).abs() <= 300 * U * want).all()
    dx = hp.layer_norm_bwd(x, x, mean, rstd, dx=y)[0]
    assert torch.equal(dx[-3:], hp.layer_norm_bwd(x[-3:], x[-3:], few[1], few[2])[0])


@pytest.mark.parametrize("C", [1 << 27, (1 << 27) - 5])
def test_layer_norm_of_the_longest_rows(C):
    """One row of ones and minus ones in turn (an odd number of values has one more of the ones), whose mean and squares are exact."""
    x = torch.ones((1, C), device="cuda")
    x[0, 1::2] = -1.0
    dy = (torch.arange(C, device="cuda", dtype=torch.int32) % 7 - 3).float().view(1, C)
    gamma = torch.full((C,), 2.0, device="cuda")
    y, mean, rstd = hp.layer_norm_fwd(x, gamma, eps=1e-5)
    m, r = float(mean), float(rstd)
    assert abs(m - C % 2 / C) <= 64 * U * (1 + C % 2 / C) and abs(r - (1 + 1e-5 - (C % 2 / C) ** 2) ** -0.5) <= 64 * U
    xh = (x.double() - m) * r
    assert ((y.double() - 2 * xh).abs() <= 2 * 8 * U).all()
    dx, dgamma, dbeta = hp.layer_norm_bwd(x, dy, mean, rstd, gamma)
    assert torch.equal(dbeta, dy[0]) and ((dgamma.double() - (dy * xh)[0]).abs() <= 4 * 3 * U).all()
    g = 2.0 * dy.double()
    want = r * (g - g.mean() - xh * (g * xh).mean())
    assert ((dx.double() - want).abs() <= (8 * 6 + 64 * 12) * U).all()


def test_filters_and_samples_past_32_bits_of_bytes():
    """Outputs of 2^31 bytes and more."""
    N, I, O = 40000, 64, 16000                                       # y: 2.56e9 bytes
    x, w = torch.randn((N, I), device="cuda", generator=_gen(2)), torch.randn((O, I), device="cuda", generator=_gen(3))
    q = hp.quantize_blocks(w, "e2m1")
    y = hp.fc_fwd_q4(x, q)
    xv, wv = hp.dequantize_blocks(hp.quantize_blocks(x[-5:].contiguous(), "e2m1")).double(), hp.dequantize_blocks(q).double()
    size = xv.abs() @ wv.abs().t().contiguous()
    assert ((y[-5:].double() - xv @ wv.t().contiguous()).abs() <= 2 * U * (I + 64) * size).all()
    kept = hp.quantize_blocks(torch.ones((3, O), device="cuda"), "e4m3")
    dw = hp.fc_bwd_filter_kept(kept, y[:3, :40000].contiguous().new_ones((3, N)))         # [N, O]: as large
    assert dw.shape == (N, O) and (dw[-1] == 3).all() and (dw[0] == 3).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,I,O", [(1, 1, (1 << 31) - 1), (1, (1 << 31) - 128, 1), (0, (1 << 31) - 1, 1), (0, 1, (1 << 31) - 1)])
def test_filter_gradient_of_the_longest_tensors(N, I, O, dtype):
    """Just below 2^31 elements: products of single values, exact."""
    q = hp.Blocks.empty(N, I, "e4m3")
    q.codes.fill_(0x38)                                              # 1, times powers of two in turn
    q.scales.copy_(127 + torch.arange(q.scales.numel(), device="cuda", dtype=torch.int32).view(q.scales.shape) % 13)
    dy = (torch.arange(O, device="cuda", dtype=torch.int32) % 251 - 125).to(dtype).view(1, O)[:N]
    dw = torch.full((O, I), float("nan"), device="cuda")
    hp.fc_bwd_filter_kept(q, dy, dw=dw)
    if N == 0:
        assert not dw.any()
    elif I == 1:
        assert torch.equal(dw.view(-1), dy.view(-1).float())
    else:
        assert torch.equal(dw.view(-1, 32), (q.scales.float() - 127).exp2().mul_(-125.0).view(-1, 1)[:I // 32].expand(-1, 32))


def test_run_together():
    """A layer as it is trained and then served: normalised, kept, its gradients, its output in 4 bits; odd sizes, one stream."""
    N, I, O = 77, 1003, 515
    rng = np.random.Generator(np.random.Philox(4))
    a = np.maximum(rng.standard_normal((N, I)), 0).astype(np.float32)
    w, gamma, beta = (0.05 * rng.standard_normal((O, I))).astype(np.float32), (1 + 0.1 * rng.standard_normal(I)).astype(np.float32), np.zeros(I, np.float32)
    dy = rng.standard_normal((N, O)).astype(np.float32)
    cuda = lambda v: torch.from_numpy(v).cuda()
    s = torch.cuda.Stream()
    at, wt, gt, bt, dt = map(cuda, (a, w, gamma, beta, dy))
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        h, mean, rstd = hp.layer_norm_fwd(at, gt, bt)
        qa, qh, qw = hp.quantize_blocks(at, "e4m3"), hp.quantize_blocks(h, "e4m3"), hp.quantize_blocks(wt, "e2m1")
        dw = hp.fc_bwd_filter_kept(qh, dt)
        dh = torch.matmul(dt, wt)
        da, dgamma, dbeta = hp.layer_norm_bwd_kept(qa, dh, mean, rstd, gt)
        y = hp.fc_fwd_q4(h, qw)
    s.synchronize()
    host = lambda t: t.double().cpu().numpy()
    values = lambda q: oracle.dequantize_blocks(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.cols, q.format)
    near = lambda got, want: np.abs(host(got) - want).max() <= 1e-5 * np.abs(want).max()
    assert near(h, oracle.layer_norm_fwd(a, gamma, beta, 1e-5)[0])
    assert np.array_equal(values(qa), oracle.dequantize_blocks(*oracle.quantize_blocks(a, "e4m3"), I, "e4m3"))
    assert near(dw, dy.astype(np.float64).T @ values(qh))
    want = oracle.layer_norm_bwd(values(qa), host(dh), host(mean), host(rstd), gamma)
    assert near(da, want[0]) and near(dgamma, want[1]) and near(dbeta, want[2])
    x4 = oracle.dequantize_blocks(*oracle.quantize_blocks(host(h), "e2m1"), I, "e2m1")
    assert near(y, x4 @ values(qw).T)
