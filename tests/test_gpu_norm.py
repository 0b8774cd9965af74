"""Group normalisation with an activation on the GPU against the oracle in 64 bits, element by element.

The bounds: u = 2^-24 is one fp32 rounding.  A sum of M fp32 values is taken in chains of at most a few hundred joined in
trees, so its error is below 64 u of the sum of magnitudes; everything else is a handful of roundings.  A result stored as
bfloat16 adds 2^-8 of itself."""
import numpy as np
import pytest
import torch

import oracle
from paper_1312_5853_amd import binding as hp

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SUM = 64 * U


def _tensors(N, C, H, W, layout, dtype, seed, mean=0.0, std=1.0):
    """x and dy as [N,C,S] float64 holding values of the type, and on the GPU as [N,C,H,W] in the layout."""
    g = np.random.Generator(np.random.Philox(seed))
    host, dev = [], []
    for off, s in ((mean, std), (0.0, 1.0)):
        a = (off + s * g.standard_normal((N, C, H * W)) * (0.5 + g.random((1, C, 1)))).astype(np.float32)
        if dtype == "bf16":
            a = oracle.bf16_round(a)
        host.append(a.astype(np.float64))
        dev.append(_dev(a.reshape(N, C, H, W), layout, dtype))
    gamma, beta = (1.0 + 0.3 * g.standard_normal(C)).astype(np.float32), (0.3 * g.standard_normal(C)).astype(np.float32)
    return host, dev, gamma, beta


def _dev(a, layout, dtype):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    if dtype == "bf16":
        t = t.to(torch.bfloat16)
    return t.contiguous(memory_format=torch.channels_last) if layout == "last" else t


def _cuda(v):
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).cuda()


def _host(t, shape=None):
    a = t.float().cpu().numpy().astype(np.float64)
    return a.reshape(shape) if shape else a


def _per_channel(v, C):
    return np.repeat(v, C // v.shape[1], axis=1)[:, :, None]


def _group_mean(v, G):
    return v.reshape(v.shape[0], G, -1).mean(2)


def _store(v, dtype):
    return np.abs(v) * (2.0 ** -8 if dtype == "bf16" else 2 * U)


def check_fwd(got, x, G, gamma, beta, eps, act, dtype):
    y, mean, rstd = got
    N, C, S = x.shape
    want, wm, wr = oracle.group_norm_act_fwd(x, G, gamma, beta, eps, act)
    big = _group_mean(np.abs(x), G)
    e_mean = SUM * big + 2 * U * np.abs(wm)
    # a mean off by e changes the variance by e^2 at most; its own sum and the deviations' rounding are relative errors
    var = 1.0 / wr ** 2
    e_var = (e_mean ** 2 + SUM * var + 4 * U * np.sqrt(var) * (big + np.abs(wm)))
    e_rstd = wr * (e_var / var / 2 + 4 * U)
    assert (np.abs(_host(mean) - wm) <= e_mean).all()
    assert (np.abs(_host(rstd) - wr) <= e_rstd).all()
    d = x - _per_channel(wm, C)
    g = np.abs(gamma)[None, :, None]
    e_z = g * (_per_channel(wr, C) * (_per_channel(e_mean, C) + 2 * U * np.abs(x)) + np.abs(d) * _per_channel(e_rstd, C))
    z = np.abs(d) * _per_channel(wr, C) * g + np.abs(beta)[None, :, None]
    e_y = 1.2 * e_z + 16 * U * z + _store(want, dtype)               # slopes of the activations are below 1.1
    err = np.abs(_host(y, x.shape) - want)
    assert (err <= e_y + 1e-37).all(), (err / (e_y + 1e-37)).max()


def check_bwd(got, x, dy, mean, rstd, gamma, beta, act, dtype):
    dx, dgamma, dbeta = got
    N, C, S = x.shape
    G = mean.shape[1]
    wx, wg, wb = oracle.group_norm_act_bwd(x, dy, mean, rstd, gamma, beta, act)
    r, m = _per_channel(rstd, C), _per_channel(mean, C)
    xh = (x - m) * r
    ga, be = gamma[None, :, None].astype(np.float64), beta[None, :, None].astype(np.float64)
    z = ga * xh + be
    e_xh = 2 * U * np.abs(xh)
    e_z = np.abs(ga) * e_xh + 2 * U * (np.abs(ga * xh) + np.abs(be))
    if act == "silu":
        e_dz = np.abs(dy) * (0.5 * e_z + 24 * U * (1.0 + np.abs(z)))
    else:
        e_dz = np.abs(dy) * 2 * U
    one = oracle.group_norm_act_bwd(x, dy, mean, rstd, np.ones(C), np.zeros(C), "none")      # (shapes only)
    assert one[0].shape == wx.shape
    slope = {"none": lambda: 1.0, "relu": lambda: (z > 0) * 1.0,
             "silu": lambda: oracle.oracle._sigmoid(z) * (1 + z * (1 - oracle.oracle._sigmoid(z)))}[act]()
    dz = dy * slope
    e_dzxh = e_dz * np.abs(xh) + np.abs(dz) * e_xh
    assert (np.abs(_host(dbeta) - wb) <= SUM * np.abs(dz).sum((0, 2)) + e_dz.sum((0, 2)) + 1e-37).all()
    assert (np.abs(_host(dgamma) - wg) <= SUM * np.abs(dz * xh).sum((0, 2)) + e_dzxh.sum((0, 2)) + 1e-37).all()
    a1, a2 = _group_mean(np.abs(ga * dz), G), _group_mean(np.abs(ga * dz * xh), G)
    e1 = SUM * a1 + _group_mean(np.abs(ga) * e_dz, G)
    e2 = SUM * a2 + _group_mean(np.abs(ga) * e_dzxh, G)
    pc = lambda v: _per_channel(v, C)
    e = r * (np.abs(ga) * e_dz + pc(e1) + np.abs(xh) * pc(e2) + e_xh * pc(a2)
             + 8 * U * (np.abs(ga * dz) + pc(a1) + np.abs(xh) * pc(a2))) + _store(wx, dtype)
    err = np.abs(_host(dx, x.shape) - wx)
    assert (err <= e + 1e-37).all(), (err / (e + 1e-37)).max()


def run_case(N, C, H, W, G, act, layout, dtype, seed=0, mean=0.0, std=1.0, eps=1e-5, affine=True):
    (x, dy), (xd, dyd), gamma, beta = _tensors(N, C, H, W, layout, dtype, seed, mean, std)
    if not affine:
        gamma, beta = np.ones(C, np.float32), np.zeros(C, np.float32)
    ga, be = (_cuda(gamma), _cuda(beta)) if affine else (None, None)
    y = torch.full_like(xd, float("nan"))
    got = hp.group_norm_act_fwd(xd, G, ga, be, eps=eps, act=act, y=y)
    check_fwd(got, x, G, gamma, beta, eps, act, dtype)
    m, r = (v.astype(np.float32).astype(np.float64) for v in oracle.group_norm_stats(x, G, eps))
    if act == "relu":
        # no gradient where rounding decides the sign of the activation's argument
        z = (x - _per_channel(m, C)) * _per_channel(r, C) * gamma[None, :, None] + beta[None, :, None]
        near = np.abs(z) < 1e-4 * (1 + np.abs(_per_channel(m, C)) * _per_channel(r, C))
        dy[near] = 0.0
        dyd = _dev(dy.reshape(N, C, H, W), layout, dtype)
    dx = torch.full_like(xd, float("nan"))
    got = hp.group_norm_act_bwd(xd, dyd, _cuda(m), _cuda(r), ga, be, act=act, dx=dx)
    check_bwd(got, x, dy, m, r, gamma, beta, act, dtype)


# N, C, H, W, groups: groups of one channel and of all, planes of one position and of a few, planes that fill no vector, a
# wavefront's worth and one more, the network's layers, a group larger than a work-group keeps
SHAPES = [
    (1, 1, 1, 1, 1), (2, 4, 1, 1, 2), (3, 32, 1, 1, 32), (2, 1030, 1, 1, 2), (5, 6, 1, 2, 3), (2, 6, 1, 3, 1),
    (2, 12, 2, 2, 4), (1, 7, 5, 1, 7), (2, 10, 1, 7, 5), (3, 24, 3, 3, 8), (2, 48, 4, 4, 3), (2, 40, 1, 17, 4), (1, 200, 6, 6, 2),
    (2, 6, 15, 17, 2), (2, 6, 16, 16, 2), (2, 6, 1, 257, 2), (3, 384, 13, 13, 32), (2, 256, 27, 27, 32),
    (2, 96, 55, 55, 32), (1, 33, 31, 45, 3), (2, 72, 31, 45, 8), (1, 62, 19, 23, 31), (1, 16, 64, 64, 1), (1, 5, 120, 130, 1),
    (1, 64, 112, 113, 2), (2, 2, 224, 224, 1), (1, 1, 401, 399, 1), (2, 9001, 1, 2, 1), (1, 4100, 3, 3, 1), (2, 16500, 1, 1, 2),
    (3, 3, 20, 30, 1), (2, 3, 200, 300, 3),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_the_oracle(shape, layout, dtype):
    N, C, H, W, G = shape
    act = ("none", "relu", "silu")[(C + H) % 3]
    run_case(N, C, H, W, G, act, layout, dtype, seed=C * H + W)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_activations(act, layout, dtype):
    run_case(2, 24, 9, 11, 4, act, layout, dtype, seed=5)


@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("mean,std", [(1e4, 1.0), (-300.0, 1e-2), (1e-20, 1e-20), (1e15, 1e13), (2.0, 0.0)])
def test_means_far_from_zero_and_extreme_scales(mean, std, layout):
    """The variance comes from distances to the mean: values of 10000 +- 1 keep it."""
    run_case(2, 12, 10, 13, 3, "silu", layout, "f32", seed=6, mean=mean, std=std)


@pytest.mark.parametrize("layout", ["planes", "last"])
def test_without_scale_and_shift(layout):
    run_case(2, 12, 7, 9, 3, "relu", layout, "f32", seed=7, affine=False)


@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_value_that_is_no_number_stays_in_its_group(bad, layout, dtype):
    (x, _), (xd, dyd), gamma, beta = _tensors(2, 12, 9, 9, layout, dtype, 8)
    ga, be = _cuda(gamma), _cuda(beta)
    want = hp.group_norm_act_fwd(xd, 4, ga, be, act="silu")
    back = hp.group_norm_act_bwd(xd, dyd, want[1], want[2], ga, be, act="silu")
    xb = xd.clone(memory_format=torch.preserve_format)
    xb[1, 4, 3, 3] = bad                                             # sample 1, group 1
    got = hp.group_norm_act_fwd(xb, 4, ga, be, act="silu")
    here = torch.zeros(2, 12, 9, 9, dtype=torch.bool)
    here[1, 3:6] = True
    assert torch.isnan(got[0].float().cpu()[here]).all()
    assert torch.equal(got[0].cpu()[~here], want[0].cpu()[~here])
    gb = hp.group_norm_act_bwd(xb, dyd, got[1], got[2], ga, be, act="silu")
    assert torch.isnan(gb[0].float().cpu()[here]).all()
    assert torch.equal(gb[0].cpu()[~here], back[0].cpu()[~here])
    assert torch.equal(gb[1].cpu()[:3], back[1].cpu()[:3]) and torch.equal(gb[1].cpu()[6:], back[1].cpu()[6:])


@pytest.mark.parametrize("layout", ["planes", "last"])
def test_empty_batch(layout):
    x = _dev(np.zeros((0, 8, 3, 3)), layout, "f32")
    y, mean, rstd = hp.group_norm_act_fwd(x, 4)
    dg, db = torch.full((8,), 7.0, device="cuda"), torch.full((8,), 7.0, device="cuda")
    hp.group_norm_act_bwd(x, x.clone(), mean, rstd, dgamma=dg, dbeta=db)
    assert y.shape == x.shape and not dg.any() and not db.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("shape", [(2, 12, 5, 7, 3), (1, 96, 55, 55, 32), (2, 6, 230, 231, 2), (3, 20, 1, 1, 4)])
def test_nothing_outside_the_outputs_is_written_and_nothing_is_left(shape, layout, dtype):
    """Outputs inside larger buffers, at addresses aligned to nothing but their elements; inputs too."""
    N, C, H, W, G = shape
    (x, dy), (xd, dyd), gamma, beta = _tensors(N, C, H, W, layout, dtype, 9)
    td = xd.dtype

    def placed(like, off, fill=None):
        buf = torch.full((like.numel() + 128,), 7.0, dtype=td, device="cuda")
        v = buf[off:off + like.numel()]
        t = v.view(N, H, W, C).permute(0, 3, 1, 2) if layout == "last" else v.view(N, C, H, W)
        t.copy_(like) if fill is None else t.fill_(fill)
        return buf, t

    nan = float("nan")
    _, xo = placed(xd, 61)
    _, dyo = placed(dyd, 63)
    by, y = placed(xd, 65, nan)
    bx, dx = placed(xd, 67, nan)
    ga, be = _cuda(gamma), _cuda(beta)
    want = hp.group_norm_act_fwd(xd, G, ga, be, act="silu")
    got = hp.group_norm_act_fwd(xo, G, ga, be, act="silu", y=y)
    back = hp.group_norm_act_bwd(xd, dyd, want[1], want[2], ga, be, act="silu")
    gb = hp.group_norm_act_bwd(xo, dyo, want[1], want[2], ga, be, act="silu", dx=dx)
    for a, b in zip(want + back, got + gb):
        assert torch.equal(a, b)
    for buf, off in ((by, 65), (bx, 67)):
        assert bool((buf[:off] == 7.0).all()) and bool((buf[off + xd.numel():] == 7.0).all())
        assert not torch.isnan(buf).any()


@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("shape", [(3, 96, 55, 55, 32), (4, 16, 160, 160, 2), (40, 24, 3, 5, 8)])
def test_same_bits_every_time(shape, layout):
    N, C, H, W, G = shape
    _, (xd, dyd), gamma, beta = _tensors(N, C, H, W, layout, "f32", 10)
    ga, be = _cuda(gamma), _cuda(beta)
    first = None
    for _ in range(3):
        f = hp.group_norm_act_fwd(xd, G, ga, be, act="relu")
        b = hp.group_norm_act_bwd(xd, dyd, f[1], f[2], ga, be, act="relu")
        now = [t.clone() for t in f + b]
        assert first is None or all(torch.equal(p, q) for p, q in zip(first, now))
        first = now


def test_a_sample_is_normalised_alone():
    """Results of a sample are its own in whatever batch it stands (up to the order of sums): a shard needs no exchange."""
    _, (xd, _), gamma, beta = _tensors(9, 48, 13, 13, "planes", "f32", 11)
    ga, be = _cuda(gamma), _cuda(beta)
    whole = hp.group_norm_act_fwd(xd, 16, ga, be)[0]
    part = hp.group_norm_act_fwd(xd[4:6], 16, ga, be)[0]
    assert torch.allclose(whole[4:6], part, rtol=1e-5, atol=1e-6)


def test_on_another_stream_and_in_a_graph():
    _, (xd, dyd), gamma, beta = _tensors(4, 96, 27, 27, "planes", "f32", 12)
    ga, be, ws = _cuda(gamma), _cuda(beta), hp.Workspace()
    want = hp.group_norm_act_fwd(xd, 32, ga, be)
    wb = hp.group_norm_act_bwd(xd, dyd, want[1], want[2], ga, be)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = hp.group_norm_act_fwd(xd, 32, ga, be, ws=ws)
        gb = hp.group_norm_act_bwd(xd, dyd, got[1], got[2], ga, be, ws=ws)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want + wb, got + gb))
    outs = [torch.empty_like(t) for t in want + wb]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hp.group_norm_act_fwd(xd, 32, ga, be, y=outs[0], mean=outs[1], rstd=outs[2], ws=ws)
        hp.group_norm_act_bwd(xd, dyd, outs[1], outs[2], ga, be, dx=outs[3], dgamma=outs[4], dbeta=outs[5], ws=ws)
    for _ in range(3):
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want + wb, outs))


def test_offsets_past_32_bits():
    """More than 2^32 bytes to a tensor: the last samples are what they are alone."""
    N, C, H, W = 150, 64, 336, 336                                  # 1.08e9 values, 4.3 GB
    x = torch.zeros((N, C, H, W), device="cuda")
    x[-2:].normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    ga, be = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    y, mean, rstd = hp.group_norm_act_fwd(x, 32, ga, be)
    y2, mean2, rstd2 = hp.group_norm_act_fwd(x[-2:].clone(), 32, ga, be)
    assert torch.allclose(y[-2:], y2, rtol=1e-5, atol=1e-5) and torch.allclose(mean[-2:], mean2, atol=1e-6)
    assert not y[:-2].any()
    dy = x
    dx = hp.group_norm_act_bwd(x, dy, mean, rstd, ga, be, dx=y)[0]
    dx2 = hp.group_norm_act_bwd(x[-2:].clone(), dy[-2:].clone(), mean2, rstd2, ga, be)[0]
    assert torch.allclose(dx[-2:], dx2, rtol=1e-4, atol=1e-4)


def test_groups_of_millions_of_channels():
    """More channels to a group than 24-bit products of their number hold.  Sums run over chains of up to 2^15 here, so the
    gradient's means may be off by 2^15 u of the mean magnitude, 1.6e-3 and 6 times that with |xh| up to 6."""
    C, S = (1 << 23) + 3000, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn((1, C, 1, S), device="cuda", generator=g) for _ in range(2))
    y, mean, rstd = hp.group_norm_act_fwd(x, 1, act="none")
    xd, dyd = x.double(), dy.double()
    m = xd.mean()
    r = (xd.sub(m).square().mean() + 1e-5).rsqrt()
    xh = (xd - m) * r
    assert abs(float(mean - m)) < 1e-4 and abs(float(rstd / r - 1)) < 1e-4
    assert float((y - xh).abs().max()) < 1e-3
    dx, dgamma, dbeta = hp.group_norm_act_bwd(x, dy, mean, rstd, act="none")
    want = r * (dyd - dyd.mean() - xh * (dyd * xh).mean())
    assert float((dx - want).abs().max()) < 0.02
    assert float((dbeta - dyd.sum((0, 2, 3))).abs().max()) < 1e-4
    assert float((dgamma - (dyd * xh).sum((0, 2, 3))).abs().max()) < 1e-2


@pytest.mark.parametrize("shape", [(512, 8192, 1, 1, 4096), (512, 8190, 1, 2, 8190)])
def test_thousands_of_small_groups_channels_last(shape):
    """The widest slabs: their channels' and groups' sums have to fit beside the threads' own."""
    N, C, H, W, G = shape
    run_case(N, C, H, W, G, "none", "last", "bf16", seed=14)


# Kernels of every plan: a wavefront to a group, a work-group to a group (one run of memory, planes of their own), tiles of
# planes and of parts of a plane; slabs of whole groups and of groups that share vectors, tiles of slabs, very wide groups
PLANS = [(1030, 4, 3, 7, 2), (3, 24, 13, 13, 4), (2, 6, 31, 45, 2), (1, 5, 120, 130, 1), (1, 2, 401, 399, 1), (2, 48, 9, 11, 3),
         (2, 64, 27, 27, 8), (1, 70, 112, 113, 2), (1, 9000, 1, 7, 1), (2, 3, 2, 1, 3)]


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", PLANS)
def test_an_infinite_gradient_wherever_it_stands(shape, layout, dtype, act):
    """Sums with one infinite term are that infinity, in the channel that holds it; the other groups do not see it."""
    N, C, H, W, G = shape
    (x, _), (xd, dyd), gamma, beta = _tensors(N, C, H, W, layout, dtype, 30)
    ga, be = _cuda(gamma), _cuda(beta)
    _, mean, rstd = hp.group_norm_act_fwd(xd, G, ga, be, act=act)
    want = hp.group_norm_act_bwd(xd, dyd, mean, rstd, ga, be, act=act)
    S, c = H * W, C // 2
    other = torch.ones(C, dtype=torch.bool, device="cuda")
    other[c] = False
    for s in sorted({p for p in (*range(9), *range(S - 18, S)) if 0 <= p < S}):
        dyi = dyd.clone(memory_format=torch.preserve_format)
        dyi[N - 1, c, s // W, s % W] = float("inf")
        dx, dgamma, dbeta = hp.group_norm_act_bwd(xd, dyi, mean, rstd, ga, be, act=act)
        xi, m, r = (float(v) for v in (xd[N - 1, c, s // W, s % W], mean[N - 1, c * G // C], rstd[N - 1, c * G // C]))
        z = float(ga[c]) * (xi - m) * r + float(be[c])
        slope = 1.0 if act == "none" else (1 + z / (1 + np.exp(z))) / (1 + np.exp(-z))
        assert float(dbeta[c]) == np.copysign(np.inf, slope), s
        assert float(dgamma[c]) == np.copysign(np.inf, slope * (xi - m)), s
        assert torch.equal(dbeta[other], want[2][other]) and torch.equal(dgamma[other], want[1][other])
        per = C // G
        same = torch.ones(N, C, dtype=torch.bool, device="cuda")
        same[N - 1, c // per * per:(c // per + 1) * per] = False
        assert torch.equal(dx[same], want[0][same])


@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", PLANS)
def test_the_mean_of_an_infinite_value_wherever_it_stands(shape, layout, dtype):
    N, C, H, W, G = shape
    (x, _), (xd, _), gamma, beta = _tensors(N, C, H, W, layout, dtype, 31)
    S, c = H * W, C // 2
    want = hp.group_norm_act_fwd(xd, G, act="relu")[1]
    for sign in (1.0, -1.0):
        for s in sorted({p for p in (*range(9), *range(S - 18, S)) if 0 <= p < S}):
            xi = xd.clone(memory_format=torch.preserve_format)
            xi[N - 1, c, s // W, s % W] = sign * float("inf")
            y, mean, rstd = hp.group_norm_act_fwd(xi, G, act="relu")
            here = (N - 1, c * G // C)
            assert float(mean[here]) == sign * float("inf") and torch.isnan(rstd[here]), s
            mean[here] = want[here]
            assert torch.equal(mean, want)


@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", PLANS)
def test_a_group_of_one_value_gives_its_shift(shape, layout, dtype):
    """Every distance from the mean is zero, however large the mean: sums of up to 2^21 times 1536 = 3 * 2^9 are exact in
    fp32, and so is their quotient."""
    N, C, H, W, G = shape
    for value in (1536.0, -96.0):
        x = _dev(np.full((N, C, H, W), value), layout, dtype)
        gamma, beta = torch.full((C,), 1.7, device="cuda"), torch.linspace(-2, 3, C, device="cuda")
        y, mean, rstd = hp.group_norm_act_fwd(x, G, gamma, beta, act="none")
        assert bool((mean == value).all())
        assert torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-6)
        assert torch.equal(y, beta.to(y.dtype)[None, :, None, None].expand_as(y))


@pytest.mark.parametrize("layout", ["planes", "last"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", PLANS)
def test_forward_and_backward_agree_where_a_relu_is_open(shape, layout, dtype):
    """With a gradient of one everywhere dbeta counts the values that pass; these are the ones that forward leaves positive,
    and gamma's gradient has the sign that follows.  Means of 1 to 1000 deviations."""
    N, C, H, W, G = shape
    for k, level in enumerate((1.0, 30.0, 1000.0)):
        _, (xd, _), gamma, beta = _tensors(N, C, H, W, layout, dtype, 20 + k, mean=level)
        ga, be = _cuda(gamma), _cuda(0.1 * beta)
        y, mean, rstd = hp.group_norm_act_fwd(xd, G, ga, be, act="relu")
        ones = torch.ones_like(xd)
        _, _, dbeta = hp.group_norm_act_bwd(xd, ones, mean, rstd, ga, be, act="relu")
        assert torch.equal(dbeta.double(), (y > 0).double().sum((0, 2, 3)))         # counts below 2^24: exact


def test_the_longest_plane():
    """2^31 - 1 positions, of which the last vector holds seven of its eight."""
    S = (1 << 31) - 1
    x = torch.empty((1, 1, 1, S), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(6))
    x += 0.5
    y, mean, rstd = hp.group_norm_act_fwd(x, 1, act="none")
    dx, dgamma, dbeta = hp.group_norm_act_bwd(x, y, mean, rstd, act="none")
    m = sum(p.double().sum().item() for p in x.view(-1).split(1 << 28)) / S
    var = sum((p.double() - m).square().sum().item() for p in x.view(-1).split(1 << 28)) / S
    assert abs(mean.item() - m) <= SUM and abs(rstd.item() * (var + 1e-5) ** 0.5 - 1) <= SUM
    for at in (slice(0, 5000), slice(S // 2, S // 2 + 5000), slice(S - 5000, S)):
        want = (x[0, 0, 0, at].double() - m) * (var + 1e-5) ** -0.5
        assert bool(((y[0, 0, 0, at].double() - want).abs() <= 2.0 ** -8 * want.abs() + SUM).all())
        # dy = y is xh up to its rounding: what is left of it after the share of xh
        left = rstd.double().item() * (y[0, 0, 0, at].double() - dbeta.item() / S - want * dgamma.item() / S)
        assert bool(((dx[0, 0, 0, at].double() - left).abs() <= 2.0 ** -8 * left.abs() + 16 * U * (1 + want.abs())).all())
    assert abs(dgamma.item() / S - 1) <= 2.0 ** -8 and abs(dbeta.item() / S) <= 2.0 ** -8


@pytest.mark.parametrize("layout,shape", [("last", (1, 4104, 64, 64, 1)), ("last", (1, 8200, 40, 40, 1)), ("planes", (1, 12, 90, 91, 3)),
                                          ("last", (200000, 4, 1, 1, 2)), ("planes", (30000, 3, 1, 5, 3))])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_sums_of_like_terms(shape, layout, dtype):
    """Terms of one sign and size, whose roundings in a long fp32 chain all go the same way (a chain of 10^4 of 0.1: 10^3 u):
    the bounds of a few hundred hold for very wide groups and for many samples as well."""
    N, C, H, W, G = shape
    g = np.random.Generator(np.random.Philox(40))
    x = 0.1 + 1e-3 * g.standard_normal((N, C, H * W))
    dy = np.full((N, C, H * W), 0.1) + 1e-4 * (g.random((N, C, H * W)) < 0.01)
    gamma, beta = np.ones(C, np.float32), np.zeros(C, np.float32)
    rnd = oracle.bf16_round if dtype == "bf16" else (lambda a: a)
    x, dy = (rnd(v.astype(np.float32)).astype(np.float64) for v in (x, dy))
    xd, dyd = (_dev(v.reshape(N, C, H, W), layout, dtype) for v in (x, dy))
    got = hp.group_norm_act_fwd(xd, G, _cuda(gamma), _cuda(beta), act="none")
    check_fwd(got, x, G, gamma, beta, 1e-5, "none", dtype)
    m, r = (v.astype(np.float32).astype(np.float64) for v in oracle.group_norm_stats(x, G, 1e-5))
    got = hp.group_norm_act_bwd(xd, dyd, _cuda(m), _cuda(r), _cuda(gamma), _cuda(beta), act="none")
    check_bwd(got, x, dy, m, r, gamma, beta, "none", dtype)


@pytest.mark.parametrize("layout", ["planes", "last"])
def test_gradient_means_of_millions_of_channels(layout):
    """dy with a mean and a share of xh, so that dx takes off two terms of the size of dy itself: rstd (64 u of the terms'
    mean magnitudes, 0.8 and 0.8 |xh| with |xh| below 6, and 8 u of what is subtracted) is below 4e-5."""
    C, S = (1 << 22) + 1500, 2
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((1, C, 1, S), device="cuda", generator=g)
    if layout == "last":
        x = x.contiguous(memory_format=torch.channels_last)
    y, mean, rstd = hp.group_norm_act_fwd(x, 1, act="none")
    xd = x.double()
    m, r = mean.double().item(), rstd.double().item()
    assert abs(m - xd.mean().item()) <= 64 * U and abs(r * (xd.var(correction=0).item() + 1e-5) ** 0.5 - 1) <= 64 * U
    xh = (xd - m) * r
    dy = (0.3 + 0.5 * xh + 0.2 * torch.randn(x.shape, device="cuda", generator=g, dtype=torch.float64)).float()
    dy = dy.contiguous(memory_format=torch.channels_last) if layout == "last" else dy.contiguous()
    dx, dgamma, dbeta = hp.group_norm_act_bwd(x, dy, mean, rstd, act="none")
    dyd = dy.double()
    m1, m2 = dyd.mean().item(), (dyd * xh).mean().item()
    assert m1 > 0.25 and m2 > 0.4
    assert float((dx - r * (dyd - m1 - xh * m2)).abs().max()) <= 4e-5
    assert float((dbeta - dyd.sum((0, 2, 3))).abs().max()) <= 1e-6 and float((dgamma - (dyd * xh).sum((0, 2, 3))).abs().max()) <= 2e-5
    # like terms: what is left of 0.1 - m1 is the error of m1 (xh's share: of sums of both signs)
    one = torch.full_like(x, 0.1)
    left = hp.group_norm_act_bwd(x, one, mean, rstd, act="none")[0].double()
    ref = 0.1 * (xh.mean().item() * xh)
    assert float((left + r * ref).abs().max()) <= r * (64 * U * 0.1 * (1 + 6 * 0.8) + 8 * U * 0.3)
