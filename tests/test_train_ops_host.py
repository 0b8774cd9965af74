"""Group normalisation and the distillation loss without a GPU: the oracle's definitions against what the mathematics
fixes, and the argument checks of the entry points."""
import ctypes

import numpy as np
import pytest
import torch

import oracle

PTR = 4096
RNG = lambda s: np.random.Generator(np.random.Philox(s))


@pytest.fixture(scope="module")
def lib():
    from paper_1312_5853_amd import binding, build
    if build.is_stale():
        build.build()
    return binding.lib()


# ------------------------------------------------------------- the oracle ---
@pytest.mark.parametrize("groups", [1, 2, 6])
def test_normalised_groups_have_mean_zero_and_variance_one(groups):
    x = RNG(1).normal(3.0, 2.0, (2, 6, 35))
    y, mean, rstd = oracle.group_norm_act_fwd(x, groups, np.ones(6), np.zeros(6), 1e-12, "none")
    v = y.reshape(2, groups, -1)
    assert np.abs(v.mean(2)).max() < 1e-12 and np.abs((v ** 2).mean(2) - 1).max() < 1e-9
    # shift and scale of a group's input change nothing but its statistics
    y2, mean2, _ = oracle.group_norm_act_fwd(5.0 * x - 7.0, groups, np.ones(6), np.zeros(6), 1e-12, "none")
    assert np.abs(y2 - y).max() < 1e-9 and np.abs(mean2 - (5.0 * mean - 7.0)).max() < 1e-12


def test_group_norm_by_hand():
    # one group of four values 1, 2, 3, 6: mean 3, variance 14/4; eps makes it 4
    y, mean, rstd = oracle.group_norm_act_fwd(np.array([[[1.0, 2.0], [3.0, 6.0]]]), 1, [2.0, 4.0], [0.5, -2.0], 0.5, "relu")
    assert mean[0, 0] == 3.0 and rstd[0, 0] == 0.5
    assert y.tolist() == [[[0.0, 0.0], [0.0, 4.0]]]        # 2*-1+.5, 2*-.5+.5, 4*0-2, 4*1.5-2


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("groups", [1, 3])
def test_group_norm_gradient_against_differences(act, groups):
    g = RNG(2)
    x, dy = g.normal(size=(2, 6, 7)), g.normal(size=(2, 6, 7))
    gamma, beta, eps = g.normal(1.0, 0.3, 6), g.normal(0, 0.3, 6), 1e-3
    f = lambda x, gamma, beta: float((oracle.group_norm_act_fwd(x, groups, gamma, beta, eps, act)[0] * dy).sum())
    _, mean, rstd = oracle.group_norm_act_fwd(x, groups, gamma, beta, eps, act)
    grads = oracle.group_norm_act_bwd(x, dy, mean, rstd, gamma, beta, act)
    args, h = [x, gamma, beta], 1e-6
    for which, grad in enumerate(grads):
        num = np.zeros_like(args[which])
        for i in np.ndindex(num.shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[which][i] += h
            down[which][i] -= h
            num[i] = (f(*up) - f(*down)) / (2 * h)
        # differences of values of size 30 at h = 1e-6: 30 * 1e-16 / 1e-6 and the third derivative's h^2
        assert np.abs(num - grad).max() < 1e-7


def test_label_loss_by_hand():
    z = np.log([[1.0, 2.0, 5.0]])
    loss, dz = oracle.distill_loss(z, labels=np.array([1]), label_weight=2.0, grad=[3.0])
    assert abs(loss[0] - 2.0 * np.log(4.0)) < 1e-14
    assert np.abs(dz - 6.0 * np.array([[0.125, 0.25 - 1.0, 0.625]])).max() < 1e-14


def test_teacher_loss_by_hand():
    # T = 2: student exp(z/2) = 1, 1, 2; teacher exp(t/2) = 1, 3 on classes 2 and 0
    z, t = 2.0 * np.log([[1.0, 1.0, 2.0]]), 2.0 * np.log([[1.0, 3.0]])
    loss, dz = oracle.distill_loss(z, top_idx=np.array([[2, 0]]), top_val=t, temperature=2.0, kd_weight=0.5)
    assert abs(loss[0] - 0.5 * 4 * (0.25 * np.log(0.25 / 0.5) + 0.75 * np.log(0.75 / 0.25))) < 1e-14
    assert np.abs(dz - 0.5 * 2 * np.array([[0.25 - 0.75, 0.25, 0.5 - 0.25]])).max() < 1e-14


def test_loss_gradient_against_differences():
    g = RNG(3)
    N, V = 5, 9
    z, labels = g.normal(size=(N, V)), np.array([0, 8, -1, 3, 9])
    idx = np.array([[1, 2, 1], [0, -1, 5], [-1, -1, -1], [4, 4, 4], [3, 9, -7]])
    val, w = g.normal(size=(N, 3)), g.normal(size=N)
    args = dict(labels=labels, top_idx=idx, top_val=val, temperature=1.7, kd_weight=0.6, label_weight=0.4)
    loss, dz = oracle.distill_loss(z, grad=w, **args)
    assert loss[2] == 0.0 and not dz[2].any()
    h, num = 1e-6, np.zeros_like(z)
    for i in np.ndindex(z.shape):
        up, down = z.copy(), z.copy()
        up[i] += h
        down[i] -= h
        num[i] = ((oracle.distill_loss(up, **args)[0] - oracle.distill_loss(down, **args)[0]) * w).sum() / (2 * h)
    assert np.abs(num - dz).max() < 1e-8
    # a row's gradient sums to zero: adding a constant to its logits changes nothing
    assert np.abs(dz.sum(1)).max() < 1e-14


def test_teacher_equal_to_the_student_costs_nothing():
    z = RNG(4).normal(size=(3, 6))
    loss, dz = oracle.distill_loss(z, top_idx=np.tile(np.arange(6), (3, 1)), top_val=z + 2.0, temperature=3.0)
    assert np.abs(loss).max() < 1e-13 and np.abs(dz).max() < 1e-13


# ------------------------------------------------------- argument checks ---
def _norm_args(**kw):
    a = dict(x=PTR, gamma=None, beta=None, y=PTR * 2, mean=None, rstd=None, N=2, C=8, S=9, groups=4, eps=1e-5, act=1,
             layout=0, dtype=0, ws=PTR, ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return list(a.values())


def test_norm_forward_argument_checks(lib):
    from paper_1312_5853_amd import binding as b
    f = lambda **kw: lib.group_norm_act_fwd(*_norm_args(**kw))
    for bad in (dict(x=None), dict(y=None), dict(y=PTR), dict(N=-1), dict(C=0), dict(S=0), dict(groups=0), dict(groups=3),
                dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(act=3), dict(act=-1), dict(layout=2)):
        assert f(**bad) == b.ERR_INVALID_ARG, bad
    assert f(dtype=5) == b.ERR_BAD_DTYPE
    assert f(C=1 << 16, S=1 << 15) == b.ERR_TOO_LARGE
    assert f(N=1 << 28) == b.ERR_TOO_LARGE
    for bad in (dict(x=PTR + 2), dict(y=PTR + 2), dict(x=PTR + 1, dtype=1), dict(gamma=PTR + 2), dict(beta=PTR + 1),
                dict(mean=PTR + 2), dict(rstd=PTR + 3)):
        assert f(**bad) == b.ERR_MISALIGNED, bad
    assert f(N=0, x=None, y=None) == b.OK


def _norm_bwd_args(**kw):
    a = dict(x=PTR, dy=PTR, gamma=None, beta=None, mean=PTR, rstd=PTR, dx=PTR * 2, dgamma=None, dbeta=None, N=2, C=8,
             S=9, groups=4, act=1, layout=0, dtype=0, ws=PTR, ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return list(a.values())


def test_norm_backward_argument_checks(lib):
    from paper_1312_5853_amd import binding as b
    f = lambda **kw: lib.group_norm_act_bwd(*_norm_bwd_args(**kw))
    for bad in (dict(x=None), dict(dy=None), dict(mean=None), dict(rstd=None), dict(dx=None), dict(dx=PTR), dict(N=-1),
                dict(groups=5), dict(act=7), dict(layout=-1)):
        assert f(**bad) == b.ERR_INVALID_ARG, bad
    assert f(dtype=3) == b.ERR_BAD_DTYPE
    for bad in (dict(dy=PTR + 2), dict(dx=PTR + 1, dtype=2), dict(dgamma=PTR + 2), dict(dbeta=PTR + 2), dict(ws=PTR + 8)):
        assert f(**bad) == b.ERR_MISALIGNED, bad
    need = lib.group_norm_act_workspace_bytes(b.OP_BWD_DATA, 2, 8, 9, 4, 0, 0)
    assert need > 0
    assert f(ws_bytes=need - 1) == b.ERR_WORKSPACE
    assert f(ws=None) == b.ERR_WORKSPACE
    assert lib.group_norm_act_workspace_bytes(b.OP_BWD_DATA, 2, 8, 9, 3, 0, 0) == 0
    assert lib.group_norm_act_workspace_bytes(b.OP_BWD_DATA, 2, 8, 9, 4, 0, 9) == 0
    assert lib.group_norm_act_workspace_bytes(9, 2, 8, 9, 4, 0, 0) == 0


def test_sizes_past_what_a_launch_or_its_counters_hold(lib):
    from paper_1312_5853_amd import binding as b
    big = dict(N=1 << 14, C=1 << 16, S=1 << 14, groups=1 << 5)                     # 2^44 values
    for layout in (0, 1):
        assert lib.group_norm_act_fwd(*_norm_args(layout=layout, **big)) == b.ERR_TOO_LARGE
        assert lib.group_norm_act_bwd(*_norm_bwd_args(layout=layout, **big)) == b.ERR_TOO_LARGE
    many = dict(N=1 << 25, C=8, S=200, groups=8)                                   # 2^28 groups of a wavefront each
    assert lib.group_norm_act_fwd(*_norm_args(**many)) == b.ERR_TOO_LARGE
    assert lib.distill_loss_fwd(*_loss_args(N=1 << 27)) == b.ERR_TOO_LARGE         # 2^27 rows of a wavefront each


def _loss_args(**kw):
    a = dict(z=PTR, z_stride=10, labels=PTR, top_idx=PTR, top_val=PTR, loss=PTR, stats=PTR, N=2, V=10, K=3, T=2.0, wk=1.0,
             wl=1.0, ib=4, td=0, dtype=0, ws=PTR, ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return list(a.values())


NAN, INF = float("nan"), float("inf")
LOSS_BAD = (dict(z=None), dict(labels=None, K=0), dict(top_idx=None), dict(top_val=None), dict(z_stride=9), dict(N=-1),
            dict(V=0), dict(K=-1), dict(T=0.0), dict(T=-1.0), dict(T=NAN), dict(T=INF), dict(wk=NAN), dict(wl=INF),
            dict(ib=2))


def test_loss_forward_argument_checks(lib):
    from paper_1312_5853_amd import binding as b
    f = lambda **kw: lib.distill_loss_fwd(*_loss_args(**kw))
    for bad in LOSS_BAD + (dict(loss=None),):
        assert f(**bad) == b.ERR_INVALID_ARG, bad
    assert f(dtype=4) == b.ERR_BAD_DTYPE and f(td=4) == b.ERR_BAD_DTYPE
    assert f(K=b.DISTILL_MAX_TOP + 1) == b.ERR_TOO_LARGE
    for bad in (dict(z=PTR + 2), dict(z=PTR + 1, dtype=1), dict(labels=PTR + 2), dict(labels=PTR + 4, ib=8),
                dict(top_idx=PTR + 1), dict(top_val=PTR + 2), dict(loss=PTR + 2), dict(stats=PTR + 2)):
        assert f(**bad) == b.ERR_MISALIGNED, bad
    assert f(N=0, z=None, labels=None, top_idx=None, top_val=None, loss=None, stats=None) == b.OK
    assert lib.distill_loss_workspace_bytes(-1, 10, 3, 0) == 0
    assert lib.distill_loss_workspace_bytes(4, 10, 3, 7) == 0


def test_loss_backward_argument_checks(lib):
    from paper_1312_5853_amd import binding as b
    base = dict(z=PTR, z_stride=10, labels=PTR, top_idx=PTR, top_val=PTR)
    size = dict(N=2, V=10, K=3, T=2.0, wk=1.0, wl=1.0, ib=4, td=0, dtype=0)
    alone = dict(base, stats=PTR, grad=None, scale=1.0, dz=PTR * 2, dz_stride=10, **size, stream=None)
    both = dict(base, grad=None, scale=1.0, loss=PTR, dz=PTR * 2, dz_stride=10, **size, ws=PTR, ws_bytes=1 << 30, stream=None)
    for f, args in ((lib.distill_loss_bwd, alone), (lib.distill_loss_fwd_bwd, both)):
        call = lambda **kw: f(*dict(args, **kw).values())
        more = (dict(dz=None), dict(dz_stride=9), dict(scale=NAN), dict(dz=PTR, dz_stride=12))
        for bad in LOSS_BAD + more + ((dict(stats=None),) if "stats" in args else (dict(loss=None),)):
            assert call(**bad) == b.ERR_INVALID_ARG, bad
        assert call(dtype=4) == b.ERR_BAD_DTYPE
        assert call(K=b.DISTILL_MAX_TOP + 1) == b.ERR_TOO_LARGE
        for bad in (dict(dz=PTR + 2), dict(grad=PTR + 2)):
            assert call(**bad) == b.ERR_MISALIGNED, bad


def test_binding_refuses_what_the_library_cannot_see(lib):
    """Shapes, types, memory orders and devices are checked before any pointer is taken."""
    from paper_1312_5853_amd import binding as b
    x = torch.zeros(2, 8, 3, 3)
    with pytest.raises(ValueError):
        b.group_norm_act_fwd(x, 4)                                          # not on a GPU
    with pytest.raises(ValueError):
        b.group_norm_act_fwd(x[:, :, ::2], 4)                               # not dense
    with pytest.raises(ValueError):
        b.group_norm_act_fwd(x, 4, y=torch.zeros(2, 8, 3, 3).contiguous(memory_format=torch.channels_last))
    with pytest.raises(ValueError):
        b.group_norm_act_fwd(x, 4, act="tanh")
    with pytest.raises(ValueError):
        b.group_norm_act_fwd(x, 4, gamma=torch.zeros(7))
    with pytest.raises(TypeError):
        b.group_norm_act_fwd(x, 4, y=torch.zeros(2, 8, 3, 3, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        b.group_norm_act_fwd(x.double(), 4)
    with pytest.raises(TypeError):
        b.group_norm_act_fwd(x, 4.0)
    with pytest.raises(ValueError):
        b.group_norm_act_bwd(x, x, torch.zeros(2, 4), torch.zeros(2, 3))
    z, lab, idx, val = torch.zeros(3, 7), torch.zeros(3, dtype=torch.int64), torch.zeros(3, 2, dtype=torch.int64), torch.zeros(3, 2)
    for bad in (dict(labels=lab), dict(labels=lab[:2]), dict(top_idx=idx), dict(top_idx=idx, top_val=val[:, :1]),
                dict(top_idx=idx[:2], top_val=val[:2]), dict(labels=lab, loss=torch.zeros(4)),
                dict(labels=lab, stats=torch.zeros(3, 2))):
        with pytest.raises(ValueError):
            b.distill_loss_fwd(z, **bad)
    with pytest.raises(ValueError):
        b.distill_loss_fwd(z.t(), labels=lab)
    for bad in (dict(labels=lab.float()), dict(labels=lab.int(), top_idx=idx, top_val=val),
                dict(top_idx=idx, top_val=val.double())):
        with pytest.raises(TypeError):
            b.distill_loss_fwd(z, **bad)
    with pytest.raises(ValueError):
        b.distill_loss_fwd_bwd(z, labels=lab, dz=torch.zeros(3, 8))
    with pytest.raises(TypeError):
        b.distill_loss_fwd_bwd(z.cuda() if torch.cuda.is_available() else z, labels=lab, dz=torch.zeros(3, 7, dtype=torch.bfloat16))


@pytest.mark.parametrize("dtype,per_tile", [(0, 8192), (1, 16384)])
def test_the_longest_plane(lib, dtype, per_tile):
    """C * S of 2^31 - 1 is within the limits: tiles of a plane, three sums each, then the group's two."""
    from paper_1312_5853_amd import binding as b
    for S in ((1 << 31) - 1, (1 << 31) - 3, (1 << 31) - 16):
        tiles = -(-S // per_tile)
        need = lib.group_norm_act_workspace_bytes(b.OP_FWD, 1, 1, S, 1, 0, dtype)
        assert need == -(-12 * tiles // 256) * 256 + 256
        assert lib.group_norm_act_fwd(*_norm_args(N=1, C=1, S=S, groups=1, dtype=dtype, ws_bytes=need - 1)) == b.ERR_WORKSPACE
        need = lib.group_norm_act_workspace_bytes(b.OP_BWD_DATA, 1, 1, S, 1, 0, dtype)
        assert need == -(-8 * tiles // 256) * 256 + 256
        assert lib.group_norm_act_bwd(*_norm_bwd_args(N=1, C=1, S=S, groups=1, dtype=dtype, ws_bytes=need - 1)) == b.ERR_WORKSPACE


def test_tensors_of_another_gpu_than_the_current_one(monkeypatch):
    """A launch goes to the current GPU, whose kernels may not reach another one's memory."""
    from paper_1312_5853_amd import binding as b

    class Stream:
        device_index, cuda_stream = 1, 77

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 55 + d, raising=False)
    assert b._current_stream(None, 1) == 56 and b._current_stream(Stream, 1) == 77
    for stream, d in ((None, 0), (Stream, 0), (type("S", (Stream,), dict(device_index=0)), 1)):
        with pytest.raises(ValueError):
            b._current_stream(stream, d)


def test_the_oracle_against_loops():
    """Both operators written out value by value, from the definitions, on sizes with several groups and entries."""
    g = RNG(9)
    N, C, S, G, eps = 2, 6, 5, 3, 1e-2
    x, dy = g.normal(size=(N, C, S)).tolist(), g.normal(size=(N, C, S)).tolist()
    gamma, beta = g.normal(1.0, 0.3, C).tolist(), g.normal(0, 0.3, C).tolist()
    y, dx = np.zeros((N, C, S)), np.zeros((N, C, S))
    dgamma, dbeta = np.zeros(C), np.zeros(C)
    means, rstds = np.zeros((N, G)), np.zeros((N, G))
    for n in range(N):
        for k in range(G):
            chans = [c for c in range(C) if c // (C // G) == k]
            M = len(chans) * S
            m = sum(x[n][c][s] for c in chans for s in range(S)) / M
            r = (sum((x[n][c][s] - m) ** 2 for c in chans for s in range(S)) / M + eps) ** -0.5
            means[n, k], rstds[n, k] = m, r
            m1 = m2 = 0.0
            dz = {}
            for c in chans:
                for s in range(S):
                    xh = (x[n][c][s] - m) * r
                    z = gamma[c] * xh + beta[c]
                    sig = 1 / (1 + np.exp(-z))
                    y[n, c, s] = z * sig
                    dz[c, s] = dy[n][c][s] * (sig + z * sig * (1 - sig))
                    dgamma[c] += dz[c, s] * xh
                    dbeta[c] += dz[c, s]
                    m1 += gamma[c] * dz[c, s] / M
                    m2 += gamma[c] * dz[c, s] * xh / M
            for c in chans:
                for s in range(S):
                    dx[n, c, s] = r * (gamma[c] * dz[c, s] - m1 - (x[n][c][s] - m) * r * m2)
    got = oracle.group_norm_act_fwd(np.array(x), G, gamma, beta, eps, "silu")
    assert all(np.abs(a - b).max() < 1e-13 for a, b in zip(got, (y, means, rstds)))
    got = oracle.group_norm_act_bwd(np.array(x), np.array(dy), means, rstds, gamma, beta, "silu")
    assert all(np.abs(a - b).max() < 1e-13 for a, b in zip(got, (dx, dgamma, dbeta)))
    V, T, wk, wl = 7, 1.6, 0.7, 0.3
    z, lab, w = g.normal(size=(4, V)), [2, -1, 6, 7], [1.0, 0.5, -2.0, 3.0]
    idx, val = [[1, 1, -1], [0, 6, 3], [9, -2, 5], [-1, 7, -1]], g.normal(size=(4, 3))
    loss, dz = np.zeros(4), np.zeros((4, V))
    for n in range(4):
        held = [k for k in range(3) if 0 <= idx[n][k] < V]
        e = {k: np.exp(val[n, k] / T) for k in held}
        for t, weight, targets in ((T, wk * T * T, {k: (idx[n][k], e[k] / sum(e.values())) for k in held}),
                                   (1.0, wl, {0: (lab[n], 1.0)} if 0 <= lab[n] < V else {})):
            total = sum(np.exp(z[n, v] / t) for v in range(V))
            for v, p in targets.values():
                loss[n] += weight * p * (np.log(p) - z[n, v] / t + np.log(total))
                dz[n, v] -= w[n] * weight / t * p
            if targets:
                for v in range(V):
                    dz[n, v] += w[n] * weight / t * np.exp(z[n, v] / t) / total
    got = oracle.distill_loss(z, np.array(lab), np.array(idx), val, T, wk, wl, w)
    assert np.abs(got[0] - loss).max() < 1e-13 and np.abs(got[1] - dz).max() < 1e-13
