"""The loss against labels and a teacher's top logits on the GPU against the oracle in 64 bits, element by element.

The bounds: u = 2^-24.  exp((z - m) / T) has a relative error of a few roundings of its argument, that is 4 u (1 + |z - m| / T)
at most; sums are taken in short chains joined in trees (32 u).  64 u of each term's magnitude covers both.  dz stored as
bfloat16 adds 2^-8 of itself."""
import numpy as np
import pytest
import torch

import oracle
from paper_1312_5853_amd import binding as hp

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
E = 64 * U
INF, NAN = float("inf"), float("nan")


def inputs(N, V, K, dtype, seed, top_dtype=None, std=2.0):
    """Logits and targets as numpy (values of the type): some rows with fewer entries, none, or no label."""
    g = np.random.Generator(np.random.Philox(seed))
    z = (std * g.standard_normal((N, V))).astype(np.float32)
    lab = g.integers(0, V, N)
    lab[g.random(N) < 0.2] = -1
    idx = val = None
    if K:
        idx = np.stack([g.permutation(V)[:K] if V >= K else g.integers(0, V, K) for _ in range(N)])
        val = (6.0 - np.sort(-std * g.standard_normal((N, K)), 1)).astype(np.float32)
        for n in range(N):
            if g.random() < 0.3:
                idx[n, g.integers(0, K + 1):] = -1
    if dtype == "bf16":
        z = oracle.bf16_round(z)
    if K and (top_dtype or dtype) == "bf16":
        val = oracle.bf16_round(val)
    return z, lab, idx, val


def dev(a, dtype=None):
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def bounds(z, lab, idx, val, T, wk, wl, grad, dtype):
    """(loss, dz, bound of the loss, bound of dz)"""
    N, V = z.shape
    loss, dz = oracle.distill_loss(z, lab, idx, val, T, wk, wl, grad)
    bl, bz = np.zeros(N), np.zeros((N, V))
    grad = np.ones(N) if grad is None else np.asarray(grad, np.float64)
    for n in range(N):
        with np.errstate(all="ignore"):
            d = z[n].astype(np.float64) - z[n].max()
            e = np.exp(d)
            if lab is not None and 0 <= lab[n] < V:
                s = e.sum()
                bl[n] += E * wl * (1 + np.log(s) + abs(d[lab[n]]))
                bz[n] += E * wl * abs(grad[n]) * np.where(e > 0, e / s * (1 - np.maximum(d, -1e30)), 0)
                bz[n, lab[n]] += E * wl * abs(grad[n])
            if idx is not None and ((idx[n] >= 0) & (idx[n] < V)).any():
                held = (idx[n] >= 0) & (idx[n] < V)
                t = val[n][held].astype(np.float64)
                t = (t - t.max()) / T
                p = np.exp(t) / np.exp(t).sum()
                eT = np.exp(d / T)
                lq = np.abs(d[idx[n][held]]) / T + np.log(eT.sum())
                use = p > 0
                bl[n] += E * wk * T * T * (1 + (p * (1 + np.abs(np.where(use, t, 0))) * (1 + np.where(use, lq, 0) + np.abs(np.log(np.where(use, p, 1)))))[use].sum())
                bz[n] += E * wk * T * abs(grad[n]) * np.where(eT > 0, eT / eT.sum() * (1 - np.maximum(d, -1e30) / T), 0)
                np.add.at(bz[n], idx[n][held], E * wk * T * abs(grad[n]) * p * (1 + np.abs(np.where(use, t, 0))))
    bl += U * np.abs(loss)
    bz += U * np.abs(dz)                                              # `want` is compared as fp32
    bz += np.abs(dz) * (2.0 ** -8 if dtype == "bf16" else U) + 1e-37
    return loss, dz, bl + 1e-37, bz


def close(got, want, bound):
    got = got.float().cpu().numpy().astype(np.float64) if isinstance(got, torch.Tensor) else got
    with np.errstate(over="ignore"):
        want = want.astype(np.float32).astype(np.float64)           # what fp32 cannot hold is infinite
    bad = np.isnan(want)
    assert (np.isnan(got) == bad).all()
    inf = np.isinf(want)
    assert (got[inf] == want[inf]).all()
    ok = ~(bad | inf)
    r = np.abs(got[ok] - want[ok]) / bound[ok]
    assert r.size == 0 or r.max() <= 1.0, r.max()


def run_case(z, lab, idx, val, T=1.0, wk=1.0, wl=1.0, dtype="f32", top_dtype=None, wide=False, grad=None, scale=1.0, zd=None):
    ints = (lambda a: None if a is None else dev(a.astype(np.int64 if wide else np.int32)))
    args = dict(labels=ints(lab), top_idx=ints(idx), top_val=dev(val, top_dtype or dtype), temperature=T, kd_weight=wk,
                label_weight=wl)
    zd = dev(z, dtype) if zd is None else zd
    gd = dev(np.asarray(grad, np.float32)) if grad is not None else None
    g = (np.ones(len(z)) if grad is None else np.asarray(grad, np.float32).astype(np.float64)) * np.float32(scale)
    loss, dz, bl, bz = bounds(z, lab, idx, val, T, wk, wl, g, dtype)
    l1, stats = hp.distill_loss_fwd(zd, **args)
    close(l1, loss, bl)
    d1 = hp.distill_loss_bwd(zd, stats, **args, grad=gd, grad_scale=scale, dz=torch.full(z.shape, NAN, dtype=zd.dtype, device="cuda"))
    close(d1, dz, bz)
    l2, d2 = hp.distill_loss_fwd_bwd(zd, **args, grad=gd, grad_scale=scale, dz=torch.full(z.shape, NAN, dtype=zd.dtype, device="cuda"))
    close(l2, loss, bl)
    close(d2, dz, bz)
    return stats, l1, d2, args


# V around the vectors, wavefronts and work-groups, and beyond what one work-group keeps
SIZES = [(1, 1, 1), (3, 2, 2), (2, 3, 5), (5, 7, 3), (4, 8, 8), (3, 9, 0), (2, 63, 4), (7, 64, 1), (3, 255, 16), (2, 257, 70), (5, 513, 10),
         (33, 1000, 10), (9, 1025, 0), (3, 2049, 33), (2, 4099, 300), (2, 8191, 64), (3, 10007, 20), (2, 16385, 1024), (1, 32771, 7),
         (2, 50021, 50), (1, 65536, 64), (2, 65539, 3), (1, 131072, 128), (1, 140001, 9), (300, 37, 5), (1500, 130, 4), (700, 1003, 6)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_against_the_oracle(size, dtype):
    N, V, K = size
    z, lab, idx, val = inputs(N, V, K, dtype, N * V + K)
    T = (1.0, 2.0, 3.3, 4.0)[(N + V) % 4]
    run_case(z, lab, idx, val, T, 0.7, 0.3, dtype, wide=V % 2 == 0, grad=np.linspace(0.5, 2.0, N), scale=1.0 / N)


@pytest.mark.parametrize("dtype,top", [("f32", "bf16"), ("bf16", "f32")])
def test_teacher_in_another_type(dtype, top):
    z, lab, idx, val = inputs(6, 300, 9, dtype, 1, top_dtype=top)
    run_case(z, lab, idx, val, 2.0, 1.0, 0.5, dtype, top_dtype=top)


def test_each_term_alone():
    z, lab, idx, val = inputs(8, 500, 12, "f32", 2)
    run_case(z, lab, None, None)
    run_case(z, None, idx, val, T=2.0)
    # a weight of zero is as good as no target: the other term's logits at -infinity do no harm
    st, l0, d0, _ = run_case(z, lab, None, None)
    z2 = z.copy()
    st, l1, d1, _ = run_case(z2, lab, np.full_like(idx, -1), val, wk=1.0)
    assert torch.allclose(l0, l1, rtol=1e-6) and torch.allclose(d0, d1, rtol=1e-5, atol=1e-9)
    off = hp.distill_loss_fwd_bwd(dev(z), labels=dev(lab), top_idx=dev(idx), top_val=dev(val), kd_weight=0.0)
    assert torch.equal(off[0], hp.distill_loss_fwd_bwd(dev(z), labels=dev(lab))[0])
    none = hp.distill_loss_fwd_bwd(dev(z), labels=dev(lab), label_weight=0.0)
    assert not none[0].any() and not none[1].any()


@pytest.mark.parametrize("V", [50, 3001, 70001])
def test_rows_without_target_are_not_looked_at(V):
    z, lab, idx, val = inputs(6, V, 5, "f32", 3)
    lab[:] = -1
    idx[::2] = -1
    z[::2] = NAN
    z[0, 1::2] = INF
    z[2, :] = -INF
    val[0] = NAN
    stats, loss, dz, _ = run_case(z, lab, idx, val, 2.0)
    assert not loss[::2].any() and not dz[::2].any() and not stats[::2].any()
    assert loss[1::2].all()


@pytest.mark.parametrize("V", [40, 5003, 70001])
@pytest.mark.parametrize("low", [-INF, -3.4028234663852886e38])
def test_classes_left_out_by_a_mask(V, low):
    """Two thirds of the classes at -infinity or at the type's lowest value have no part in the softmax."""
    z, lab, idx, val = inputs(5, V, 4, "f32", 4)
    mask = (np.arange(V) % 3) != 0
    z[:, mask] = low
    idx = np.where(idx >= 0, idx // 3 * 3, -1)
    lab = np.where(lab >= 0, lab // 3 * 3, -1)
    stats, loss, dz, _ = run_case(z, lab, idx, val, 0.7)
    rows = dz.cpu().numpy()[:, mask]
    assert not rows.any()


@pytest.mark.parametrize("V", [40, 5003, 70001])
def test_rows_that_a_mask_leaves_empty_and_targets_left_out(V):
    z, lab, idx, val = inputs(5, V, 4, "f32", 5)
    lab[:], idx[:] = 3, [0, 1, 2, 3]
    z[0] = -INF                                              # no class left: no distribution
    z[1, 1] = -INF                                           # a class that the teacher names
    z[2, 3] = -INF                                           # the label's
    val[3, 1] = -INF                                         # the teacher leaves a class out ...
    z[3, 1] = -INF                                           # ... that the student leaves out too
    z[4] = -INF
    z[4, 3] = 1.0                                            # one class left: the label
    idx[4] = 3
    stats, loss, dz, _ = run_case(z, lab, idx, val, 2.0)
    l = loss.cpu().numpy()
    assert np.isnan(l[0]) and l[1] == INF and l[2] == INF and np.isfinite(l[3]) and np.isfinite(l[4])
    assert torch.isnan(dz[0]).all() and torch.isfinite(dz[1:]).all()


@pytest.mark.parametrize("V", [40, 5003, 70001])
@pytest.mark.parametrize("value", [-3.4028234663852886e38, 3.4028234663852886e38, 1e37, -2e30])
def test_rows_of_extreme_finite_logits(V, value):
    """A row of nothing but the type's lowest (or largest) value is an even distribution; one class above it takes all."""
    z, lab, idx, val = inputs(4, V, 4, "f32", 13)
    z[:2] = value
    z[1, 2] = value / 2 if value < 0 else value
    lab[:], idx[:] = 2, [0, 1, 2, 3]
    for T in (1.0, 2.0, 3.0, 4.0, 0.25):
        run_case(z, lab, idx, val, T)


@pytest.mark.parametrize("T", [1.0, 2.0, 4.0, 2.5])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_far_from_zero(T, dtype):
    """A maximum of some thousands is taken off before anything is rounded away."""
    z, lab, idx, val = inputs(5, 3001, 6, "f32", 14)
    z = (z + np.array([[5000.0], [-5000.0], [1e6], [-3e7], [123.4]])).astype(np.float32)
    if dtype == "bf16":
        z, val = oracle.bf16_round(z), oracle.bf16_round(val)
    run_case(z, lab, idx, val, T, dtype=dtype)


@pytest.mark.parametrize("V", [40, 5003, 70001])
def test_a_logit_that_is_no_number_spoils_its_row_alone(V):
    z, lab, idx, val = inputs(3, V, 4, "f32", 6)
    lab[:], idx[:] = 1, [4, 7, 9, 11]
    z[1, V - 1] = NAN
    loss, dz = hp.distill_loss_fwd_bwd(dev(z), labels=dev(lab), top_idx=dev(idx), top_val=dev(val))
    assert torch.isnan(loss[1]) and torch.isnan(dz[1]).all()
    assert torch.isfinite(loss[[0, 2]]).all() and torch.isfinite(dz[[0, 2]]).all()


@pytest.mark.parametrize("V", [64, 5000, 70000])
def test_classes_named_twice_and_indexes_that_name_none(V):
    z, lab, idx, val = inputs(4, V, 9, "f32", 7)
    idx[:] = [5, 5, 5, -1, V, V - 1, 2, V - 1, -2 ** 31]
    lab[:] = [5, V, -1, V - 1]
    run_case(z, lab, idx, val, 2.0)
    wide = idx.astype(np.int64)
    wide[:, 3], wide[:, 4] = 2 ** 32 + 1, -2 ** 40
    run_case(z, lab, wide, val, 2.0, wide=True)


@pytest.mark.parametrize("T", [0.05, 0.5, 20.0, 1000.0])
@pytest.mark.parametrize("std", [1e-3, 30.0, 1e4])
def test_temperatures_and_magnitudes(T, std):
    z, lab, idx, val = inputs(6, 777, 8, "f32", 8, std=std)
    run_case(z, lab, idx, val, T, 0.5, 0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 5, 1000, 4099, 70003])
def test_rows_apart_and_unaligned(V, dtype):
    """Logits and gradient as column slices of wider buffers: the rest stays as it is."""
    N, K, pad = 4, min(V, 6), 5
    z, lab, idx, val = inputs(N, V, K, dtype, 9)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    wide = torch.full((N, V + pad), NAN, dtype=td, device="cuda")
    wide[:, 3:3 + V] = dev(z, dtype)
    zd = wide[:, 3:3 + V]
    run_case(z, lab, idx, val, 2.0, 1.0, 1.0, dtype, zd=zd)
    out = torch.full((N, V + pad + 2), 7.0, dtype=td, device="cuda")
    args = dict(labels=dev(lab), top_idx=dev(idx), top_val=dev(val, dtype), temperature=2.0)
    want = hp.distill_loss_fwd_bwd(dev(z, dtype), **args)
    got = hp.distill_loss_fwd_bwd(zd, **args, dz=out[:, 1:1 + V])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert bool((out[:, :1] == 7.0).all()) and bool((out[:, 1 + V:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(7, 1000), (1, 9001), (5, 70001), (600, 300)])
def test_gradient_in_place_of_the_logits(N, V, dtype):
    z, lab, idx, val = inputs(N, V, 6, dtype, 10)
    args = dict(labels=dev(lab), top_idx=dev(idx), top_val=dev(val, dtype), temperature=2.0)
    want = hp.distill_loss_fwd_bwd(dev(z, dtype), **args)
    zd = dev(z, dtype)
    got = hp.distill_loss_fwd_bwd(zd, **args, dz=zd)
    assert torch.equal(got[0], want[0]) and torch.equal(zd, want[1])
    zd = dev(z, dtype)
    loss, stats = hp.distill_loss_fwd(zd, **args)
    apart = hp.distill_loss_bwd(zd, stats, **args)
    hp.distill_loss_bwd(zd, stats, **args, dz=zd)
    assert torch.equal(zd, apart)


@pytest.mark.parametrize("N,V", [(40, 1000), (3, 70001), (2000, 100)])
def test_same_bits_every_time(N, V):
    z, lab, idx, val = inputs(N, V, 20, "f32", 11)
    idx[:, 3] = idx[:, 1]
    args = dict(labels=dev(lab), top_idx=dev(idx), top_val=dev(val), temperature=2.0)
    first = hp.distill_loss_fwd_bwd(dev(z), **args)
    for _ in range(3):
        again = hp.distill_loss_fwd_bwd(dev(z), **args)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_no_rows():
    z = torch.empty((0, 10), device="cuda")
    lab = torch.empty((0,), dtype=torch.int64, device="cuda")
    loss, stats = hp.distill_loss_fwd(z, labels=lab)
    dz = hp.distill_loss_bwd(z, stats, labels=lab)
    both = hp.distill_loss_fwd_bwd(z, labels=lab)
    assert loss.shape == (0,) and dz.shape == (0, 10) and both[1].shape == (0, 10)


def test_on_another_stream_and_in_a_graph():
    for N, V in ((64, 1000), (3, 70001)):
        z, lab, idx, val = inputs(N, V, 10, "f32", 12)
        zd, ws = dev(z), hp.Workspace()
        args = dict(labels=dev(lab), top_idx=dev(idx), top_val=dev(val), temperature=4.0, grad_scale=1.0 / N)
        want = hp.distill_loss_fwd_bwd(zd, **args)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = hp.distill_loss_fwd_bwd(zd, **args, ws=ws)
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, got))
        loss, dz = torch.empty_like(want[0]), torch.empty_like(want[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            hp.distill_loss_fwd_bwd(zd, **args, loss=loss, dz=dz, ws=ws)
        for _ in range(3):
            loss.fill_(NAN)
            dz.fill_(NAN)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(loss, want[0]) and torch.equal(dz, want[1])


def test_offsets_past_32_bits():
    """More than 2^32 bytes of logits: the last rows are what they are alone."""
    N, V = 17000, 65536                                               # 4.5 GB
    z = torch.zeros((N, V), device="cuda")
    z[-3:].normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    lab = torch.full((N,), -1, device="cuda")
    lab[-3:] = torch.tensor([0, 65535, 77])
    want = hp.distill_loss_fwd_bwd(z[-3:].clone(), labels=lab[-3:].clone())
    loss, dz = hp.distill_loss_fwd_bwd(z, labels=lab, dz=z)
    assert not loss[:-3].any() and not dz[:-3].any()
    assert torch.allclose(loss[-3:], want[0], rtol=1e-6) and torch.allclose(dz[-3:], want[1], rtol=1e-4, atol=1e-9)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 5003, 70001])
@pytest.mark.parametrize("value", [1e8, 1e9, -1e9, 1e10, -1e10, 1e12, -1e15, 1e20, -1e20, 1e28, -1e28])
def test_even_rows_of_large_logits(V, value, dtype):
    """Rows of one value, with and without a class above it, at magnitudes whose products with log2 e have no small rounding."""
    z, lab, idx, val = inputs(4, V, 4, "f32", 15)
    z[:2] = value
    z[1, 2] = value + abs(value) / 2
    lab[:], idx[:] = 2, [0, 1, 2, 3]
    if dtype == "bf16":
        z, val = oracle.bf16_round(z), oracle.bf16_round(val)
    for T in (1.0, 1.5, 2.0, 4.0, 0.05, 0.01):
        run_case(z, lab, idx, val, T, dtype=dtype)


@pytest.mark.parametrize("V,first,last", [(5003, 0, 4200), (5003, 900, 5003), (70001, 0, 40000), (70001, 20000, 70001)])
@pytest.mark.parametrize("low", [-1e9, -1e10, -1e20, -1e28])
def test_classes_left_out_side_by_side(V, first, last, low):
    """Whole wavefronts and parts of a row at a large negative value, beside ordinary logits."""
    z, lab, idx, val = inputs(5, V, 4, "f32", 16)
    z[:, first:last] = low
    free = np.setdiff1d(np.arange(V), np.arange(first, last))
    idx = np.where(idx >= 0, free[idx % free.size], -1)
    lab = np.where(lab >= 0, free[lab % free.size], -1)
    for T in (1.0, 2.0, 4.0, 0.7):
        stats, loss, dz, _ = run_case(z, lab, idx, val, T)
        assert torch.isfinite(loss).all() and not dz[:, first:last].any()


@pytest.mark.parametrize("V", [40, 5003, 70001])
def test_a_term_of_weight_zero_is_absent_whatever_its_logits(V):
    """Classes at -infinity that only the term of weight zero names: the other term is what it is without that one."""
    z, lab, idx, val = inputs(5, V, 4, "f32", 17)
    lab[:], idx[:] = [1, 2, 3, V - 1, 1], [5, 6, 7, 8]
    for out, wk, wl in (([5, 8], 0.0, 0.6), ([1, 2, 3, V - 1], 0.6, 0.0)):
        y = z.copy()
        y[:, out] = -INF
        alone = (lab, None, None) if wk == 0.0 else (None, idx, val)
        _, loss, dz, _ = run_case(y, *alone, 2.0, wk, wl)
        args = dict(labels=dev(lab), top_idx=dev(idx), top_val=dev(val), temperature=2.0, kd_weight=wk, label_weight=wl)
        both = hp.distill_loss_fwd_bwd(dev(y), **args)
        got, stats = hp.distill_loss_fwd(dev(y), **args)
        assert torch.equal(got, loss) and torch.equal(both[0], loss)
        assert torch.equal(hp.distill_loss_bwd(dev(y), stats, **args), dz) and torch.isfinite(dz).all()
