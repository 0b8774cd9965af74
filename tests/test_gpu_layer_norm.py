"""Layer normalisation on the GPU against the oracle in 64 bits, element by element.

The bounds: u = 2^-24 is one fp32 rounding.  A row's sum is taken in chains of at most 32 values joined in trees of at most
ten levels, or in 64 bits: below 64 u of the sum of magnitudes.  A column's sum runs over at most 256 rows one after the other
in fp32 and 16 such sums side by side, then in 64 bits: below (256 + 16) u.  Everything else is a handful of roundings.  A
result stored as bfloat16 adds 2^-8 of itself."""
import numpy as np
import pytest
import torch

import oracle
from paper_1312_5853_amd import binding as hp

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SUM = 64 * U
TINY = 1e-37
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _values(shape, dtype, g, mean=0.0, std=1.0):
    a = (mean + std * g.standard_normal(shape) * (0.5 + g.random((1, shape[1])))).astype(np.float32)
    return oracle.bf16_round(a) if dtype == "bf16" else a


def _dev(a, dtype="f32", pitch=0, off=0):
    """On the GPU, rows `pitch` elements apart and `off` elements into its memory; what lies between them is not zero."""
    N, C = a.shape
    pitch = pitch or C
    buf = torch.full((off + max(N, 1) * pitch,), 77.0, dtype=DTYPES[dtype], device="cuda")
    t = buf[off:off + N * pitch].view(N, pitch)[:, :C]
    t.copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)))
    return t


def _vec(v):
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).cuda()


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _store(v, dtype):
    return np.abs(v) * (2.0 ** -8 if dtype == "bf16" else 2 * U)


def _within(got, want, bound):
    err = np.abs(got - want)
    assert (err <= bound + TINY).all(), (err / (bound + TINY)).max()


def check_fwd(got, x, gamma, beta, eps, dtype):
    y, mean, rstd = map(_host, got)
    wy, wm, wr = oracle.layer_norm_fwd(x, gamma, beta, eps)
    x = x.astype(np.float64)
    big = np.abs(x).mean(1)
    e_mean = SUM * big + 2 * U * np.abs(wm)
    var = 1.0 / wr ** 2
    e_rstd = wr * ((e_mean ** 2 + SUM * var + 4 * U * np.sqrt(var) * (big + np.abs(wm))) / var / 2 + 4 * U)
    _within(mean, wm, e_mean)
    _within(rstd, wr, e_rstd)
    d, c = np.abs(x - wm[:, None]), lambda v: v[:, None]
    e = np.abs(gamma) * (c(wr) * (c(e_mean) + 2 * U * np.abs(x)) + d * c(e_rstd)) + 16 * U * (d * c(wr) * np.abs(gamma) + np.abs(beta))
    _within(y, wy, e + _store(wy, dtype))


def check_bwd(got, x, dy, mean, rstd, gamma, dtype):
    dx, dgamma, dbeta = map(_host, got)
    wx, wg, wb = oracle.layer_norm_bwd(x, dy, mean, rstd, gamma)
    x, dy, c = x.astype(np.float64), dy.astype(np.float64), lambda v: np.asarray(v, np.float64)[:, None]
    xh = np.abs(x - c(mean)) * c(rstd)
    e_xh = 4 * U * xh
    g = np.abs(dy * gamma)
    col = (min(len(x), 256) + 16) * U
    _within(dbeta, wb, col * np.abs(dy).sum(0) + 2 * U * np.abs(wb))
    _within(dgamma, wg, (col + 6 * U) * (np.abs(dy) * xh).sum(0) + 2 * U * np.abs(wg))
    a1, a2 = g.mean(1), (g * xh).mean(1)
    e = c(rstd) * (4 * U * g + c((SUM + 4 * U) * a1) + xh * c((SUM + 10 * U) * a2) + e_xh * c(a2) + 8 * U * (g + c(a1) + xh * c(a2)))
    _within(dx, wx, e + _store(wx, dtype))


def run_case(N, C, dtype, seed=0, mean=0.0, std=1.0, eps=1e-5, affine=True, pitch=0, off=0):
    g = np.random.Generator(np.random.Philox(seed))
    x, dy = _values((N, C), dtype, g, mean, std), _values((N, C), dtype, g)
    gamma, beta = (1.0 + 0.3 * g.standard_normal(C)).astype(np.float32), (0.3 * g.standard_normal(C)).astype(np.float32)
    if not affine:
        gamma, beta = np.ones(C, np.float32), np.zeros(C, np.float32)
    ga, be = (_vec(gamma), _vec(beta)) if affine else (None, None)
    xd, dyd = _dev(x, dtype, pitch, off), _dev(dy, dtype, pitch and pitch + 1, off)
    out = lambda: _dev(np.full((N, C), np.nan), dtype, pitch and pitch + 2, off)
    check_fwd(hp.layer_norm_fwd(xd, ga, be, eps=eps, y=out()), x, gamma, beta, eps, dtype)
    _, m, r = oracle.layer_norm_fwd(x, gamma, beta, eps)
    m, r = m.astype(np.float32), r.astype(np.float32)
    check_bwd(hp.layer_norm_bwd(xd, dyd, _vec(m), _vec(r), ga, dx=out()), x, dy, m, r, gamma, dtype)
    # the same from 8 bits
    q = hp.quantize_blocks(xd, "e4m3")
    held = oracle.dequantize_blocks(*oracle.quantize_blocks(x, "e4m3"), C, "e4m3")
    check_bwd(hp.layer_norm_bwd_kept(q, dyd, _vec(m), _vec(r), ga, dx=out()), held, dy, m, r, gamma, dtype)


# N, C: one value, less than a vector, one more; a wavefront's worth of vectors and one more; several rows to a work-group; rows of
# several vectors to a thread and of several wavefronts; the longest that a work-group keeps, forward and backward, and longer
# ones; more rows than work-groups
SHAPES = [(1, 1), (3, 1), (1, 2), (5, 3), (2, 5), (2, 7), (4, 8), (3, 9), (7, 64), (300, 65), (9, 127), (33, 255), (2, 256), (5, 257),
          (3, 511), (2, 513), (3, 1003), (2, 1024), (11, 1025), (5, 2049), (2, 4096), (1, 4097), (3, 5003), (2, 8200), (4, 9216),
          (2, 16384), (3, 16385), (2, 20001), (2, 32768), (2, 32769), (3, 40001), (1, 70000), (5003, 33), (1100, 520), (700, 4099),
          (2100, 1000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C", SHAPES)
def test_against_the_oracle(N, C, dtype):
    run_case(N, C, dtype, seed=N + 7 * C)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C", [(5, 1), (6, 100), (4, 1001), (3, 5000), (2, 33001), (601, 70)])
def test_rows_apart_at_any_address(N, C, dtype):
    run_case(N, C, dtype, seed=C, pitch=C + 3, off=1)


@pytest.mark.parametrize("C", [7, 300, 5001, 40001])
@pytest.mark.parametrize("mean,std", [(1e4, 1.0), (-300.0, 1e-2), (1e-20, 1e-20), (1e15, 1e13), (2.0, 0.0)])
def test_means_far_from_zero_and_extreme_scales(mean, std, C):
    """The variance comes from distances to the mean: values of 10000 +- 1 keep it."""
    run_case(3, C, "f32", seed=6, mean=mean, std=std)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_scale_and_shift(dtype):
    run_case(4, 130, dtype, seed=7, affine=False)
    run_case(2, 33000, dtype, seed=8, affine=False)


@pytest.mark.parametrize("C", [50, 3000, 33001])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_value_that_is_no_number_stays_in_its_row(bad, C):
    g = np.random.Generator(np.random.Philox(9))
    x, dy = _dev(_values((5, C), "f32", g)), _dev(_values((5, C), "f32", g))
    want = hp.layer_norm_fwd(x)
    back = hp.layer_norm_bwd(x, dy, want[1], want[2])
    x[2, C // 2] = bad
    got = hp.layer_norm_fwd(x)
    gb = hp.layer_norm_bwd(x, dy, got[1], got[2])
    rest = [0, 1, 3, 4]
    for a, b in ((got[0], want[0]), (gb[0], back[0])):
        assert torch.isnan(a[2]).all() and torch.equal(a[rest], b[rest])
    assert torch.isnan(gb[1]).all() and torch.equal(gb[2], back[2])      # the row's values are in every column's sum


def test_empty_batch():
    x = torch.zeros((0, 40), device="cuda")
    y, mean, rstd = hp.layer_norm_fwd(x)
    assert y.shape == (0, 40) and mean.shape == (0,)
    for call in (lambda **k: hp.layer_norm_bwd(x, x, mean, rstd, **k),
                 lambda **k: hp.layer_norm_bwd_kept(hp.Blocks.empty(0, 40, "e4m3"), x, mean, rstd, **k)):
        dg, db = torch.full((40,), 7.0, device="cuda"), torch.full((40,), 7.0, device="cuda")
        call(dgamma=dg, dbeta=db)
        assert not dg.any() and not db.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C", [(3, 5), (4, 130), (2, 5003), (2, 33003), (601, 70)])
def test_nothing_outside_the_outputs_is_written(N, C, dtype):
    g = np.random.Generator(np.random.Philox(10))
    x, dy = _dev(_values((N, C), dtype, g), dtype), _dev(_values((N, C), dtype, g), dtype)
    pitch, td = C + 5, DTYPES[dtype]
    _, mean, rstd = hp.layer_norm_fwd(x)
    q = hp.quantize_blocks(x, "e4m3")
    for call in (lambda o: hp.layer_norm_fwd(x, y=o), lambda o: hp.layer_norm_bwd(x, dy, mean, rstd, dx=o),
                 lambda o: hp.layer_norm_bwd_kept(q, dy, mean, rstd, dx=o)):
        buf = torch.full((3 + N * pitch + 64,), 7.0, dtype=td, device="cuda")
        out = buf[3:3 + N * pitch].view(N, pitch)[:, :C]
        out.fill_(float("nan"))
        call(out)
        assert not torch.isnan(out).any()
        out.fill_(7.0)
        assert (buf == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C", [(50, 300), (1300, 1000), (6, 40000)])
def test_the_same_bits_every_time(N, C, dtype):
    g = np.random.Generator(np.random.Philox(11))
    x, dy = _dev(_values((N, C), dtype, g), dtype), _dev(_values((N, C), dtype, g), dtype)
    first = hp.layer_norm_fwd(x)
    back = hp.layer_norm_bwd(x, dy, first[1], first[2])
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(hp.layer_norm_fwd(x), first))
        assert all(torch.equal(a, b) for a, b in zip(hp.layer_norm_bwd(x, dy, first[1], first[2]), back))


def test_columns_over_many_rows():
    """A column of ones among many rows: its sums stay exact, 2^20 rows long."""
    N = 1 << 20
    x = torch.zeros((N, 4), device="cuda")
    x[:, 0] = 1.0
    dy = torch.ones((N, 4), device="cuda")
    mean, rstd = torch.zeros(N, device="cuda"), torch.ones(N, device="cuda")
    dx, dgamma, dbeta = hp.layer_norm_bwd(x, dy, mean, rstd)
    assert dbeta.tolist() == [N] * 4 and dgamma.tolist() == [N, 0, 0, 0]


def test_columns_of_rows_longer_than_a_work_group_keeps_over_many():
    """4096 times 1 + 0.75 2^-17, each sum of a thread over 256 of them: one after the other in fp32, from 128 on every one would lose
    what it has behind the 1, 2^-18.7 of the result.  Four are summed in fp32 (3 u), then in 64 bits but for a rounding to a part's
    32 bits, one to a work-group's and one of the result."""
    N, C, v = 4096, 131072, 1 + 0.75 * 2.0 ** -17
    x, dy = torch.zeros((N, C), device="cuda"), torch.full((N, C), v, device="cuda")
    dx, dgamma, dbeta = hp.layer_norm_bwd(x, dy, torch.full((N,), -1.0, device="cuda"), torch.ones(N, device="cuda"))
    for got in (dgamma, dbeta):
        assert (np.abs(_host(got) - N * v) <= 6 * U * N * v).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C", [(3, 1), (3, 5), (2, 9), (4, 300), (2, 4096), (2, 4100), (3, 5003), (2, 9217), (2, 16001), (2, 33000),
                                 (3, 33003), (700, 301), (700, 4099), (4100, 4099), (700, 9217), (700, 16001)])
def test_rows_whose_mean_times_rstd_is_past_fp32(N, C, dtype):
    """2^110 throughout, with the statistics of eps = 1e-12: every distance from the mean is zero and so is xh, whatever the threads
    without a value of the row make of the mean, -2^110 1e6 = -1.3e39."""
    g = np.random.Generator(np.random.Philox(C))
    x, dy = np.full((N, C), 2.0 ** 110, np.float32), _values((N, C), dtype, g)
    gamma = (1.0 + 0.3 * g.standard_normal(C)).astype(np.float32)
    xd, dyd = _dev(x, dtype), _dev(dy, dtype)
    _, m, r = hp.layer_norm_fwd(xd, eps=1e-12)
    mean, rstd = _host(m).astype(np.float32), _host(r).astype(np.float32)
    assert (mean == 2.0 ** 110).all() and (np.abs(rstd - 1e6) <= 1).all()
    check_bwd(hp.layer_norm_bwd(xd, dyd, m, r, _vec(gamma)), x, dy, mean, rstd, gamma, dtype)
    check_bwd(hp.layer_norm_bwd_kept(hp.quantize_blocks(xd, "e4m3"), dyd, m, r, _vec(gamma)), x, dy, mean, rstd, gamma, dtype)


# more rows than take their columns' sums in the same launch, of 8193 to 12288 values (16 to a thread with the sums) and of more (24, the
# columns in a launch of their own)
MANY = [(700, 9216), (1301, 8200), (650, 12288), (645, 12287), (700, 16001), (641, 18432)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C", MANY)
def test_many_long_rows(N, C, dtype, block_plans):
    p, V = block_plans.layer_norm(hp.OP_BWD_DATA, N, C, 0 if dtype == "f32" else 1), 4 if dtype == "f32" else 8
    assert not p["wide"] and not p["columns"] and p["apart"] == (C > 12288) and p["regs"] * V == (24 if C > 12288 else 16)
    assert p["blocks"] < N                                           # some work-groups take several rows
    run_case(N, C, dtype, seed=N + C)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C", [(5, 300), (900, 70), (700, 5003), (700, 16001), (300, 20001)])
def test_sums_and_statistics_that_nobody_wants(N, C, dtype):
    """Through the C calls: NULL for dgamma, dbeta, or both, for mean and rstd of the forward pass, and no scratch where no sums are
    made.  What is written is what a call for everything writes."""
    g = np.random.Generator(np.random.Philox(N))
    x, dy = _dev(_values((N, C), dtype, g), dtype), _dev(_values((N, C), dtype, g), dtype)
    code, lib, stream = 0 if dtype == "f32" else 1, hp.lib(), torch.cuda.current_stream().cuda_stream
    gamma, ptr = _vec(1.0 + 0.3 * g.standard_normal(C)), lambda t: 0 if t is None else t.data_ptr()
    want = hp.layer_norm_fwd(x, gamma)
    for keep in ((False, False), (True, False), (False, True)):
        y = torch.full_like(x, float("nan"))
        stats = [torch.full((N,), float("nan"), device="cuda") if k else None for k in keep]
        assert lib.layer_norm_fwd(x.data_ptr(), C, gamma.data_ptr(), 0, y.data_ptr(), C, ptr(stats[0]), ptr(stats[1]), N, C, 1e-5, code,
                                  stream) == hp.OK
        assert torch.equal(y, want[0]) and all(s is None or torch.equal(s, w) for s, w in zip(stats, want[1:]))
    mean, rstd = want[1:]
    q = hp.quantize_blocks(x, "e4m3")
    need = lib.layer_norm_workspace_bytes(hp.OP_BWD_DATA, N, C, code)
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    for name, source, whole in (("layer_norm_bwd", (x.data_ptr(), C), hp.layer_norm_bwd(x, dy, mean, rstd, gamma)),
                                ("layer_norm_bwd_kept", (q.codes.data_ptr(), q.scales.data_ptr()),
                                 hp.layer_norm_bwd_kept(q, dy, mean, rstd, gamma))):
        for keep in ((False, False), (True, False), (False, True)):
            dx = torch.full_like(x, float("nan"))
            sums = [torch.full((C,), float("nan"), device="cuda") if k else None for k in keep]
            scratch = (ws.data_ptr(), need) if any(keep) else (0, 0)
            assert getattr(lib, name)(*source, dy.data_ptr(), C, gamma.data_ptr(), mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), C,
                                      ptr(sums[0]), ptr(sums[1]), N, C, code, *scratch, stream) == hp.OK
            # (dx by another form of the kernel, whose sums the compiler may contract elsewhere)
            assert all(s is None or torch.equal(s, w) for s, w in zip(sums, whole[1:]))
            m, r = _host(mean), _host(rstd)
            src = _host(x) if name == "layer_norm_bwd" else _host(hp.dequantize_blocks(q))
            zero = [torch.from_numpy(v).float().cuda() for v in oracle.layer_norm_bwd(src, _host(dy), m, r, _host(gamma))[1:]]
            check_bwd((dx, *zero), src, _host(dy), m, r, _host(gamma), dtype)


@pytest.mark.parametrize("N,C", [(4095, 4097), (4096, 4097), (4099, 5003), (4200, 8192)])
def test_two_rows_at_a_time(N, C):
    """bfloat16 rows of 4097 to 8192 values, from 4096 rows on two at a time."""
    run_case(N, C, "bf16", seed=N)
