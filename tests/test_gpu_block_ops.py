"""Tensors held in blocks of 8 and 4 bits on the GPU, the filter gradient and the forward pass of a fully connected layer on
them, against the oracle in 64 bits.

Codes, exponents and the values read back are compared bit for bit.  The bounds of the products: u = 2^-24 is one fp32
rounding; every single product is exact, and a sum of n of them, in whatever order the matrix instructions take it, with every
addition rounded or cut off (2 u), is within 2 u n of the sum of magnitudes.  A result stored as bfloat16 adds 2^-8 of itself."""
import numpy as np
import pytest
import torch

import oracle
from paper_1312_5853_amd import binding as hp

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FORMS = ["e4m3", "e2m1"]
RNG = lambda s: np.random.Generator(np.random.Philox(s))


def _values(shape, dtype, seed, std=1.0):
    g = RNG(seed)
    a = (std * g.standard_normal(shape) * np.exp2(g.integers(-6, 6, (shape[0], 1)))).astype(np.float32)
    a[g.random(shape) < 0.2] = 0.0
    return oracle.bf16_round(a) if dtype == "bf16" else a


def _dev(a, dtype="f32", pitch=0, off=0):
    N, C = a.shape
    pitch = pitch or C
    buf = torch.full((off + max(N, 1) * pitch,), 77.0, dtype=DTYPES[dtype], device="cuda")
    t = buf[off:off + N * pitch].view(N, pitch)[:, :C]
    t.copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)))
    return t


def _held(a, form):
    """An array in blocks on the GPU, made by the oracle, and its values."""
    codes, scales = oracle.quantize_blocks(a, form)
    q = hp.Blocks(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), a.shape[1], form)
    return q, oracle.dequantize_blocks(codes, scales, a.shape[1], form)


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def check_blocks(x, form, dtype, **place):
    N, C = x.shape
    q = hp.Blocks.empty(N, C, form)
    q.codes.fill_(0xA5)
    q.scales.fill_(0xA5)
    assert hp.quantize_blocks(_dev(x, dtype, **place), form, out=q) is q
    codes, scales = oracle.quantize_blocks(x, form)
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(q.codes.cpu().numpy(), codes)
    want = oracle.dequantize_blocks(codes, scales, C, form)
    for d in ("f32", "bf16"):
        out = _dev(np.full((N, C), 5.0), d, **place)
        assert hp.dequantize_blocks(q, x=out) is out
        with np.errstate(over="ignore"):
            assert np.array_equal(_host(out), want.astype(np.float32).astype(np.float64), equal_nan=True)
    return q


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("N,C", [(1, 1), (3, 2), (2, 7), (5, 8), (4, 31), (3, 32), (2, 33), (7, 100), (2, 127), (9, 128), (3, 129), (1, 2048),
                                 (2, 2049), (130, 40), (33, 1000), (17, 4097), (1, 70001)])
def test_blocks_bit_for_bit(N, C, form, dtype):
    check_blocks(_values((N, C), dtype, N * 1000 + C), form, dtype)
    if C > 4:
        check_blocks(_values((N, C), dtype, N * 1000 + C), form, dtype, pitch=C + 3, off=1)


@pytest.mark.parametrize("form", FORMS)
def test_every_magnitude(form):
    """Every exponent of fp32, normal and not, ties, zeros of both signs, the largest finite values, infinities and NaN."""
    g = RNG(1)
    x = (g.uniform(1, 2, (255, 96)) * np.where(g.random((255, 96)) < 0.5, -1, 1)).astype(np.float32)
    x = np.ldexp(x, np.arange(-127, 128)[:, None] + g.integers(-14, 1, (255, 96))).astype(np.float32)
    x[:, 5], x[:, 40] = 0.0, -0.0
    check_blocks(x, form, "f32")
    steps = np.concatenate([oracle.block_magnitudes(form), (oracle.block_magnitudes(form)[1:] + oracle.block_magnitudes(form)[:-1]) / 2])
    ties = np.zeros((len(steps), 64), np.float32)
    ties[:, 0], ties[:, 1], ties[:, 2] = oracle.block_magnitudes(form)[-1], steps, -steps
    ties[:, 32:] = np.ldexp(ties[:, :32], -30)
    check_blocks(ties, form, "f32")
    odd = np.ones((8, 40), np.float32)
    odd[0, 3], odd[1, 35], odd[2, 0], odd[3, 39] = np.inf, np.nan, -np.inf, np.nan
    odd[4, 1], odd[5, 33], odd[6, :], odd[7, 2] = 3.4028235e38, -3.4028235e38, 1e-45, np.float32(2.0 ** 126)
    check_blocks(odd, form, "f32")


def test_empty_and_untouched():
    for form in FORMS:
        q = hp.quantize_blocks(torch.zeros((0, 9), device="cuda"), form)
        assert q.shape == (0, 9) and hp.dequantize_blocks(q).shape == (0, 9)
        x = torch.full((4, 50), 7.0, device="cuda")
        hp.dequantize_blocks(hp.quantize_blocks(torch.ones((4, 45), device="cuda"), form), x=x[:, :45])
        assert (x[:, :45] == 1.0).all() and (x[:, 45:] == 7.0).all()


# --------------------------------------------------------- the filter gradient
def check_grad(x, dy, dtype):
    q, held = _held(x, "e4m3")
    dw = torch.full((dy.shape[1], x.shape[1]), float("nan"), device="cuda")
    got = _host(hp.fc_bwd_filter_kept(q, _dev(dy, dtype), dw=dw))
    dy = dy.astype(np.float64)
    want, size = dy.T @ held, np.abs(dy).T @ np.abs(held)
    n = len(x) * (3 if dtype == "f32" else 1) + 64                   # products, and the joins of the sum's parts
    err = np.abs(got - want)
    assert (err <= 2 * U * n * size + 1e-37).all(), (err / (2 * U * n * size + 1e-37)).max()
    return got


GRADS = [(1, 1, 1), (1, 130, 5), (2, 32, 33), (3, 7, 300), (15, 127, 31), (16, 128, 128), (17, 129, 127), (31, 64, 129), (32, 300, 257),
         (33, 255, 256), (64, 256, 255), (65, 520, 100), (128, 384, 640), (129, 1000, 70), (500, 40, 24), (1000, 96, 1000), (3000, 130, 130),
         (9001, 33, 5)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", GRADS)
def test_filter_gradient(N, I, O, dtype):
    check_grad(_values((N, I), dtype, N + I), _values((N, O), dtype, N + O, 1e-3), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("O", [1, 2, 3, 4, 7])
@pytest.mark.parametrize("N", [129, 160, 263, 1280])
def test_filter_gradient_of_fewer_outputs_than_a_load_takes(N, O, dtype):
    check_grad(_values((N, 70), dtype, N + 70), _values((N, O), dtype, N + O, 1e-3), dtype)


@pytest.mark.parametrize("off", [0, 1, 8, 32])
@pytest.mark.parametrize("N,I,O", [(40, 128, 70), (128, 160, 260), (7, 96, 31), (300, 128, 130)])
def test_filter_gradient_at_any_address(N, I, O, off):
    """Whole cache lines of the result and parts of them; whole numbers, whose sums are exact."""
    g = np.random.Generator(np.random.Philox(N + off))
    x, dy = (g.integers(-4, 5, (N, k)).astype(np.float32) for k in (I, O))
    buf = torch.full((off + O * I + 40,), 7.0, device="cuda")
    hp.fc_bwd_filter_kept(_held(x, "e4m3")[0], _dev(dy), dw=buf[off:off + O * I].view(O, I))
    got = _host(buf)
    assert np.array_equal(got[off:off + O * I].reshape(O, I), dy.T.astype(np.float64) @ x)
    assert (got[:off] == 7).all() and (got[off + O * I:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", [(5, 40, 9), (130, 300, 260), (4100, 64, 100)])
def test_filter_gradient_of_whole_numbers_is_exact(N, I, O, dtype):
    """Sums of products of small whole numbers are whole numbers below 2^24."""
    g = RNG(N)
    x, dy = g.integers(-8, 9, (N, I)).astype(np.float32), g.integers(-16, 17, (N, O)).astype(np.float32)
    q, held = _held(x, "e4m3")
    assert np.array_equal(held, x)
    assert np.array_equal(_host(hp.fc_bwd_filter_kept(q, _dev(dy, dtype))), dy.astype(np.float64).T @ x)


def test_filter_gradient_keeps_every_bit_of_fp32():
    """One sample of ones: dw is dy, whatever its magnitude; 24 bits of it, far ones too.  The last of the three parts holds
    what lies 2^-23 of a value's leading bit and above in steps of 2^-133 at least, bfloat16's least: values from 2^-110 on
    (2^-110 2^-23 = 2^-133) are held exactly, and of smaller ones less than 2^-133 is cut off."""
    g = RNG(2)
    dy = np.ldexp(g.uniform(1, 2, (1, 254)), np.arange(-126, 128)).astype(np.float32)
    dy[0, :3] = 3.4028235e38, -3.4028235e38, 1.1754944e-38
    q, _ = _held(np.ones((1, 70), np.float32), "e4m3")
    got = hp.fc_bwd_filter_kept(q, _dev(dy)).cpu().numpy()
    far = np.abs(dy[0]) >= 2.0 ** -110
    assert np.array_equal(got[far], np.repeat(dy.T[far], 70, axis=1))
    assert (np.abs(got.astype(np.float64) - dy.T.astype(np.float64)) < 2.0 ** -133).all(axis=1)[~far].all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_no_numbers_in_the_gradient(dtype):
    x, dy = np.ones((70, 200), np.float32), np.ones((70, 90), np.float32)
    dy[3, 5], dy[60, 7], dy[1, 80] = np.inf, -np.inf, np.nan
    got = _host(hp.fc_bwd_filter_kept(_held(x, "e4m3")[0], _dev(dy, dtype)))
    assert (got[5] == np.inf).all() and (got[7] == -np.inf).all() and np.isnan(got[80]).all()
    rest = [o for o in range(90) if o not in (5, 7, 80)]
    assert (got[rest] == 70).all()
    x[9, 40] = np.nan                                              # block 1 of sample 9 is no number
    got = _host(hp.fc_bwd_filter_kept(_held(x, "e4m3")[0], _dev(np.ones((70, 90), np.float32), dtype)))
    assert np.isnan(got[:, 32:64]).all() and (got[:, :32] == 70).all() and (got[:, 64:] == 70).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", [(1, 40, 33), (15, 70, 90), (16, 64, 32), (17, 130, 20), (100, 200, 40), (128, 64, 129), (129, 130, 70),
                                   (160, 70, 7), (300, 150, 200), (3000, 130, 130), (1030, 4000, 4003)])
def test_infinite_inputs_in_the_gradient(N, I, O, dtype):
    """A value that comes back as an infinity (3.4e38 is past 248 2^120, half way to 2^128) makes its column what the formula makes
    of it: an infinity of the gradient's sign, no number where the gradient is zero or two of them have different signs."""
    g = RNG(N + I)
    x, dy = _values((N, I), dtype, N + I), _values((N, O), dtype, N + O, 1e-3)
    dy[:, ::3] = g.choice([0.0, 0.5, -1.0, 2.0, 3.0], (N, len(dy[0, ::3])))       # their second and third parts are zero
    big = np.float32(3.4e38) if dtype == "f32" else oracle.bf16_round(np.float32([3.38e38]))[0]
    x[N - 1, I // 2] = big
    x[0, I - 1], x[N // 2, I - 1], x[N // 3, 3] = big, -big, -big
    q, held = _held(x, "e4m3")
    with np.errstate(over="ignore", invalid="ignore"):
        held = held.astype(np.float32).astype(np.float64)
        columns = np.flatnonzero(np.isinf(held).any(axis=0))
        assert {3, I // 2, I - 1} == set(columns.tolist())
        got = _host(hp.fc_bwd_filter_kept(q, _dev(dy, dtype)))
        d = dy.astype(np.float64)
        for i in columns:
            want = (d * held[:, i:i + 1]).sum(axis=0)
            assert not np.isfinite(want).any() and np.array_equal(got[:, i], want, equal_nan=True), i
    rest = np.setdiff1d(np.arange(I), columns)
    want, size = d.T @ held[:, rest], np.abs(d).T @ np.abs(held[:, rest])
    assert (np.abs(got[:, rest] - want) <= 2 * U * (N * (3 if dtype == "f32" else 1) + 64) * size + 1e-37).all()


# whole numbers, which the sums keep exactly, in random places: a step's values in another's buffer would show
FEW_STEPS = [(1, 9216, 4096), (9, 9217, 4001), (20, 9216, 4096), (50, 9216, 4096), (64, 9250, 4100), (100, 9230, 4096), (128, 9216, 4096),
             (128, 50000, 130), (33, 100001, 70), (17, 100000, 20)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", FEW_STEPS)
def test_filter_gradient_over_many_steps_of_inputs(N, I, O, dtype, block_plans):
    """Few samples, and so many inputs that a work-group goes through three 64s of them at least, in its two buffers."""
    p = block_plans.kept_grad(N, I, O, 0 if dtype == "f32" else 1)
    assert p["slices"] and p["rows_per_split"] >= 3
    _whole_gradient(N, I, O, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O,tile", [(255, 300, 260, 128), (1000, 300, 260, 128), (900, 2100, 2100, 128), (2100, 4096, 3900, 256)])
def test_filter_gradient_over_many_steps_of_rows(N, I, O, tile, dtype, block_plans):
    """Tiles whose sums take four steps at least, most of them many more: all but the last two are of the loop that loads, converts
    and multiplies at a time."""
    p = block_plans.kept_grad(N, I, O, 0 if dtype == "f32" else 1)
    assert not p["slices"] and p["tile"] == tile and p["rows_per_split"] >= 4 * p["step"]
    _whole_gradient(N, I, O, dtype)


def _whole_gradient(N, I, O, dtype):
    g = torch.Generator(device="cuda").manual_seed(N + I)
    x, dy = (torch.randint(-8, 9, (N, k), device="cuda", generator=g).float() for k in (I, O))
    q = hp.quantize_blocks(x, "e4m3")
    assert torch.equal(hp.dequantize_blocks(q), x)
    dw = torch.full((O, I), float("nan"), device="cuda")
    hp.fc_bwd_filter_kept(q, dy.to(DTYPES[dtype]), dw=dw)
    assert torch.equal(dw, (dy.t().contiguous().double() @ x.double()).float())


@pytest.mark.parametrize("N,I,O,tile,step", [(130, 200, 150, 128, 16), (256, 130, 260, 128, 16), (300, 200, 150, 128, 32),
                                             (1100, 4000, 4000, 256, 32), (1100, 4003, 4001, 256, 32)])
def test_filter_gradient_in_tiles_keeps_every_bit_of_fp32(N, I, O, tile, step, block_plans):
    """One sample of ones among zeros: dw is its dy, all 24 bits of it, in whichever step and row of a step it lies."""
    p = block_plans.kept_grad(N, I, O, 0)
    assert not p["slices"] and (p["tile"], p["step"]) == (tile, step)
    g = torch.Generator(device="cuda").manual_seed(N)
    dy = torch.randn((N, O), device="cuda", generator=g)
    assert (dy.view(torch.int32) & 255 != 0).float().mean() > 0.9    # (the third part is there)
    for n in sorted({0, 1, 2, 3, 5, 15, step - 1, step, 2 * step + 7, N // 2, N - step, N - 3, N - 2, N - 1, (N - 1) // step * step}):
        x = torch.zeros((N, I), device="cuda")
        x[n] = 1.0
        dw = hp.fc_bwd_filter_kept(hp.quantize_blocks(x, "e4m3"), dy)
        assert torch.equal(dw, dy[n].view(O, 1).expand(O, I)), n


def test_filter_gradient_of_no_samples():
    dw = torch.full((7, 40), 3.0, device="cuda")
    hp.fc_bwd_filter_kept(hp.Blocks.empty(0, 40, "e4m3"), torch.zeros((0, 7), device="cuda"), dw=dw)
    assert not dw.any()


# --------------------------------------------------------- the forward pass in 4 bits
def check_prod(x, w, bias, relu, dtype, out_bf16=False):
    q, held = _held(w, "e2m1")
    xv = oracle.dequantize_blocks(*oracle.quantize_blocks(x, "e2m1"), x.shape[1], "e2m1")
    N, O = len(x), len(w)
    y = torch.full((N, O), float("nan"), device="cuda", dtype=torch.bfloat16 if out_bf16 else torch.float32)
    b = None if bias is None else torch.from_numpy(bias).cuda()
    got = _host(hp.fc_fwd_q4(_dev(x, dtype), q, b, relu=relu, y=y))
    want, size = xv @ held.T, np.abs(xv) @ np.abs(held).T
    if bias is not None:
        want, size = want + bias.astype(np.float64), size + np.abs(bias)
    if relu:
        want = np.maximum(want, 0.0)
    bound = 2 * U * (x.shape[1] + 64) * size + (2.0 ** -8 * np.abs(want) if out_bf16 else 0.0) + 1e-37
    if out_bf16:
        bound = bound * (1 + 2.0 ** -8)                            # of a sum that is itself off by as much
    err = np.abs(got - want)
    assert (err <= bound).all(), (err / bound).max()
    return got


PRODS = [(1, 1, 1), (1, 128, 16), (1, 4096, 40), (2, 33, 100), (3, 1000, 17), (4, 129, 31), (7, 256, 1000), (8, 640, 33), (15, 127, 300),
         (16, 384, 64), (17, 512, 129), (31, 40, 48), (32, 2000, 65), (33, 96, 257), (64, 128, 128), (65, 260, 127), (100, 1025, 70),
         (128, 512, 256), (129, 300, 384), (257, 900, 130), (300, 640, 513), (1000, 64, 24)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", PRODS)
def test_forward_in_four_bits(N, I, O, dtype):
    g = RNG(N + I + O)
    x, w, bias = _values((N, I), dtype, N + I), _values((O, I), "f32", I + O, 0.05), g.normal(size=O).astype(np.float32)
    check_prod(x, w, bias, (N + I) % 2 == 0, dtype)
    check_prod(x, w, None, False, dtype, out_bf16=dtype == "bf16")


@pytest.mark.parametrize("N,I,O", [(1, 100, 20), (5, 1000, 70), (16, 4096, 33), (40, 300, 60), (260, 520, 300)])
def test_forward_of_whole_numbers_is_exact(N, I, O):
    g = RNG(N)
    x = g.choice([0, 1, 2, 3, 4, 6, -1, -2, -3, -4, -6], (N, I)).astype(np.float32)
    w = g.choice([0, 1, 2, 3, 4, 6, -1, -2, -3, -4, -6], (O, I)).astype(np.float32)
    x[:, ::32] = 6.0
    w[:, ::32] = -6.0
    q, held = _held(w, "e2m1")
    assert np.array_equal(held, w)
    bias = g.integers(-9, 9, O).astype(np.float32)
    want = x.astype(np.float64) @ w.T + bias
    assert np.array_equal(_host(hp.fc_fwd_q4(_dev(x), q, torch.from_numpy(bias).cuda())), want)
    assert np.array_equal(_host(hp.fc_fwd_q4(_dev(x), q, torch.from_numpy(bias).cuda(), relu=True)), np.maximum(want, 0))


# as above: so many steps that every wavefront refills its ring of three buffers (x put into blocks in the call; by a launch of its own
# in the three forms for few samples), and tiles that refill their four
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O,kind", [(1, 9216, 70, "fused"), (3, 8320, 40, "fused"), (2, 16300, 33, "fused"), (12, 9216, 50, "rows"),
                                        (16, 20000, 20, "rows"), (24, 9300, 100, "rows"), (32, 16384, 33, "rows"), (64, 8192, 300, "rows"),
                                        (100, 9216, 70, "rows"), (128, 9216, 4096, "rows"), (1000, 4200, 1100, "tiles128"), (600, 1300, 2100, "tiles128"),
                                        (1024, 4096, 4096, "tiles128"), (3600, 2200, 4000, "tiles256")])
def test_forward_of_whole_numbers_over_many_steps(N, I, O, kind, dtype, block_plans):
    p = block_plans.q4(N, I, O)
    assert kind == ("fused" if p["fused"] else "tiles%d" % p["tile"] if p["tile"] else "rows")
    if p["tile"]:
        assert p["steps"] > 2 * 4
    else:                                                            # pairs of steps to a wavefront
        assert (p["steps"] + 1) // 2 // (4 if p["wide"] == 4 else 8) > 3
    g = torch.Generator(device="cuda").manual_seed(N + I)
    values = torch.tensor([0, 1, 2, 3, 4, 6, -1, -2, -3, -4, -6], device="cuda", dtype=torch.float32)
    x, w = (values[torch.randint(0, 11, (k, I), device="cuda", generator=g)] for k in (N, O))
    x[:, ::32] = 6.0
    w[:, ::32] = -6.0
    bias = torch.randint(-9, 10, (O,), device="cuda", generator=g).float()
    q = hp.quantize_blocks(w, "e2m1")
    assert torch.equal(hp.dequantize_blocks(q), w)
    want = (x.double() @ w.double().t().contiguous() + bias.double()).float()
    assert want.abs().max() < 2 ** 24
    y = torch.full((N, O), float("nan"), device="cuda")
    assert torch.equal(hp.fc_fwd_q4(x.to(DTYPES[dtype]), q, bias, y=y), want)
    assert torch.equal(hp.fc_fwd_q4(x.to(DTYPES[dtype]), q, bias, relu=True), want.clamp_min(0.0))
    if dtype == "bf16":
        assert torch.equal(hp.fc_fwd_q4(x.bfloat16(), q, bias, out_bf16=True), want.bfloat16())


@pytest.mark.parametrize("N", [1, 3, 40, 200])
def test_values_that_are_no_numbers_in_the_forward_pass(N):
    """A sample's make its own outputs NaN, a filter's its own output; ReLU keeps them."""
    x, w = np.ones((N, 300), np.float32), np.ones((70, 300), np.float32)
    x[N - 1, 290], w[33, 5] = np.inf, np.nan
    got = _host(hp.fc_fwd_q4(_dev(x), _held(w, "e2m1")[0], relu=True))
    assert np.isnan(got[N - 1]).all() and np.isnan(got[:, 33]).all()
    rest = [o for o in range(70) if o != 33]
    assert (got[:N - 1][:, rest] == 300).all()


def test_forward_of_far_exponents():
    """Products whose factors are far apart in size."""
    x, w = np.full((3, 64), 2.0 ** 100, np.float32), np.full((5, 64), 2.0 ** -100, np.float32)
    x[:, 32:] = 2.0 ** -90
    w[:, 32:] = 2.0 ** 80
    got = _host(hp.fc_fwd_q4(_dev(x), _held(w, "e2m1")[0]))
    assert np.array_equal(got, np.full((3, 5), 32 + 32 * 2.0 ** -10))


@pytest.mark.parametrize("I", [64, 300, 512])
@pytest.mark.parametrize("N", [1, 3, 40, 200])
def test_forward_of_exponents_whose_product_is_past_fp32(N, I):
    """2^126 times 2^126 is an infinity, times a zero it is zero, in an odd number of steps and an even one."""
    x, w = np.zeros((N, I), np.float32), np.zeros((5, I), np.float32)
    x[:, I - 7] = w[1, I - 7] = w[2, I - 6] = 2.0 ** 126
    w[3, I - 7] = -2.0 ** 126
    got = _host(hp.fc_fwd_q4(_dev(x), _held(w, "e2m1")[0]))
    assert np.array_equal(got, np.tile([0, np.inf, 0, -np.inf, 0], (N, 1)))


def test_forward_of_no_samples():
    assert hp.fc_fwd_q4(torch.zeros((0, 40), device="cuda"), hp.Blocks.empty(9, 40, "e2m1")).shape == (0, 9)


@pytest.mark.parametrize("N,I,O", [(1, 300, 50), (9, 2000, 40), (130, 300, 260)])
def test_nothing_outside_the_outputs_is_written(N, I, O):
    w, _ = _held(_values((O, I), "f32", 3), "e2m1")
    q, _ = _held(_values((N, I), "f32", 4), "e4m3")
    x, dy = _dev(_values((N, I), "f32", 5)), _dev(_values((N, O), "f32", 6))
    for count, shape, call in ((N * O, (N, O), lambda o: hp.fc_fwd_q4(x, w, y=o)), (O * I, (O, I), lambda o: hp.fc_bwd_filter_kept(q, dy, dw=o))):
        buf = torch.full((count + 131,), 7.0, device="cuda")
        out = buf[3:3 + count].view(shape)
        out.fill_(float("nan"))
        call(out)
        assert not torch.isnan(out).any()
        out.fill_(7.0)
        assert (buf == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_same_bits_every_time(dtype):
    q, _ = _held(_values((900, 200), dtype, 7), "e4m3")
    w, _ = _held(_values((300, 1500), "f32", 8), "e2m1")
    dy, x, few = _dev(_values((900, 170), dtype, 9), dtype), _dev(_values((200, 1500), dtype, 10), dtype), _dev(_values((2, 1500), dtype, 11), dtype)
    first = [hp.fc_bwd_filter_kept(q, dy), hp.fc_fwd_q4(x, w), hp.fc_fwd_q4(few, w)]
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, [hp.fc_bwd_filter_kept(q, dy), hp.fc_fwd_q4(x, w), hp.fc_fwd_q4(few, w)]))
