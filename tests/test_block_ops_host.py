"""Tensors held in blocks, layer normalisation and the passes on them without a GPU: the oracle's definitions against what the
mathematics and the formats fix, and the argument checks of the entry points."""
import numpy as np
import pytest
import torch

import oracle

PTR = 4096
RNG = lambda s: np.random.Generator(np.random.Philox(s))
FORMS = ["e4m3", "e2m1"]
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    from paper_1312_5853_amd import binding, build
    if build.is_stale():
        build.build()
    return binding.lib()


# ------------------------------------------------------------- the oracle ---
def test_magnitudes_of_the_formats():
    assert oracle.block_magnitudes("e2m1").tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    m = oracle.block_magnitudes("e4m3")
    assert len(m) == 127 and m[1] == 2.0 ** -9 and m[8] == 2.0 ** -6 and m[-1] == 448 and (np.diff(m) > 0).all()
    every = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(every, m)


def test_eight_bit_codes_against_torch():
    """Blocks whose largest value is 448 have the exponent 0: the codes are those of a plain conversion."""
    x = np.concatenate([RNG(1).normal(size=4000) * np.exp2(RNG(2).uniform(-12, 8, 4000)), [0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10]])
    x = np.clip(x, -448, 448).astype(np.float32)
    x = np.concatenate([x, np.zeros(-len(x) % 31, np.float32)]).reshape(-1, 31)
    x = np.concatenate([x, np.full((len(x), 1), 448, np.float32)], axis=1).reshape(1, -1)
    codes, scales = oracle.quantize_blocks(x, "e4m3")
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(codes[:, :x.shape[1]], want) and (scales[:, :x.shape[1] // 32] == 127).all()


@pytest.mark.parametrize("form", FORMS)
def test_blocks_by_hand(form):
    top = {"e4m3": 448.0, "e2m1": 6.0}[form]
    x = np.zeros((1, 32 * 6))
    x[0, 0] = top                                    # exponent 0
    x[0, 32] = np.nextafter(top, INF)                # a little more: 1
    x[0, 64] = -top / 4                              # -2
    x[0, 96] = 1e-45                                 # the least exponent, and nothing left
    x[0, 128:130] = INF, 1.0
    x[0, 160:162] = 1.0, NAN
    codes, scales = oracle.quantize_blocks(x, form)
    assert scales[0, :6].tolist() == [127, 128, 125, 127 + {"e4m3": -117, "e2m1": -125}[form], 255, 255]
    v = oracle.dequantize_blocks(codes, scales, 192, form)[0]
    assert v[0] == top and v[32] == top and v[64] == -top / 4 and v[96] == 0
    assert np.isnan(v[128:]).all() and not np.isnan(v[:128]).any()
    assert (v[1:32] == 0).all() and codes.shape[1] == (256 if form == "e4m3" else 128) and scales.shape[1] == 8
    assert (scales[0, 6:] == 127 + {"e4m3": -117, "e2m1": -125}[form]).all()


@pytest.mark.parametrize("form", FORMS)
def test_held_values_are_near_and_stay(form):
    """Within half a step of the values; what is held comes back unchanged when it is put into blocks again."""
    x = RNG(3).normal(size=(7, 300)) * np.exp2(RNG(4).integers(-60, 60, (7, 300)))
    v = oracle.dequantize_blocks(*oracle.quantize_blocks(x, form), 300, form)
    top, rel, least = {"e4m3": (448.0, 2.0 ** -4, 2.0 ** -10), "e2m1": (6.0, 0.25, 0.25)}[form]
    amax = np.abs(np.pad(x, ((0, 0), (0, 20))).reshape(7, -1, 32)).max(axis=2)
    scale = np.repeat(np.exp2(np.ceil(np.log2(amax / top))), 32, axis=1)[:, :300]
    assert (np.abs(v - x) <= np.maximum(rel * np.abs(x), least * scale) * (1 + 1e-12)).all()
    again = oracle.dequantize_blocks(*oracle.quantize_blocks(v, form), 300, form)
    assert np.array_equal(v, again)
    assert np.array_equal(oracle.dequantize_blocks(*oracle.quantize_blocks(-x, form), 300, form), -v)


def test_layer_norm_is_group_norm_of_one_group():
    g = RNG(5)
    x, dy, gamma, beta = g.normal(2.0, 3.0, (4, 11)), g.normal(size=(4, 11)), g.normal(size=11), g.normal(size=11)
    y, mean, rstd = oracle.layer_norm_fwd(x, gamma, beta, 1e-3)
    want = oracle.group_norm_act_fwd(x[:, :, None], 1, gamma, beta, 1e-3, "none")
    assert np.abs(y - want[0][:, :, 0]).max() < 1e-13 and np.abs(mean - want[1][:, 0]).max() < 1e-14
    got = oracle.layer_norm_bwd(x, dy, mean, rstd, gamma)
    want = oracle.group_norm_act_bwd(x[:, :, None], dy[:, :, None], want[1], want[2], gamma, beta, "none")
    assert np.abs(got[0] - want[0][:, :, 0]).max() < 1e-13
    assert np.abs(got[1] - want[1]).max() < 1e-13 and np.abs(got[2] - want[2]).max() < 1e-13


def test_layer_norm_by_hand():
    y, mean, rstd = oracle.layer_norm_fwd(np.array([[1.0, 2.0, 3.0, 6.0]]), [2.0, 2.0, 4.0, 4.0], [0.5, 0.5, -2.0, -2.0], 0.5)
    assert mean[0] == 3.0 and rstd[0] == 0.5 and y.tolist() == [[-1.5, -0.5, -2.0, 4.0]]


def test_layer_norm_gradient_against_differences():
    g = RNG(6)
    x, dy, gamma, beta, eps = g.normal(size=(3, 7)), g.normal(size=(3, 7)), g.normal(1, 0.3, 7), g.normal(0, 0.3, 7), 1e-3
    f = lambda x, gamma, beta: float((oracle.layer_norm_fwd(x, gamma, beta, eps)[0] * dy).sum())
    _, mean, rstd = oracle.layer_norm_fwd(x, gamma, beta, eps)
    args, h = [x, gamma, beta], 1e-6
    for which, grad in enumerate(oracle.layer_norm_bwd(x, dy, mean, rstd, gamma)):
        for i in np.ndindex(grad.shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[which][i] += h
            down[which][i] -= h
            # differences of values of size 10 at h = 1e-6: 10 * 1e-16 / 1e-6 and the third derivative's h^2
            assert abs((f(*up) - f(*down)) / (2 * h) - grad[i]) < 1e-7


# ------------------------------------------------------ argument checks -----
def _caller(f, args):
    return lambda **kw: f(*dict(args, **kw).values())


def test_block_argument_checks(lib):
    from paper_1312_5853_amd import binding as b
    to = dict(x=PTR, xs=40, codes=PTR * 2, scales=PTR * 3, N=2, C=40, form=0, dtype=0, stream=None)
    back = dict(codes=PTR * 2, scales=PTR * 3, x=PTR, xs=40, N=2, C=40, form=0, dtype=0, stream=None)
    for f in (_caller(lib.quantize_blocks, to), _caller(lib.dequantize_blocks, back)):
        for bad in (dict(x=None), dict(codes=None), dict(scales=None), dict(xs=39), dict(N=-1), dict(C=0), dict(form=2), dict(form=-1),
                    dict(codes=PTR), dict(scales=PTR), dict(scales=PTR * 2)):
            assert f(**bad) == b.ERR_INVALID_ARG, bad
        assert f(dtype=3) == b.ERR_BAD_DTYPE
        assert f(C=(1 << 30) + 1, xs=1 << 31) == b.ERR_TOO_LARGE
        assert f(N=1 << 20, C=1 << 15, xs=1 << 15) == b.ERR_TOO_LARGE
        assert f(N=(1 << 27) + 1, C=1) == b.ERR_TOO_LARGE                # filled up to 128 values each
        for bad in (dict(x=PTR + 2), dict(x=PTR + 1, dtype=1), dict(codes=PTR * 2 + 8), dict(scales=PTR * 3 + 2)):
            assert f(**bad) == b.ERR_MISALIGNED, bad
        assert f(N=0, x=None, codes=None, scales=None) == b.OK


def test_layer_norm_argument_checks(lib):
    from paper_1312_5853_amd import binding as b
    fwd = dict(x=PTR, xs=40, gamma=None, beta=None, y=PTR * 2, ys=40, mean=None, rstd=None, N=2, C=40, eps=1e-5, dtype=0, stream=None)
    f = _caller(lib.layer_norm_fwd, fwd)
    for bad in (dict(x=None), dict(y=None), dict(y=PTR), dict(xs=39), dict(ys=39), dict(N=-1), dict(C=0), dict(eps=0.0), dict(eps=-1.0),
                dict(eps=NAN), dict(eps=INF)):
        assert f(**bad) == b.ERR_INVALID_ARG, bad
    assert f(dtype=3) == b.ERR_BAD_DTYPE
    assert f(C=(1 << 27) + 1, xs=1 << 30, ys=1 << 30) == b.ERR_TOO_LARGE
    assert f(N=1 << 20, C=1 << 20, xs=1 << 20, ys=1 << 20) == b.ERR_TOO_LARGE
    for bad in (dict(x=PTR + 2), dict(y=PTR * 2 + 1, dtype=1), dict(gamma=PTR + 2), dict(beta=PTR + 2), dict(mean=PTR + 2),
                dict(rstd=PTR + 1)):
        assert f(**bad) == b.ERR_MISALIGNED, bad
    assert f(N=0, x=None, y=None) == b.OK
    rest = dict(dy=PTR * 2, dys=40, gamma=None, mean=PTR, rstd=PTR, dx=PTR * 3, dxs=40, dgamma=PTR * 4, dbeta=PTR * 5, N=2, C=40,
                dtype=0, ws=PTR, ws_bytes=1 << 30, stream=None)
    plain, kept = dict(x=PTR, xs=40, **rest), dict(codes=PTR, scales=PTR * 6, **rest)
    need = lib.layer_norm_workspace_bytes(b.OP_BWD_DATA, 1000, 40, 0)
    assert need > 0
    for f, own in ((_caller(lib.layer_norm_bwd, plain), (dict(x=None), dict(dx=PTR), dict(xs=39))),
                   (_caller(lib.layer_norm_bwd_kept, kept), (dict(codes=None), dict(scales=None), dict(dx=PTR), dict(dx=PTR * 6)))):
        for bad in own + (dict(dy=None), dict(mean=None), dict(rstd=None), dict(dx=None), dict(dx=PTR * 2), dict(dys=39), dict(dxs=39),
                          dict(N=-1), dict(C=0)):
            assert f(**bad) == b.ERR_INVALID_ARG, bad
        assert f(dtype=3) == b.ERR_BAD_DTYPE
        assert f(C=(1 << 27) + 1, dys=1 << 30, dxs=1 << 30, **({"xs": 1 << 30} if own[0].get("x", 1) is None else {})) == b.ERR_TOO_LARGE
        for bad in (dict(dy=PTR * 2 + 2), dict(dx=PTR * 3 + 1, dtype=2), dict(gamma=PTR + 2), dict(mean=PTR + 2), dict(rstd=PTR + 2),
                    dict(dgamma=PTR + 2), dict(dbeta=PTR + 2), dict(N=1000, ws=PTR + 8)):
            assert f(**bad) == b.ERR_MISALIGNED, bad
        assert f(N=1000, ws_bytes=need - 1) == b.ERR_WORKSPACE and f(N=1000, ws=None) == b.ERR_WORKSPACE
    assert _caller(lib.layer_norm_bwd_kept, kept)(codes=PTR + 8) == b.ERR_MISALIGNED
    assert _caller(lib.layer_norm_bwd_kept, kept)(scales=PTR + 2) == b.ERR_MISALIGNED
    for bad in ((b.OP_BWD_DATA, -1, 40, 0), (b.OP_BWD_DATA, 2, 0, 0), (b.OP_BWD_DATA, 2, 40, 3), (9, 2, 40, 0), (b.OP_FWD, 2, 40, 0)):
        assert lib.layer_norm_workspace_bytes(*bad) == 0


def test_fully_connected_argument_checks(lib):
    from paper_1312_5853_amd import binding as b
    grad = dict(codes=PTR, scales=PTR * 2, dy=PTR * 3, dw=PTR * 4, N=4096, I=40, O=24, dtype=0, ws=PTR, ws_bytes=1 << 30, stream=None)
    f = _caller(lib.fc_bwd_filter_kept, grad)
    for bad in (dict(codes=None), dict(scales=None), dict(dy=None), dict(dw=None), dict(dw=PTR * 3), dict(dw=PTR), dict(dw=PTR * 2),
                dict(N=-1), dict(I=0), dict(O=-3)):
        assert f(**bad) == b.ERR_INVALID_ARG, bad
    assert f(dtype=5) == b.ERR_BAD_DTYPE
    for bad in (dict(N=1 << 24), dict(N=1 << 20, O=1 << 11), dict(I=1 << 16, O=1 << 15, N=1)):
        assert f(**bad) == b.ERR_TOO_LARGE, bad
    for bad in (dict(codes=PTR + 8), dict(scales=PTR + 2), dict(dy=PTR + 2), dict(dy=PTR + 1, dtype=1), dict(dw=PTR + 2), dict(ws=PTR + 16)):
        assert f(**bad) == b.ERR_MISALIGNED, bad
    need = lib.fc_kept_workspace_bytes(4096, 40, 24, 0)
    assert need > 0 and f(ws_bytes=need - 1) == b.ERR_WORKSPACE and f(ws=None) == b.ERR_WORKSPACE
    prod = dict(x=PTR, codes=PTR * 2, scales=PTR * 3, bias=None, y=PTR * 4, N=4, I=40, O=24, relu=0, dtype=0, ws=PTR, ws_bytes=1 << 30,
                stream=None)
    f = _caller(lib.fc_fwd_q4, prod)
    for bad in (dict(x=None), dict(codes=None), dict(scales=None), dict(y=None), dict(y=PTR), dict(y=PTR * 2), dict(y=PTR * 3),
                dict(N=-1), dict(I=0), dict(O=0)):
        assert f(**bad) == b.ERR_INVALID_ARG, bad
    assert f(dtype=5) == b.ERR_BAD_DTYPE
    for bad in (dict(N=1 << 24), dict(O=1 << 24, N=1), dict(N=1 << 16, O=1 << 15)):
        assert f(**bad) == b.ERR_TOO_LARGE, bad
    for bad in (dict(x=PTR + 2), dict(x=PTR + 1, dtype=1), dict(codes=PTR + 8), dict(scales=PTR + 2), dict(bias=PTR + 2),
                dict(y=PTR * 4 + 2), dict(y=PTR * 4 + 2, dtype=1), dict(y=PTR * 4 + 1, dtype=2)):
        assert f(**bad) == b.ERR_MISALIGNED, bad
    for N in (100, 1000):
        need = lib.fc_q4_workspace_bytes(N, 40, 24, 0)
        assert need > 0 and f(N=N, ws_bytes=need - 1) == b.ERR_WORKSPACE and f(N=N, ws=None) == b.ERR_WORKSPACE
        assert f(N=N, ws=PTR + 16) == b.ERR_MISALIGNED
    assert f(N=0, x=None, codes=None, scales=None, y=None, ws=None, ws_bytes=0) == b.OK
    for bad in ((-1, 40, 24, 0), (4, 0, 24, 0), (4, 40, 0, 0), (4, 40, 24, 9)):
        assert lib.fc_kept_workspace_bytes(*bad) == 0 and lib.fc_q4_workspace_bytes(*bad) == 0


def test_binding_refuses_what_the_library_cannot_see(lib):
    """Shapes, types, memory orders and devices are checked before any pointer is taken."""
    from paper_1312_5853_amd import binding as b
    byte = lambda *s: torch.zeros(s, dtype=torch.uint8)
    x, q8, q4 = torch.zeros(3, 40), b.Blocks(byte(3, 128), byte(3, 4), 40, "e4m3"), b.Blocks(byte(3, 64), byte(3, 4), 40, "e2m1")
    assert q8.shape == (3, 40) and q8.nbytes == 3 * 132 and q4.nbytes == 3 * 68
    for bad in ((byte(3, 127), byte(3, 4), 40, "e4m3"), (byte(3, 128), byte(3, 5), 40, "e4m3"), (byte(3, 128), byte(3, 4), 129, "e4m3"),
                (byte(3, 128), byte(3, 4), 0, "e4m3"), (byte(3, 128), byte(3, 4), 40, "e2m1"), (byte(3, 128), byte(2, 4), 40, "e4m3"),
                (byte(128, 3).t(), byte(3, 4), 40, "e4m3"), (byte(384), byte(3, 4), 40, "e4m3"), (byte(3, 128), byte(3, 4), 40, "e5m2")):
        with pytest.raises(ValueError):
            b.Blocks(*bad)
    with pytest.raises(TypeError):
        b.Blocks(torch.zeros(3, 128), byte(3, 4), 40, "e4m3")
    with pytest.raises(TypeError):
        b.Blocks(byte(3, 128), byte(3, 4), 40.0, "e4m3")
    for call in (lambda: b.quantize_blocks(x, "e4m3"), lambda: b.quantize_blocks(x.t(), "e4m3"), lambda: b.quantize_blocks(x, "e5m2"),
                 lambda: b.dequantize_blocks(q8), lambda: b.dequantize_blocks(q8, x=torch.zeros(3, 41)),
                 lambda: b.dequantize_blocks(q8, x=torch.zeros(40, 3).t()),
                 lambda: b.layer_norm_fwd(x), lambda: b.layer_norm_fwd(torch.zeros(2, 3, 4)), lambda: b.layer_norm_fwd(x[:, ::2]),
                 lambda: b.layer_norm_bwd(x, x, torch.zeros(3), torch.zeros(3)),
                 lambda: b.layer_norm_bwd(x, torch.zeros(3, 39), torch.zeros(3), torch.zeros(3)),
                 lambda: b.layer_norm_bwd_kept(q4, x, torch.zeros(3), torch.zeros(3)),
                 lambda: b.layer_norm_bwd_kept(q8, torch.zeros(4, 40), torch.zeros(3), torch.zeros(3)),
                 lambda: b.fc_bwd_filter_kept(q4, torch.zeros(3, 5)), lambda: b.fc_bwd_filter_kept(q8, torch.zeros(4, 5)),
                 lambda: b.fc_bwd_filter_kept(q8, torch.zeros(5, 3).t()), lambda: b.fc_bwd_filter_kept(q8, torch.zeros(3, 5)),
                 lambda: b.fc_fwd_q4(x, q8), lambda: b.fc_fwd_q4(torch.zeros(2, 41), q4), lambda: b.fc_fwd_q4(torch.zeros(40, 2).t(), q4),
                 lambda: b.fc_fwd_q4(x, q4)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: b.quantize_blocks(x.double(), "e4m3"), lambda: b.dequantize_blocks(x), lambda: b.layer_norm_fwd(x.half()),
                 lambda: b.dequantize_blocks(q8, x=torch.zeros(3, 40, dtype=torch.float16)),
                 lambda: b.layer_norm_bwd(x, x.bfloat16(), torch.zeros(3), torch.zeros(3)), lambda: b.layer_norm_bwd_kept(x, x, x, x),
                 lambda: b.fc_bwd_filter_kept(x, x), lambda: b.fc_fwd_q4(x, x), lambda: b.fc_fwd_q4(x.half(), q4)):
        with pytest.raises(TypeError):
            call()


def test_binding_refuses_sizes_past_a_c_int(lib):
    """A size of 2^32 + 1 must not reach the library as 1."""
    from paper_1312_5853_amd import binding as b
    far = (1 << 32) + 1
    meta = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="meta")
    byte = lambda *s: meta(*s, dtype=torch.uint8)
    q8, q4 = b.Blocks(byte(1, 128), byte(1, 4), 1, "e4m3"), b.Blocks(byte(5, 64), byte(5, 4), 1, "e2m1")
    for call in (lambda: b.quantize_blocks(meta(far, 1), "e4m3"), lambda: b.quantize_blocks(meta(1, far), "e4m3"),
                 lambda: b.dequantize_blocks(q8, x=meta(far, 1)), lambda: b.layer_norm_fwd(meta(far, 1)),
                 lambda: b.layer_norm_bwd(meta(far, 1), meta(far, 1), meta(far), meta(far)),
                 lambda: b.layer_norm_bwd_kept(q8, meta(far, 1), meta(1), meta(1)),
                 lambda: b.distill_loss_fwd(meta(far, 3), labels=meta(far, dtype=torch.int32)),
                 lambda: b.fc_bwd_filter_kept(q8, meta(1, far)), lambda: b.fc_fwd_q4(meta(far, 1), q4),
                 lambda: b.Blocks(byte(1, 128 * 2 ** 25), byte(1, 4 * 2 ** 25), far - 1, "e4m3"), lambda: b.Blocks.empty(far, 1, "e2m1", "meta")):
        with pytest.raises(b.ConvError) as e:
            call()
        assert e.value.status == b.ERR_TOO_LARGE
