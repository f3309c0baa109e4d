"""The 8-bit path without a GPU: pins of the oracle (oracle/fp8_oracle.py) and refusals of the C entry
points (include/aeris_fp8.h), which check their arguments before anything is launched."""
import ctypes

import numpy as np
import pytest

from oracle import fp8_oracle as fo
from paper_2509_13523_amd import binding as B


# ------------------------------------------------------------------------------------- oracle
def test_e4m3_values_by_hand():
    assert fo.TABLE[0] == 0 and fo.TABLE[1] == 2.0 ** -9 and fo.TABLE[7] == 7 * 2.0 ** -9
    assert fo.TABLE[8] == 2.0 ** -6 and fo.TABLE[0x38] == 1.0 and fo.TABLE[0x39] == 1.125
    assert fo.TABLE[0x7e] == 448.0 and (np.diff(fo.TABLE) > 0).all()
    assert fo.decode(np.array([0xb8]))[0] == -1.0 and np.isnan(fo.decode(np.array([0x7f, 0xff]))).all()
    # ties to even: between 1 (0x38) and 1.125 (0x39), between 1.125 and 1.25 (0x3a); half the smallest
    assert list(fo.encode([1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, -1.0625])) == [0x38, 0x3a, 0, 2, 0xb8]


def test_every_code_comes_back():
    codes = np.array([c for c in range(256) if c & 127 != 127], dtype=np.uint8)
    values = fo.decode(codes)
    assert (fo.encode(values) == codes).all()
    torch = pytest.importorskip("torch")
    assert (torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy() == values).all()


def test_scales_by_hand():
    x = np.zeros((1, 192))
    x[0, :128] = 448.0
    x[0, 128:] = 448.0 * (1 + 2.0 ** -30)
    codes, scales = fo.quantize(x)
    assert list(scales[0]) == [127, 128, 127, 127]
    assert (codes[0, :128] == 0x7e).all() and (codes[0, 128:] == 0x76).all()      # 448, and 224 at scale 2
    codes, scales = fo.quantize(np.full((1, 64), 1e-45))
    assert scales[0, 0] == 1 and (codes == 0).all()
    codes, scales = fo.quantize(np.array([[np.inf] + [1.0] * 63]))
    assert scales[0, 0] == 119 and codes[0, 0] == 0x7f and fo.dequantize(codes, scales)[0, 1] == 1.0


def test_round_trip_is_within_half_a_step():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((40, 320)) * np.exp(3 * rng.standard_normal((40, 320)))
    codes, scales = fo.quantize(x)
    err = np.abs(fo.dequantize(codes, scales) - x)
    assert (err <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * fo.per_column(scales, 320))).all()
    # the largest of a block uses the upper half of the range
    for b in range(3):
        most = np.abs(x[:, b * 128:(b + 1) * 128]).max(axis=1) / 2.0 ** (scales[:, b] - 127.0)
        assert ((most > 224) & (most <= 448)).all()


def test_gradients_against_differences():
    """<dx, u> and <dw, v> are the derivatives of sum(y dy) along u and v; dy is chosen representable, so that
    quantising it changes nothing."""
    rng = np.random.default_rng(5)
    x, w = rng.standard_normal((6, 64)), rng.standard_normal((10, 64))
    dy = fo.round_trip(rng.standard_normal((6, 10)))
    dx, dw = fo.linear_bwd(x, w.T, dy)
    u, v, h = rng.standard_normal(x.shape), rng.standard_normal(w.shape), 1e-4
    by = lambda a, b: float((fo.linear_fwd(a, b) * dy).sum())
    assert abs((by(x + h * u, w) - by(x - h * u, w)) / (2 * h) - (dx * u).sum()) < 1e-8
    assert abs((by(x, w + h * v) - by(x, w - h * v)) / (2 * h) - (dw * v).sum()) < 1e-8


# ------------------------------------------------------------------------------------- refusals
A = ctypes.c_void_p(4096)          # a non-null, aligned address that is never dereferenced
ODD = ctypes.c_void_p(4096 + 8)


def test_scale_pitch():
    assert [B.aeris_fp8_scale_pitch(c) for c in (64, 512, 576, 2048, 5504, 65536)] == [4, 4, 8, 16, 44, 512]
    assert [B.aeris_fp8_scale_pitch(c) for c in (0, -64, 32, 100, 65600)] == [0] * 5


def quantize(**kw):
    return B.load().aeris_fp8_quantize(*[kw.get(k, d) for k, d in (
        ("x", A), ("dtype", 0), ("n", 128), ("c", 128), ("x8", A), ("xs", A), ("xt8", A), ("xts", A))], None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), -1), (dict(x8=None), -1), (dict(xts=None), -1), (dict(x8=None, xs=None, xt8=None, xts=None), -1),
    (dict(dtype=2), -10), (dict(dtype=-1), -10), (dict(n=0), -2), (dict(n=-5), -2), (dict(c=0), -2),
    (dict(c=32), -2), (dict(c=65600), -2), (dict(c=100), -3), (dict(n=100), -3), (dict(n=65600), -2),
    (dict(n=1 << 40, xt8=None, xts=None), -2), (dict(x=ODD), -7), (dict(xs=ODD), -7), (dict(xt8=ODD), -7)])
def test_quantize_refuses(change, code):
    assert quantize(**change) == code


def norm(**kw):
    return B.load().aeris_residual_norm_fp8_fwd(*[kw.get(k, d) for k, d in (
        ("x", A), ("y", A), ("alpha", A), ("w", A), ("gamma", A), ("beta", A), ("eps", 1e-6), ("n", 8), ("rps", 4),
        ("c", 64), ("s", A), ("r", A), ("h8", A), ("hs", A))], None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), -1), (dict(w=None), -1), (dict(h8=None), -1), (dict(hs=None), -1), (dict(alpha=None), -1),
    (dict(s=None), -1), (dict(n=0), -2), (dict(rps=0), -2), (dict(rps=3), -3), (dict(c=96), -3), (dict(c=4160), -2),
    (dict(eps=-1.0), -2), (dict(eps=float("nan")), -2), (dict(x=ODD), -7), (dict(s=ODD), -7), (dict(alpha=ODD), -7),
    (dict(r=ctypes.c_void_p(4098)), -7), (dict(hs=ODD), -7), (dict(n=1 << 22, rps=1), -2)])
def test_residual_norm_refuses(change, code):
    assert norm(**change) == code


def test_swiglu_refuses():
    call = lambda uv=A, n=8, h=64, g8=A, gs=A: B.load().aeris_swiglu_fp8_fwd(uv, n, h, g8, gs, None)
    assert call(uv=None) == -1 and call(g8=None) == -1 and call(gs=None) == -1
    assert call(n=0) == -2 and call(h=0) == -2 and call(h=65600) == -2 and call(h=72) == -3
    assert call(uv=ODD) == -7 and call(gs=ODD) == -7


def test_linear_refuses():
    def call(**kw):
        return B.load().aeris_linear_fp8_fwd(*[kw.get(k, d) for k, d in (
            ("x8", A), ("xs", A), ("w8", A), ("ws", A), ("n", 8), ("c", 128), ("f", 192), ("y", A))], None)
    for name in ("x8", "xs", "w8", "ws", "y"):
        assert call(**{name: None}) == -1 and call(**{name: ODD}) == -7
    assert call(n=0) == -2 and call(c=0) == -2 and call(f=0) == -2 and call(c=65600) == -2 and call(f=65600) == -2
    assert call(c=96) == -3 and call(f=72) == -3
    assert call(n=1 << 39, f=65536) == -2                       # more tiles than a launch holds


@pytest.mark.parametrize("f", [64, 192, 65536])
def test_linear_takes_as_many_tiles_as_a_launch_holds(f):
    most = ((1 << 25) - 1) // (f // 64) * 64
    assert B.aeris_linear_fp8_plan(most, 128, f)[0] in (64, 128, 256)
    with pytest.raises(B.AerisError):
        B.aeris_linear_fp8_plan(most + 1, 128, f)


def test_linear_bwd_refuses_and_sizes_its_workspace():
    lib = B.load()
    n, c, f = 1000, 192, 320
    need = B.aeris_linear_fp8_bwd_workspace_bytes(n, c, f)
    up = lambda v: -(-v // 256) * 256
    for_dx = up(n * f) + up(n * B.aeris_fp8_scale_pitch(f))
    assert need == max(for_dx, up(n * c * 2) + B.aeris_linear_bwd_workspace_bytes(n, c, f))
    for bad in ((0, c, f), (n, 100, f), (n, c, 72), (n, 65600, f), (n, 65536, 65536)):
        assert B.aeris_linear_fp8_bwd_workspace_bytes(*bad) == 0

    def call(**kw):
        return lib.aeris_linear_fp8_bwd(*[kw.get(k, d) for k, d in (
            ("x8", A), ("xs", A), ("wt8", A), ("wts", A), ("dy", A), ("n", n), ("c", c), ("f", f), ("dx", A),
            ("dw", A), ("space", A), ("bytes", need))], None)
    for name in ("x8", "xs", "wt8", "wts", "dy", "space"):
        assert call(**{name: None}) == -1 and call(**{name: ODD}) == -7
    assert call(dx=None, dw=None) == -1 and call(dx=ODD) == -7 and call(dw=ODD) == -7
    assert call(bytes=need - 1) == -8 and call(n=0) == -2 and call(c=96) == -3 and call(f=72) == -3


def test_linear_tells_its_parts():
    assert [B.aeris_linear_fp8_parts(*v) for v in ((1, 2048, 12288), (128, 5504, 2048), (172800, 2048, 11008))] == [8, 4, 1]
    with pytest.raises(B.AerisError):
        B.aeris_linear_fp8_parts(8, 96, 64)


def test_linear_bwd_workspace_of_what_is_wanted():
    lib = B.load()
    up = lambda v: -(-v // 256) * 256
    size = B.aeris_linear_fp8_bwd_workspace_bytes_for
    for n, c, f in ((1, 64, 64), (1000, 192, 320), (40, 128, 2048), (172800, 5504, 2048)):
        for_dx = up(n * f) + up(n * B.aeris_fp8_scale_pitch(f))
        for_dw = up(n * c * 2) + B.aeris_linear_bwd_workspace_bytes(n, c, f)
        assert size(n, c, f, True, False) == for_dx and size(n, c, f, False, True) == for_dw
        assert size(n, c, f, True, True) == max(for_dx, for_dw) == B.aeris_linear_fp8_bwd_workspace_bytes(n, c, f)
        for dx, dw in ((A, None), (None, A), (A, A)):                  # one byte less is refused
            assert lib.aeris_linear_fp8_bwd(A, A, A, A, A, n, c, f, dx, dw, A, size(n, c, f, dx, dw) - 1, None) == -8
    assert size(172800, 5504, 2048, True, False) < 360e6              # 2466 MB for both
    for bad in ((0, 64, 64), (8, 100, 64), (8, 64, 72), (8, 65536, 65536)):
        assert size(*bad, True, False) == 0 and size(*bad, False, True) == 0


def test_a_wrong_gradient_shows_along_itself():
    """The check that the GPU's gradients go through (gradient_check.py) passes the oracle's, with its forward products
    rounded to bf16, and fails a gradient of zeros and those that lack 64 features or 64 tokens of their sum."""
    import gradient_check as gc
    half_step = lambda rng, a: a * (1 + 2.0 ** -8 * rng.uniform(-1, 1, a.shape))
    for n, c, f in ((96, 256, 192), (333, 192, 320), (500, 448, 576)):
        rng = np.random.default_rng(n + c + f)
        rows = lambda r, k: fo.round_trip(rng.standard_normal((r, k)) * np.exp(rng.standard_normal(k)))
        x, dy, weight = rows(n, c), rows(n, f), rng.standard_normal((f, c)) / np.sqrt(c)
        w, wt = fo.round_trip(weight), fo.round_trip(weight.T)
        dx, dw = fo.linear_bwd(x, wt, dy)
        u, v = fo.round_trip(dx), fo.round_trip(dw)
        along_dx = lambda dx: gc.along_dx(half_step(rng, fo.linear_fwd(u, w)), dx, u, dy, w, wt)
        along_dw = lambda dw: gc.along_dw(half_step(rng, fo.linear_fwd(x, v)), dw, v, dy, x)
        for along, right, wrong in (
                (along_dx, half_step(rng, dx), [0 * dx, fo.linear_bwd(x, wt[:, 64:], dy[:, 64:])[0]]),
                (along_dw, dw, [0 * dw, fo.linear_bwd(x[64:], wt, dy[64:])[1]])):
            gap, allow, size = along(right)
            assert gap <= allow <= 0.02 * size
            for g in wrong:
                gap, allow, _ = along(g)
                assert gap > 2 * allow
