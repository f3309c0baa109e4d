"""GPU parity of the 8-bit path (include/aeris_fp8.h) against oracle/fp8_oracle.py and oracle/block_oracle.py.

Quantised bf16 and fp32 rows have to be the oracle's to the bit: a power-of-two scale is exact and e4m3 of it is
one rounding.  Where a value is computed first (norm, gate) it carries fp32 errors into that rounding:
  |q scale - h| <= 2^-4 |h| (half a step of e4m3) or 2^-10 scale (half its smallest) + 4e-6 of the terms of h,
and a scale may be the neighbour of the oracle's only if the block's largest value lies within 4e-6 of the border.
Products: the bf16 result is within 2^-8 of the value (half a step), and three errors of sums are added:
  7 * 2^-13 * sum over groups of eight channels of the largest |x w| (what the matrix instruction drops, stated in
  the header), bounded by the group's largest |x| times its largest |w|;
  (channels / 32 + 8) * 2^-23 * sum |x w| (fp32 additions of the groups and steps, truncating ones included).
"""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from oracle import fp8_oracle as fo
from paper_2509_13523_amd import binding as B
from paper_2509_13523_amd import synth
import gradient_check as gc
import parity_log

pytestmark = pytest.mark.gpu

SLACK = 4e-6            # of the sum of magnitudes of an element's terms: about 30 fp32 roundings of 2^-24 and the
                        # hardware's reciprocal and exponential of one unit each


def to_f64(t):
    return t.double().cpu().numpy()


def bf16(a):
    """(device tensor, its values) of an array rounded to bf16."""
    bits = synth.f32_to_bf16_bits(np.asarray(a, dtype=np.float32))
    return torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16), synth.bf16_bits_to_f64(bits)


def f32(a):
    a = np.asarray(a, dtype=np.float32)
    return torch.from_numpy(a).cuda(), a.astype(np.float64)


def codes(q, scales):
    return q.view(torch.uint8).cpu().numpy(), scales.view(torch.uint8).cpu().numpy()


def dev(q, scales):
    return (torch.from_numpy(q).cuda().view(torch.float8_e4m3fn),
            torch.from_numpy(scales).cuda().view(torch.float8_e8m0fnu))


def same_codes(got, want):
    """Equal but for the sign of NaN."""
    nan = (want & 127) == 127
    assert got.shape == want.shape and (got[~nan] == want[~nan]).all() and ((got[nan] & 127) == 127).all()


def rows_with_gain(rng, n, c):
    return rng.standard_normal((n, c)) * np.exp(rng.standard_normal(c))


# ------------------------------------------------------------------------------------- quantise
def hard_rows(rng, n, c, most):
    """Rows with what a block can meet: zeros, one value alone, values at the border of a scale, values that are not
    finite, and magnitudes from the smallest to the largest."""
    x = rows_with_gain(rng, n, c)
    for i in range(n):
        kind, at = i % 9, rng.integers(c)
        if kind == 1: x[i] = 0.0
        elif kind == 2: x[i] = 0.0; x[i, at] = -3.0
        elif kind == 3: x[i] = np.clip(x[i], -1, 1) * 100; x[i, at] = 448.0 * 2.0 ** (i % 7 - 3)
        elif kind == 4: x[i, at] = np.inf; x[i, (at + 5) % c] = -np.inf; x[i, (at + 77) % c] = np.nan
        elif kind == 5: x[i] *= 2.0 ** -120
        elif kind == 6: x[i] *= most / np.abs(x[i]).max()
        elif kind == 7: x[i] = np.nan
        elif kind == 8: x[i] *= np.exp2(rng.integers(-20, 20, c))
    return x


@pytest.mark.parametrize("n,c,transposed", [
    (1, 64, False), (1, 128, False), (3, 192, False), (17, 448, False), (200, 2048, False), (33, 5504, False),
    (64, 64, True), (128, 128, True), (192, 320, True), (64, 1088, True), (1152, 192, True), (320, 512, True)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_is_the_oracle_to_the_bit(n, c, transposed, dtype):
    rng = np.random.default_rng(100 * n + c)
    t, x = (bf16 if dtype == "bf16" else f32)(hard_rows(rng, n, c, 3.3e38))
    x8, xs, xt8, xts = B.aeris_fp8_quantize(t, transposed=transposed)
    torch.cuda.synchronize()
    got, want = codes(x8, xs), fo.quantize(x)
    same_codes(got[0], want[0])
    assert (got[1] == want[1]).all()
    if not transposed:
        assert xt8 is None and xts is None
        return
    got, want = codes(xt8, xts), fo.quantize(x.T)
    same_codes(got[0], want[0])
    assert (got[1] == want[1]).all()
    none, none2, a, b = B.aeris_fp8_quantize(t, rows=False, transposed=True)
    torch.cuda.synchronize()
    assert none is None and none2 is None
    assert torch.equal(a.view(torch.uint8), xt8.view(torch.uint8)) and torch.equal(b.view(torch.uint8), xts.view(torch.uint8))


# ------------------------------------------------------------------------------------- computed values
def close_quantized(name, got, h, mag):
    """got: (codes, scales); h: what was quantised, in 64 bits; mag: sum of magnitudes of each value's terms."""
    q, scales = got
    n, c = h.shape
    value = fo.dequantize(q, scales)
    allow = np.maximum(2.0 ** -4 * np.abs(h), 2.0 ** -10 * fo.per_column(scales, c)) + 1.07 * SLACK * mag
    err = np.abs(value - h)
    parity_log.add(name, "e4m3", np.linalg.norm(err) / np.linalg.norm(h), err.max(), np.abs(h).max(), allow.max())
    assert (err <= allow).all()
    want = fo.quantize(h)[1]
    blocks = -(-c // 128)
    assert (scales[:, blocks:] == 127).all()
    for b in range(blocks):
        part = np.abs(h[:, b * 128:(b + 1) * 128])
        off = scales[:, b].astype(int) - want[:, b].astype(int)
        slack = (SLACK * mag[:, b * 128:(b + 1) * 128]).max(axis=1)
        border = 448.0 * 2.0 ** (np.minimum(scales[:, b], want[:, b]) - 127.0)
        assert ((off == 0) | ((np.abs(off) == 1) & (np.abs(part.max(axis=1) - border) <= slack))).all()


@pytest.mark.parametrize("samples,rows,c,residual", [
    (1, 1, 64, True), (1, 3, 128, False), (2, 5, 192, True), (3, 37, 320, False), (1, 130, 576, True),
    (5, 9, 1088, True), (1, 70, 2048, True), (2, 33, 2112, False), (1, 20, 4096, True), (300, 1, 64, True)])
def test_residual_norm(samples, rows, c, residual):
    rng = np.random.default_rng(7 * c + rows)
    n, eps = samples * rows, 1e-6
    tx, x = bf16(rows_with_gain(rng, n, c))
    ty, y = bf16(rows_with_gain(rng, n, c))
    (tw, w), (ta, a), (tg, g), (tb, b) = [f32(v) for v in (
        1 + 0.1 * rng.standard_normal(c), 0.8 * rng.standard_normal((samples, c)),
        0.3 * rng.standard_normal((samples, c)), 0.5 * rng.standard_normal((samples, c)))]
    s, r, h8, hs = B.aeris_residual_norm_fp8_fwd(tx, ty if residual else None, ta if residual else None, tw, tg, tb,
                                                 eps, rows)
    torch.cuda.synchronize()
    if residual:
        assert torch.equal(s.view(torch.int16), B.aeris_gate_residual_fwd(tx, ty, ta, rows).view(torch.int16))
        exact = x + np.repeat(a, rows, 0) * y
        # half a bf16 step, and one fp32 rounding of the sum before it (an ulp where it meets a border)
        assert (np.abs(to_f64(s) - exact) <= 2.0 ** -8 * np.abs(exact) + 2.0 ** -23 * (np.abs(x) + np.abs(np.repeat(a, rows, 0) * y))).all()
    else:
        assert s is tx
    _, r_apart = B.aeris_rmsnorm_adaln_fwd(s, tw, tg, tb, eps, rows)
    assert torch.equal(r, r_apart)
    h, _ = bo.rmsnorm_adaln_fwd(to_f64(s), w, g, b, eps, rows)
    mag = np.abs(h - np.repeat(b, rows, 0)) + np.abs(np.repeat(b, rows, 0))
    close_quantized("h", codes(h8, hs), h, mag)
    s2, r2, h82, hs2 = B.aeris_residual_norm_fp8_fwd(tx, ty if residual else None, ta if residual else None, tw, tg,
                                                     tb, eps, rows, want_r=False)
    torch.cuda.synchronize()
    assert r2 is None and torch.equal(h8.view(torch.uint8), h82.view(torch.uint8))
    assert torch.equal(hs.view(torch.uint8), hs2.view(torch.uint8))


@pytest.mark.parametrize("c", [192, 1024])
def test_residual_norm_in_place(c):
    rng = np.random.default_rng(c)
    n = 45
    tx, _ = bf16(rows_with_gain(rng, n, c))
    ty, _ = bf16(rows_with_gain(rng, n, c))
    ta, tw, tg, tb = [f32(rng.standard_normal(v))[0] for v in ((1, c), c, (1, c), (1, c))]
    s, r, h8, hs = B.aeris_residual_norm_fp8_fwd(tx, ty, ta, tw, tg, tb, 1e-6, n)
    for which in (0, 1):
        pair = [tx.clone(), ty.clone()]
        s2, r2, h82, hs2 = B.aeris_residual_norm_fp8_fwd(*pair, ta, tw, tg, tb, 1e-6, n, s=pair[which])
        torch.cuda.synchronize()
        assert s2 is pair[which]
        for p, q in ((s, s2), (r, r2), (h8, h82), (hs, hs2)):
            assert torch.equal(p.view(torch.uint8), q.view(torch.uint8))
        assert torch.equal(pair[1 - which], (tx, ty)[1 - which])


def test_residual_norm_rows_that_are_not_finite_stay_alone():
    rng = np.random.default_rng(2)
    n, c = 12, 320
    x = rows_with_gain(rng, n, c)
    x[3, 7], x[8, 200], x[10] = np.inf, np.nan, 0.0
    tx, _ = bf16(x)
    tw, tg, tb = [f32(rng.standard_normal(v))[0] for v in (c, (1, c), (1, c))]
    _, r, h8, hs = B.aeris_residual_norm_fp8_fwd(tx, None, None, tw, tg, tb, 1e-6, n)
    torch.cuda.synchronize()
    value = fo.dequantize(*codes(h8, hs))
    assert np.isnan(value[8]).all() and np.isnan(value[3, 7])
    fine = [i for i in range(n) if i not in (3, 8)]
    assert np.isfinite(value[fine]).all()
    assert np.allclose(value[10], fo.round_trip(to_f64(tb))[0])            # a row of zeros: beta


@pytest.mark.parametrize("n,hidden", [(1, 64), (2, 128), (5, 192), (61, 576), (300, 1344), (40, 5504)])
def test_swiglu(n, hidden):
    rng = np.random.default_rng(hidden + n)
    uv = rows_with_gain(rng, n, 2 * hidden)
    uv[0, :8] = [0.0, -0.0, 90.0, -90.0, 300.0, -300.0, 1e-30, -1e-30]
    t, v = bf16(uv)
    g8, gs = B.aeris_swiglu_fp8_fwd(t)
    torch.cuda.synchronize()
    g = bo.swiglu_fwd(v)
    close_quantized("g", codes(g8, gs), g, np.abs(g))


# ------------------------------------------------------------------------------------- projection
def operand(rng, n, c):
    """A quantised matrix as (device pair, values)."""
    q, scales = fo.quantize(rows_with_gain(rng, n, c))
    return dev(q, scales), fo.dequantize(q, scales)


def product_slack(x, w):
    """What the sums of x w^T may be off by, see the head of this file."""
    c = x.shape[1]
    groups = lambda a: np.abs(a).reshape(a.shape[0], c // 8, 8).max(axis=2)
    return 7 * 2.0 ** -13 * (groups(x) @ groups(w).T) + (c / 32 + 8) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T)


def close_product(name, got, x, w):
    ref, slack = fo.linear_fwd(x, w), product_slack(x, w)
    got = to_f64(got)
    err = np.abs(got - ref)
    allow = 2.0 ** -8 * np.abs(ref) + 1.01 * slack + 1e-30
    rel = np.linalg.norm(err) / np.linalg.norm(ref)
    parity_log.add(name, "bf16", rel, err.max(), np.abs(ref).max(), allow.max())
    assert np.isfinite(got).all() and (err <= allow).all()
    if ref.size >= 4096:
        assert rel <= 3e-3      # output rounding alone is 2^-9 / sqrt 3 * (up to 2, by the mantissa) = 1.7e-3


SIZES = [
    # rows, channels, out features
    (1, 64, 64), (1, 2048, 192), (1, 192, 1088), (3, 128, 64), (15, 320, 128), (16, 576, 320), (17, 512, 64),
    (31, 1024, 256), (33, 64, 448), (48, 640, 192), (63, 704, 64), (64, 128, 128), (65, 2112, 64), (127, 192, 192),
    (128, 256, 576), (129, 1088, 320), (257, 128, 1600), (1000, 64, 2048), (700, 448, 4160), (4100, 192, 1088),
    (2500, 1600, 2112),
]


@pytest.mark.parametrize("n,c,f", SIZES)
def test_linear(n, c, f):
    rng = np.random.default_rng(n + 3 * c + 7 * f)
    (x8, xs), x = operand(rng, n, c)
    (w8, ws), w = operand(rng, f, c)
    guard = torch.full((n + 2, f), 123.0, dtype=torch.bfloat16, device="cuda")
    y = B.aeris_linear_fp8_fwd(x8, xs, w8, ws, y=guard[1:n + 1])
    torch.cuda.synchronize()
    close_product("y", y, x, w)
    assert (guard[0] == 123).all() and (guard[n + 1] == 123).all()       # rows beside the output are left as they were
    again = B.aeris_linear_fp8_fwd(x8, xs, w8, ws)
    torch.cuda.synchronize()
    assert torch.equal(y.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("n,c,f,plan", [
    # a few rows: one, two and four blocks of 16; steps shared by eight waves, fewer steps than waves, half a last step
    (1, 2048, 12288, (16, False)), (1, 1600, 64, (16, False)), (16, 5504, 192, (16, False)), (17, 64, 64, (16, False)),
    (31, 1216, 320, (16, False)), (33, 448, 192, (16, False)), (64, 2112, 128, (16, False)),
    (64, 2048, 11008, (64, False)),          # as few rows, but many features: tiles
    (65, 2112, 64, (64, False)), (129, 1088, 320, (64, False)), (1000, 64, 2048, (64, False)),
    (4100, 192, 1088, (128, False)), (2500, 1600, 2112, (128, False)),
    # the largest tiles: two steps, and lengths that leave 0 to 3 steps in the last group of scales; last blocks of 128
    # and of 64 channels; one tile per workgroup and several; both orders of tiles; rows and features past whole tiles
    (16217, 256, 896, (256, True)), (16310, 192, 832, (256, True)), (26827, 192, 1664, (256, False)),
    (8178, 320, 1920, (256, True)), (18458, 320, 1728, (256, False)), (11760, 384, 2112, (256, True)),
    (8128, 448, 1984, (256, True)), (24740, 512, 960, (256, True)), (8085, 576, 2048, (256, True)),
    (22383, 576, 1088, (256, True)), (24675, 576, 1088, (256, False)), (22105, 640, 1088, (256, True)),
    (16473, 704, 1472, (256, True)),
])
def test_linear_by_its_plan(n, c, f, plan):
    """Sizes that reach each way of computing the product; every row of a workgroup tile's ends is there."""
    assert B.aeris_linear_fp8_plan(n, c, f) == plan
    test_linear(n, c, f)


@pytest.mark.parametrize("n,c,f", [(172801, 1216, 2112), (400000, 320, 960), (20011, 5504, 2048), (4608, 2048, 65536)])
def test_linear_of_many_tiles_on_samples(n, c, f):
    """Long walks over tiles: sampled rows and features, among them those where tiles meet and end."""
    rng = np.random.default_rng(n)
    gen = torch.Generator(device="cuda").manual_seed(n)
    x8, xs, _, _ = B.aeris_fp8_quantize(torch.randn(n, c, device="cuda", dtype=torch.bfloat16, generator=gen))
    w8, ws, _, _ = B.aeris_fp8_quantize(torch.randn(f, c, device="cuda", generator=gen))
    y = B.aeris_linear_fp8_fwd(x8, xs, w8, ws)
    torch.cuda.synchronize()
    assert B.aeris_linear_fp8_plan(n, c, f)[0] == 256
    rows = np.unique(np.concatenate([[0, 1, 255, 256, n - 257, n - 256, n - 255, n - 2, n - 1], rng.integers(0, n, 40)]))
    cols = np.unique(np.concatenate([[0, 63, 255, 256, f - 257, f - 256, f - 1], rng.integers(0, f, 40)]))
    x = fo.dequantize(*codes(x8[rows], xs.view(torch.uint8)[rows].view(torch.float8_e8m0fnu)))
    w = fo.dequantize(*codes(w8[cols], ws.view(torch.uint8)[cols].view(torch.float8_e8m0fnu)))
    close_product("y", y[rows][:, cols], x, w)


@pytest.mark.parametrize("n", [2, 40, 300, 3000])
def test_linear_applies_each_block_its_scale(n):
    """Blocks of very unlike scales; whole numbers whose sums fp32 holds, so the result is exact before its rounding."""
    rng = np.random.default_rng(n)
    c, f = 1216, 192
    q = lambda rows: fo.encode(rng.integers(-8, 9, (rows, c)).astype(float))
    scales = lambda rows: np.concatenate([rng.integers(124, 131, (rows, 10)), np.full((rows, 2), 127)], 1).astype(np.uint8)
    xq, xs, wq, ws = q(n), scales(n), q(f), scales(f)
    y = B.aeris_linear_fp8_fwd(*dev(xq, xs), *dev(wq, ws))
    torch.cuda.synchronize()
    ref = fo.linear_fwd(fo.dequantize(xq, xs), fo.dequantize(wq, ws))     # multiples of 2^-6, below 2^18: exact
    want = torch.from_numpy(ref).float().bfloat16()
    assert torch.equal(y.cpu().view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("n,c,f", [(5, 192, 64), (100, 704, 192), (600, 320, 1088)])
def test_linear_keeps_nan_to_its_rows_and_features(n, c, f):
    rng = np.random.default_rng(9)
    xq, xs = fo.quantize(rows_with_gain(rng, n, c))
    wq, ws = fo.quantize(rows_with_gain(rng, f, c))
    xq[n // 2, c - 1], wq[f // 3, 0], xs[n - 1, 0] = 0x7f, 0xff, 127 + 100
    y = to_f64(B.aeris_linear_fp8_fwd(*dev(xq, xs), *dev(wq, ws)))
    bad = np.isnan(y)
    assert bad[n // 2].all() and bad[:, f // 3].all()
    bad[n // 2], bad[:, f // 3] = False, False
    assert not bad.any()


@pytest.mark.parametrize("n,c,f", [(1, 64, 64), (40, 128, 192), (64, 2048, 64), (131, 192, 576), (1000, 576, 320),
                                   (2125, 64, 128), (1100, 1088, 1600)])
def test_linear_bwd(n, c, f):
    rng = np.random.default_rng(n + c + f)
    (x8, xs), x = operand(rng, n, c)
    tw, w = bf16(rng.standard_normal((f, c)) / np.sqrt(c))
    _, _, wt8, wts = B.aeris_fp8_quantize(tw, rows=False, transposed=True)
    tdy, dy = bf16(rows_with_gain(rng, n, f))
    dx, dw = B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, tdy)
    torch.cuda.synchronize()
    wt = fo.dequantize(*codes(wt8, wts))
    close_product("dx", dx, fo.round_trip(dy), wt)
    # dW: the values are exact in bf16, so it is the gradient of a bf16 projection of them to the bit
    _, want = B.aeris_linear_bwd(torch.from_numpy(x).cuda().bfloat16(), tw, tdy, want_dx=False)
    assert torch.equal(dw, want)
    err, mag = np.abs(to_f64(dw) - dy.T @ x), np.abs(dy).T @ np.abs(x)
    assert (err <= max(1e-5, 4.0 * np.sqrt(n) * 2.0 ** -24) * mag).all()
    # each alone, without the other's operands
    dx2, none = B.aeris_linear_fp8_bwd(None, None, wt8, wts, tdy, want_dweight=False)
    none2, dw2 = B.aeris_linear_fp8_bwd(x8, xs, None, None, tdy, want_dx=False)
    torch.cuda.synchronize()
    assert none is None and none2 is None
    assert torch.equal(dx.view(torch.int16), dx2.view(torch.int16)) and torch.equal(dw, dw2)


def test_linear_gradients_against_differences():
    """Sums of y dy along two directions of the quantised operands, from the library's own forward products: y is
    linear in each operand, so a difference is exact up to the rounding of y (2^-8 of each |y dy|)."""
    rng = np.random.default_rng(31)
    n, c, f = 96, 256, 192
    (x8, xs), x = operand(rng, n, c)
    (u8, us), u = operand(rng, n, c)
    tw, _ = bf16(rng.standard_normal((f, c)) / 16.0)
    tv, _ = bf16(rng.standard_normal((f, c)) / 16.0)
    w8, ws, wt8, wts = B.aeris_fp8_quantize(tw, transposed=True)
    v8, vs, _, _ = B.aeris_fp8_quantize(tv)
    tdy, dy = bf16(fo.round_trip(rng.standard_normal((n, f))))            # quantising it again changes nothing
    dx, dw = B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, tdy)
    w, v = fo.dequantize(*codes(w8, ws)), fo.dequantize(*codes(v8, vs))
    # the transposed weight is quantised along the other side: equal where no value fell below the range of its block
    assert (fo.dequantize(*codes(wt8, wts)).T == w).mean() > 0.99
    for (a8, a_s, b8, b_s), inner in (((u8, us, w8, ws), (to_f64(dx) * u).sum()),
                                      ((x8, xs, v8, vs), (to_f64(dw) * v).sum())):
        y = to_f64(B.aeris_linear_fp8_fwd(a8, a_s, b8, b_s))
        assert abs((y * dy).sum() - inner) <= 2.0 ** -8 * (np.abs(y) * np.abs(dy)).sum() + 2.0 ** -8 * (np.abs(to_f64(dx) * u)).sum()


# ------------------------------------------------------------------------------------- used together
def feed_forward(t, rows):
    """The feed-forward half of a layer, forward and backward, as a training step runs it."""
    s, r, h8, hs = B.aeris_residual_norm_fp8_fwd(t["x"], t["y"], t["alpha"], t["w"], t["gamma"], t["beta"], 1e-6, rows)
    up8, ups, upt8, upts = B.aeris_fp8_quantize(t["up"], transposed=True)
    down8, downs, downt8, downts = B.aeris_fp8_quantize(t["down"], transposed=True)
    uv = B.aeris_linear_fp8_fwd(h8, hs, up8, ups)
    g8, gs = B.aeris_swiglu_fp8_fwd(uv)
    out = B.aeris_linear_fp8_fwd(g8, gs, down8, downs)
    dg, ddown = B.aeris_linear_fp8_bwd(g8, gs, downt8, downts, t["dout"])
    duv = B.aeris_swiglu_bwd(uv, dg)
    dh, dup = B.aeris_linear_fp8_bwd(h8, hs, upt8, upts, duv)
    ds, dw, dgamma, dbeta = B.aeris_rmsnorm_adaln_bwd(s, t["w"], t["gamma"], r, dh, rows, dres=t["ds"])
    dy, dalpha = B.aeris_gate_residual_bwd(t["y"], t["alpha"], ds, rows)
    return dict(s=s, r=r, uv=uv, out=out, ddown=ddown, dup=dup, dx=ds, dy=dy, dw=dw, dgamma=dgamma, dbeta=dbeta,
                dalpha=dalpha, dg=dg, duv=duv, dh=dh, h=(h8, hs), g=(g8, gs), up8=(up8, ups), upt8=(upt8, upts),
                down8=(down8, downs), downt8=(downt8, downts))


def same_bits(a, b):
    return all(same_bits(p, q) for p, q in zip(a, b)) if isinstance(a, tuple) else torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def feed_forward_inputs(rng, samples, rows, c, hidden):
    n = samples * rows
    arrays = dict(x=rows_with_gain(rng, n, c), y=rng.standard_normal((n, c)), dout=rng.standard_normal((n, c)),
                  ds=rng.standard_normal((n, c)), up=rng.standard_normal((2 * hidden, c)) / np.sqrt(c),
                  down=rng.standard_normal((c, hidden)) / np.sqrt(hidden))
    t = {k: bf16(v) for k, v in arrays.items()}
    t.update(w=f32(1 + 0.1 * rng.standard_normal(c)), alpha=f32(0.8 * rng.standard_normal((samples, c))),
             gamma=f32(0.3 * rng.standard_normal((samples, c))), beta=f32(0.5 * rng.standard_normal((samples, c))))
    return {k: v[0] for k, v in t.items()}, {k: v[1] for k, v in t.items()}


def test_feed_forward_half_of_a_layer():
    """Against the chain in 64 bits with the same roundings to 8 bits (straight through in the backward pass).

    How far the two may be apart.  A relative difference d in front of a rounding to 8 bits (steps of 1/16 to 1/8 of
    the value, 0.09 in the mean) moves a value by a step with the probability d * 0.8 / 0.09, so the quantised values
    differ by sqrt(0.072 d) in the mean.  s is rounded to bf16 here and not there: d = 1.7e-3, so h8 and with it uv
    differ by 1.1e-2.  The gate has two such factors: 1.6e-2 in front of g8, behind it sqrt(0.072 * 1.6e-2) = 3.4e-2
    (out, ddown).  duv has uv's difference twice or less, so its quantised form, dh and the sums over dh (dw, dgamma,
    dbeta, dx, dy, dalpha) differ by 3.4e-2 too.  Allowed is twice that; uv alone 2.2e-2, s and r 3.4e-3."""
    rng = np.random.default_rng(41)
    samples, rows, c, hidden = 2, 150, 256, 704
    t, a = feed_forward_inputs(rng, samples, rows, c, hidden)
    got = feed_forward(t, rows)
    torch.cuda.synchronize()
    ref = {}
    ref["s"] = bo.gate_residual_fwd(a["x"], a["y"], a["alpha"], rows)
    h, ref["r"] = bo.rmsnorm_adaln_fwd(ref["s"], a["w"], a["gamma"], a["beta"], 1e-6, rows)
    h = fo.round_trip(h)
    ref["uv"] = fo.linear_fwd(h, fo.round_trip(a["up"]))
    g = fo.round_trip(bo.swiglu_fwd(ref["uv"]))
    ref["out"] = fo.linear_fwd(g, fo.round_trip(a["down"]))
    dg, ref["ddown"] = fo.linear_bwd(g, fo.round_trip(a["down"].T), a["dout"])
    duv = bo.swiglu_bwd(ref["uv"], dg)
    dh, ref["dup"] = fo.linear_bwd(h, fo.round_trip(a["up"].T), duv)
    ref["dx"], ref["dw"], ref["dgamma"], ref["dbeta"] = bo.rmsnorm_adaln_bwd_residual(
        ref["s"], a["w"], a["gamma"], a["beta"], 1e-6, rows, dh, a["ds"])
    _, ref["dy"], ref["dalpha"] = bo.gate_residual_bwd(a["y"], a["alpha"], ref["dx"], rows)
    for name in ref:
        x, want = to_f64(got[name]), ref[name]
        rel = np.linalg.norm(x - want) / np.linalg.norm(want)
        allow = dict(s=3.4e-3, r=3.4e-3, uv=2.2e-2).get(name, 6.8e-2)
        parity_log.add(name, "", rel, np.abs(x - want).max(), np.abs(want).max(), allow)
        assert rel <= allow, name


def test_stages_of_the_feed_forward_half():
    """Each stage from the operands that the stage before it left, to the bounds of the single calls."""
    rng = np.random.default_rng(41)
    samples, rows, c, hidden = 2, 150, 256, 704
    t, a = feed_forward_inputs(rng, samples, rows, c, hidden)
    got = feed_forward(t, rows)
    torch.cuda.synchronize()
    held = lambda name: fo.dequantize(*codes(*got[name]))
    v = {k: to_f64(got[k]) for k in ("s", "uv", "dg", "duv")}
    h, _ = bo.rmsnorm_adaln_fwd(v["s"], a["w"], a["gamma"], a["beta"], 1e-6, rows)
    beta = np.abs(np.repeat(a["beta"], rows, 0))
    close_quantized("h", codes(*got["h"]), h, np.abs(h) + 2 * beta)
    close_product("uv", got["uv"], held("h"), held("up8"))
    g = bo.swiglu_fwd(v["uv"])
    close_quantized("g", codes(*got["g"]), g, np.abs(g))
    close_product("out", got["out"], held("g"), held("down8"))
    close_product("dg", got["dg"], fo.round_trip(a["dout"]), held("downt8"))
    close_product("dh", got["dh"], fo.round_trip(v["duv"]), held("upt8"))
    for name, dy, x in (("ddown", a["dout"], held("g")), ("dup", v["duv"], held("h"))):
        assert (np.abs(to_f64(got[name]) - dy.T @ x) <= 1e-5 * np.abs(dy).T @ np.abs(x)).all()


@pytest.mark.parametrize("n,c,f", [(30000, 1216, 1088), (40, 1216, 192)])
def test_linear_scales_in_other_shapes(n, c, f):
    """As test_linear_applies_each_block_its_scale, for the largest tiles (groups of four scales) and a few rows."""
    assert B.aeris_linear_fp8_plan(n, c, f)[0] == (256 if n == 30000 else 16)
    gen = torch.Generator(device="cuda").manual_seed(5)
    whole = lambda rows: torch.randint(-8, 9, (rows, c), device="cuda", generator=gen)
    powers = lambda rows: torch.cat([torch.randint(124, 131, (rows, 10), device="cuda", generator=gen),
                                     torch.full((rows, 2), 127, device="cuda")], 1).to(torch.uint8)
    xq, xs, wq, ws = whole(n), powers(n), whole(f), powers(f)
    y = B.aeris_linear_fp8_fwd(xq.float().to(torch.float8_e4m3fn), xs.view(torch.float8_e8m0fnu),
                               wq.float().to(torch.float8_e4m3fn), ws.view(torch.float8_e8m0fnu))
    value = lambda q, s: q.double() * torch.exp2(s.double() - 127).repeat_interleave(128, 1)[:, :c]
    want = value(xq, xs) @ value(wq, ws).t().contiguous()                # multiples of 2^-6, below 2^18: exact
    assert torch.equal(y, want.float().bfloat16())


def test_captured_and_replayed_beside_eager_calls():
    """The whole half in a HIP graph: replays with new inputs in place, eager work on other inputs between them."""
    rng = np.random.default_rng(43)
    rows, c, hidden = 90, 192, 320
    sets = [feed_forward_inputs(rng, 1, rows, c, hidden)[0] for _ in range(3)]
    want = [feed_forward(t, rows) for t in sets]
    held = {k: v.clone() for k, v in sets[0].items()}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        feed_forward(held, rows)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = feed_forward(held, rows)
    for i in (1, 0, 2, 1):
        for k in held:
            held[k].copy_(sets[i][k])
        graph.replay()
        feed_forward(sets[(i + 1) % 3], rows)
        torch.cuda.synchronize()
        for k in got:
            assert same_bits(got[k], want[i][k]), k


def test_calls_on_two_streams_at_once():
    rng = np.random.default_rng(47)
    rows, c, hidden = 200, 256, 448
    sets = [feed_forward_inputs(rng, 1, rows, c, hidden)[0] for _ in range(2)]
    want = [feed_forward(t, rows) for t in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(3):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(feed_forward(sets[i], rows))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            for k in g:
                assert same_bits(g[k], want[i][k]), k


# ------------------------------------------------------------------------------------- refusals
def test_errors_are_reported():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.AerisError) as e:
        B.aeris_fp8_quantize(bf(8, 100))
    assert e.value.code == -3
    with pytest.raises(B.AerisError) as e:
        B.aeris_fp8_quantize(bf(100, 64), transposed=True)
    assert e.value.code == -3
    with pytest.raises(B.AerisError) as e:
        B.aeris_fp8_quantize(bf(64, 64), rows=False)
    assert e.value.code == -1
    with pytest.raises(B.AerisError) as e:
        B.aeris_swiglu_fp8_fwd(bf(8, 144))
    assert e.value.code == -3
    z = torch.zeros
    with pytest.raises(B.AerisError) as e:
        B.aeris_residual_norm_fp8_fwd(bf(8, 64), bf(8, 64), None, z(64, device="cuda"), z(2, 64, device="cuda"),
                                      z(2, 64, device="cuda"), 1e-6, 4)
    assert e.value.code == -1
    x8, xs, _, _ = B.aeris_fp8_quantize(bf(64, 128))
    w8, ws, wt8, wts = B.aeris_fp8_quantize(bf(64, 64), transposed=True)
    with pytest.raises(AssertionError):
        B.aeris_linear_fp8_fwd(x8, xs, w8, ws)                        # 128 and 64 channels
    with pytest.raises(AssertionError):
        B.aeris_linear_fp8_fwd(x8, xs[:, :2].contiguous(), w8, ws)    # scales of another size
    with pytest.raises(ValueError):
        B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, bf(64, 64), want_dx=False, want_dweight=False)
    with pytest.raises(B.AerisError) as e:
        B.aeris_linear_fp8_bwd(w8, ws, wt8, wts, bf(64, 64), workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -8


@pytest.mark.parametrize("change", ["w", "gamma", "beta", "alpha", "y", "s"])
def test_residual_norm_refuses_operands_of_another_size(change):
    rows = lambda n: torch.zeros(n, 64, dtype=torch.bfloat16, device="cuda")
    z = lambda n: torch.zeros(n, 64, device="cuda")
    k = dict(x=rows(8), y=rows(8), alpha=z(2), w=z(1), gamma=z(2), beta=z(2), eps=1e-6, rows_per_sample=4, s=rows(8))
    B.aeris_residual_norm_fp8_fwd(**k)
    k[change] = rows(4) if change in "ys" else torch.zeros(32, device="cuda") if change == "w" else z(1)
    with pytest.raises(AssertionError):
        B.aeris_residual_norm_fp8_fwd(**k)


def test_linear_refuses_operands_of_another_place():
    q = lambda n, c: B.aeris_fp8_quantize(torch.zeros(n, c, dtype=torch.bfloat16, device="cuda"))[:2]
    (x8, xs), (w8, ws) = q(3, 64), q(64, 64)
    for at in range(4):
        args = [x8, xs, w8, ws]
        args[at] = args[at].cpu()
        with pytest.raises(AssertionError):
            B.aeris_linear_fp8_fwd(*args)
    with pytest.raises(AssertionError):
        B.aeris_linear_fp8_fwd(x8, xs, w8, ws, y=torch.zeros(3, 128, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(AssertionError):
        B.aeris_linear_fp8_bwd(w8, ws, w8, ws, torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda"),
                               workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda")[::2])


@pytest.mark.parametrize("n,c,f,parts", [
    (2048, 2048, 2048, 2), (1990, 1344, 1984, 2), (500, 1600, 7104, 2), (2048, 5504, 1984, 2), (1999, 1216, 2048, 2),
    (64, 2048, 11008, 4), (65, 5504, 64, 4), (192, 2112, 128, 4), (129, 1088, 128, 4), (1000, 1216, 1024, 4), (65, 704, 64, 4),
    (257, 448, 64, 4), (1000, 64, 2048, 1), (2500, 1600, 2112, 1), (1, 5504, 2048, 8), (17, 5504, 2048, 8), (64, 768, 2304, 8),
])
def test_linear_in_parts_of_the_channels(n, c, f, parts):
    """Groups of waves that share the channels: parts of equal and unequal length, half a last block, ends of tiles."""
    assert B.aeris_linear_fp8_parts(n, c, f) == parts
    test_linear(n, c, f)


def test_linear_keeps_scales_and_nan_in_parts_of_the_channels():
    """Blocks of unlike scales in every part, whole numbers: exact.  A row that is not finite stays alone."""
    n, c, f = 200, 1344, 128
    assert B.aeris_linear_fp8_parts(n, c, f) == 4
    rng = np.random.default_rng(3)
    q = lambda rows: fo.encode(rng.integers(-8, 9, (rows, c)).astype(float))
    scales = lambda rows: np.concatenate([rng.integers(124, 131, (rows, 11)), np.full((rows, 1), 127)], 1).astype(np.uint8)
    xq, xs, wq, ws = q(n), scales(n), q(f), scales(f)
    want = fo.dequantize(xq, xs) @ fo.dequantize(wq, ws).T               # multiples of 2^-6, below 2^18: exact
    want = torch.from_numpy(want).float().bfloat16()
    y = B.aeris_linear_fp8_fwd(*dev(xq, xs), *dev(wq, ws)).cpu()
    assert torch.equal(y, want)
    xq[150, c - 1] = 0x7f
    y = B.aeris_linear_fp8_fwd(*dev(xq, xs), *dev(wq, ws)).cpu()
    assert torch.isnan(y[150]).all() and torch.equal(y[:150], want[:150]) and torch.equal(y[151:], want[151:])


@pytest.mark.parametrize("power", [-126, -132, -140])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_rows_of_subnormal_numbers(power, dtype):
    """Blocks below the smallest normal number: the smallest scale, codes down to zero, their signs kept."""
    rng = np.random.default_rng(-power)
    t, x = (bf16 if dtype == "bf16" else f32)(np.ldexp(rng.standard_normal((64, 192)), power))
    x8, xs, xt8, xts = B.aeris_fp8_quantize(t, transposed=True)
    torch.cuda.synchronize()
    for got, want in ((codes(x8, xs), fo.quantize(x)), (codes(xt8, xts), fo.quantize(x.T))):
        same_codes(got[0], want[0])
        assert (got[1] == want[1]).all()


def test_captured_gradients_and_products_of_few_tiles():
    """Calls whose waves share the channels and both layouts of the gradients' workspace, captured and replayed with new
    inputs in place, eager work between the replays."""
    sizes = [(130, 1088, 192), (2100, 64, 128), (17, 2112, 64)]
    ins, graph, outs = [], torch.cuda.CUDAGraph(), []
    gen = torch.Generator(device="cuda").manual_seed(9)
    draw = lambda *shape: torch.randn(*shape, device="cuda", generator=gen).bfloat16()
    def call(x, w, dy):
        x8, xs, _, _ = B.aeris_fp8_quantize(x)
        w8, ws, wt8, wts = B.aeris_fp8_quantize(w, transposed=True)
        return (B.aeris_linear_fp8_fwd(x8, xs, w8, ws),) + B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, dy)
    for n, c, f in sizes:
        ins.append((draw(n, c), draw(f, c), draw(n, f)))
    for v in ins:
        call(*v)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        outs = [call(*v) for v in ins]
    for _ in range(3):
        for v in ins:
            for t in v:
                t.copy_(draw(*t.shape))
        want = [call(*v) for v in ins]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert all(same_bits(p, q) for p, q in zip(a, b))
        draw(1000, 1000).float().sum().item()


@pytest.mark.parametrize("n,hidden,v_power", [(41, 64, 0), (41, 192, 20), (130, 576, 90), (130, 576, 125)])
def test_swiglu_far_below_zero(n, hidden, v_power):
    """Blocks of nothing but u < -80, where silu(u) v is held as long as the format holds it: 1 + exp(-u) passes fp32
    below -88.7 and silu(u) leaves the normal numbers below -92, their product with a large v not before -180."""
    rng = np.random.default_rng(n + hidden + v_power)
    u = -80.0 - (12.0 + 0.8 * v_power) * rng.random((n, 1)) - rng.random((n, hidden))
    v = rng.standard_normal((n, hidden)) * 2.0 ** v_power
    u[0], u[1], u[2] = -87.0, -87.5, -3e38                # the border of the two ways, and a gate of zero
    t, uv = bf16(np.concatenate([u, v], 1))
    q, scales = codes(*B.aeris_swiglu_fp8_fwd(t))
    g = bo.swiglu_fwd(uv)
    assert (np.abs(g).max(1) > 2.0 ** -126).sum() > 3
    # below the normal numbers fp32 has multiples of 2^-149, to half of which g is rounded: 1.07 * SLACK * 2^-131 covers it
    close_quantized("g far", (q, scales), g, np.abs(g) + 2.0 ** -131)


def test_swiglu_far_beside_near():
    """Far values beside ordinary ones change nothing of those, and values that are not finite stay alone."""
    rng = np.random.default_rng(53)
    n, hidden = 24, 320
    u, v = rng.standard_normal((2, n, hidden))
    t, _ = bf16(np.concatenate([u, v], 1))
    near = codes(*B.aeris_swiglu_fp8_fwd(t))
    u[:, 9::16] = -90.0 - 50.0 * rng.random((n, hidden // 16))
    u[5, 9], u[6, 9], u[7, 9] = -np.inf, np.inf, np.nan
    t, uv = bf16(np.concatenate([u, v], 1))
    q, scales = codes(*B.aeris_swiglu_fp8_fwd(t))
    with np.errstate(invalid="ignore"):
        g = bo.swiglu_fwd(uv)
    lost = np.zeros((n, hidden), dtype=bool)
    lost[5:8, 9] = True
    assert ((q & 127) == 127)[lost].all() and not ((q & 127) == 127)[~lost].any()
    g[lost], q[lost] = 0.0, 0
    close_quantized("g mixed", (q, scales), g, np.abs(g))
    ordinary = np.ones(hidden, dtype=bool)
    ordinary[9::16] = False
    same = np.repeat(scales[:, :3] == near[1][:, :3], 128, 1)[:, :hidden] & ordinary     # blocks of the same scale
    assert same.sum() > n * hidden // 2 and (q[same] == near[0][same]).all()


# --------------------------------------------------------------------------- sums over many channels
MANY_CHANNELS = [(15, 65536, 64, 16, 8), (40, 65472, 64, 64, 4), (1000, 65536, 2048, 64, 1), (2500, 65472, 512, 64, 1),
                 (700, 65536, 2048, 128, 2), (1500, 65472, 1024, 128, 2), (2500, 65472, 2048, 128, 1),
                 (2500, 65536, 4096, 256, 1), (2500, 65472, 4096, 256, 1)]


@pytest.mark.parametrize("n,c,f,tile,parts", MANY_CHANNELS)
def test_sums_of_many_channels_beside_a_large_block(n, c, f, tile, parts):
    """A first block that sums to one, thousands of products below its last bit, a last block that takes the one away
    again; so in every part of the channels.  What is left shows each error of the sums, of which the header states
        7 * 2^-13 * sum over groups of eight channels of the largest |x w|  +  (channels / 16 + 8) * 2^-23 * sum |x w|.
    With one part the first term covers half of the errors here: each block brings only its largest product into it,
    while each 16 channels lose up to a last bit of the one."""
    assert B.aeris_linear_fp8_plan(n, c, f)[0] == tile and B.aeris_linear_fp8_parts(n, c, f) == parts
    kinds, steps = 15, -(-c // 128)
    x = np.outer(np.arange(1, kinds + 1) * 2.0 ** -30, np.ones(c))
    for part in range(parts):
        first, last = steps * part // parts, steps * (part + 1) // parts - 1
        x[:, first * 128:first * 128 + 128] = 2.0 ** -7
        x[:, last * 128:last * 128 + 128] = -1.0 / (min(c, last * 128 + 128) - last * 128)
    xq, xs = fo.quantize(x)
    assert (fo.dequantize(xq, xs) == x).all()
    kind = torch.arange(n, device="cuda") % kinds
    tile_rows = lambda a: torch.from_numpy(a).cuda()[kind]
    w8, ws = fo.quantize(np.ones((1, c)))
    repeat = lambda a: torch.from_numpy(a).cuda().expand(f, -1).contiguous()
    y = B.aeris_linear_fp8_fwd(tile_rows(xq).view(torch.float8_e4m3fn), tile_rows(xs).view(torch.float8_e8m0fnu),
                               repeat(w8).view(torch.float8_e4m3fn), repeat(ws).view(torch.float8_e8m0fnu))
    torch.cuda.synchronize()
    assert (y == y[:, :1]).all() and (y[:, 0] == y[:kinds, 0][kind]).all()
    got, ref = to_f64(y[:kinds, 0]), x.sum(1)
    most, mag = np.abs(x).reshape(kinds, -1, 8).max(2).sum(1), np.abs(x).sum(1)
    err = np.abs(got - ref)
    print("error / sum |x w|", (err / mag).max(), "first term", (7 * 2.0 ** -13 * most / mag).min())
    assert (err <= 2.0 ** -8 * np.abs(ref) + 7 * 2.0 ** -13 * most + (c / 16 + 8) * 2.0 ** -23 * mag).all()


@pytest.mark.parametrize("n,c,f,tile", [(3, 65536, 64, 16), (40, 65472, 64, 64), (129, 65536, 128, 64)])
def test_linear_of_the_most_channels(n, c, f, tile):
    assert B.aeris_linear_fp8_plan(n, c, f)[0] == tile
    test_linear(n, c, f)


@pytest.mark.parametrize("n,c,f", [(40, 128, 2048), (131, 192, 576), (2125, 64, 128), (1100, 1088, 1600)])
def test_linear_bwd_within_the_workspace_of_what_is_wanted(n, c, f):
    """Each output alone, and both, with no byte more than is asked for and nothing written behind it."""
    rng = np.random.default_rng(n)
    (x8, xs), _ = operand(rng, n, c)
    _, _, wt8, wts = B.aeris_fp8_quantize(bf16(rng.standard_normal((f, c)))[0], rows=False, transposed=True)
    tdy, _ = bf16(rows_with_gain(rng, n, f))
    want = B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, tdy)
    for which in ((True, True), (True, False), (False, True)):
        need = B.aeris_linear_fp8_bwd_workspace_bytes_for(n, c, f, *which)
        space = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
        got = B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, tdy, *which, workspace=space[:need])
        torch.cuda.synchronize()
        assert (space[need:] == 0x5a).all()
        for wanted, g, w in zip(which, got, want):
            assert torch.equal(g, w) if wanted else g is None
        with pytest.raises(B.AerisError) as e:
            B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, tdy, *which, workspace=space[:need - 1])
        assert e.value.code == -8


# ------------------------------------------------------------------------------------- results passed in
def results_of_each_call():
    """(call with keyword arguments for its results, names of the results, those of a call without)."""
    rng = np.random.default_rng(61)
    t, _ = bf16(rows_with_gain(rng, 128, 192))
    y, _ = bf16(rows_with_gain(rng, 128, 192))
    uv, _ = bf16(rows_with_gain(rng, 128, 384))
    ta, tw, tg, tb = [f32(rng.standard_normal(v))[0] for v in ((2, 192), 192, (2, 192), (2, 192))]
    quantize = lambda **kw: B.aeris_fp8_quantize(t, transposed=True, **kw)
    norm = lambda **kw: B.aeris_residual_norm_fp8_fwd(t, y, ta, tw, tg, tb, 1e-6, 64, **kw)
    gate = lambda **kw: B.aeris_swiglu_fp8_fwd(uv, **kw)
    return [(call, names, call()) for call, names in (
        (quantize, ("x8", "xs", "xt8", "xts")), (norm, ("s", "r", "h8", "hs")), (gate, ("g8", "gs")))]


def test_results_passed_in():
    """All of them and each alone: written to the bits of a call that allocates, and returned as they are."""
    raw = lambda v: v.view(torch.uint8)
    for call, names, want in results_of_each_call():
        for given in (names,) + tuple((n,) for n in names):
            outs = {n: torch.empty_like(w) for n, w in zip(names, want) if n in given}
            for o in outs.values():
                raw(o).fill_(0x33)
            got = call(**outs)
            torch.cuda.synchronize()
            for name, g, w in zip(names, got, want):
                assert torch.equal(raw(g), raw(w)) and (name not in outs or g is outs[name])


def test_results_passed_in_are_refused_where_they_do_not_fit():
    for call, names, want in results_of_each_call():
        for name, w in zip(names, want):
            wide = torch.empty((2 * w.shape[0],) + w.shape[1:], dtype=w.dtype, device="cuda")
            for bad in (w[:-1], wide, wide[::2], torch.empty_like(w, dtype=torch.float16), w.cpu()):
                with pytest.raises(AssertionError):
                    call(**{name: bad})
    x = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    x8, xs, xt8, xts = B.aeris_fp8_quantize(x, transposed=True)
    for kw in (dict(rows=False, transposed=True, x8=x8), dict(rows=False, transposed=True, xs=xs), dict(xt8=xt8), dict(xts=xts)):
        with pytest.raises(AssertionError):
            B.aeris_fp8_quantize(x, **kw)


def test_norm_without_residual_refuses_a_sum_of_its_own():
    """Without y nothing is written to s, so that a buffer passed in for it would stay as it was; alpha is not read."""
    rng = np.random.default_rng(67)
    t, _ = bf16(rows_with_gain(rng, 8, 64))
    ta, tw, tg, tb = [f32(rng.standard_normal(v))[0] for v in ((2, 64), 64, (2, 64), (2, 64))]
    call = lambda alpha=None, **kw: B.aeris_residual_norm_fp8_fwd(t, None, alpha, tw, tg, tb, 1e-6, 4, **kw)
    with pytest.raises(AssertionError):
        call(s=torch.empty_like(t))
    want = call()
    for got in (call(s=t), call(alpha=ta), call(alpha=torch.full_like(ta, float("nan")))):
        assert got[0] is t and all(same_bits(g, w) for g, w in zip(got, want))


@pytest.mark.parametrize("n,c,f", [(96, 256, 192), (17, 1088, 64), (333, 192, 320), (500, 448, 576), (2500, 1600, 2112)])
def test_linear_gradients_along_themselves(n, c, f):
    """The library's gradients against its own forward products along them (gradient_check.py says what is allowed;
    test_a_wrong_gradient_shows_along_itself that wrong ones fail).  A gradient that lacks 64 terms of its sum is off by
    about 64 / terms of what is compared: less than that is allowed.  What is allowed grows with the square root of the
    terms (sums of magnitudes beside a sum of either sign): 0.8 % at 192, 2.0 % at 2112, 2.1 % at 2500 of them."""
    rng = np.random.default_rng(n + c + f)
    (x8, xs), x = operand(rng, n, c)
    tw, _ = bf16(rng.standard_normal((f, c)) / np.sqrt(c))
    w8, ws, wt8, wts = B.aeris_fp8_quantize(tw, transposed=True)
    tdy, dy = bf16(fo.round_trip(rows_with_gain(rng, n, f)))              # quantising it again changes nothing
    assert (fo.round_trip(dy) == dy).all()
    dx, dw = (to_f64(g) for g in B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, tdy))
    u, v = fo.quantize(dx), fo.quantize(dw)
    along_u = to_f64(B.aeris_linear_fp8_fwd(*dev(*u), w8, ws))
    along_v = to_f64(B.aeris_linear_fp8_fwd(x8, xs, *dev(*v)))
    w, wt = fo.dequantize(*codes(w8, ws)), fo.dequantize(*codes(wt8, wts))
    for (gap, allow, size), terms in ((gc.along_dx(along_u, dx, fo.dequantize(*u), dy, w, wt), f),
                                      (gc.along_dw(along_v, dw, fo.dequantize(*v), dy, x), n)):
        print("gap %.3e allowed %.3e of %.3e" % (gap, allow, size))
        assert gap <= allow <= min(0.05, 64 / terms) * size


# ------------------------------------------------------------------------------------- every form
def drawn_operand(gen, n, c):
    """A quantised matrix drawn on the device."""
    gain = torch.randn(c, device="cuda", generator=gen).exp()
    x = torch.randn(n, c, device="cuda", generator=gen) * gain
    return B.aeris_fp8_quantize(x)[:2]


def drawn_values(q, scales):
    """What it stands for, exact in bf16."""
    power = torch.exp2(scales.view(torch.uint8).float() - 127.0).repeat_interleave(128, 1)[:, :q.shape[1]]
    return (q.float() * power).bfloat16()


def sampled(rng, n, side):
    """Where tiles meet and end, and more."""
    edges = [0, 1, side - 1, side, n - side - 1, n - side, n - 2, n - 1]
    return np.unique(np.clip(np.concatenate([edges, rng.integers(0, n, 40)]), 0, n - 1))


@pytest.mark.parametrize("n,c,f,dx_form,dw_side,together", [
    (65, 1344, 2368, (64, 4), 128, True), (849, 2368, 128, (128, 1), 64, True), (16435, 128, 64, (128, 1), 64, False),
    (2435, 1152, 960, (128, 1), 128, True), (18569, 128, 2240, (128, 2), 128, False), (21193, 192, 1920, (128, 1), 128, False),
    (2241, 2432, 1728, (128, 1), 256, True), (8047, 1856, 256, (256, 1), 64, True), (99835, 256, 320, (256, 1), 64, False),
    (16207, 960, 448, (256, 1), 128, True), (114803, 448, 320, (256, 1), 128, False), (20701, 448, 1472, (256, 1), 256, True),
    (8445, 1024, 1600, (256, 1), 256, True), (116309, 448, 448, (256, 1), 256, False), (104617, 256, 832, (256, 1), 256, False)])
def test_linear_bwd_of_every_form(n, c, f, dx_form, dw_side, together):
    """Both gradients in each form of dx and side of dW's tiles, with dy's 8-bit rows inside dW's workspace, which dW's
    partial sums take over from them (`together`), and in the place of all of it; rows, channels and features past tiles."""
    assert (B.aeris_linear_fp8_plan(n, f, c)[0], B.aeris_linear_fp8_parts(n, f, c)) == dx_form
    assert B.aeris_linear_bwd_plan(n, c, f)[0] == dw_side
    for_dx = B.aeris_linear_fp8_bwd_workspace_bytes_for(n, c, f, True, False)
    assert (for_dx <= B.aeris_linear_bwd_workspace_bytes(n, c, f)) == together
    rng, gen = np.random.default_rng(n), torch.Generator(device="cuda").manual_seed(n)
    x8, xs = drawn_operand(gen, n, c)
    tw = torch.randn(f, c, device="cuda", generator=gen).bfloat16()
    _, _, wt8, wts = B.aeris_fp8_quantize(tw, rows=False, transposed=True)
    tdy = (torch.randn(n, f, device="cuda", generator=gen) * torch.randn(f, device="cuda", generator=gen).exp()).bfloat16()
    dx, dw = B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, tdy)
    torch.cuda.synchronize()
    # dx: sampled rows and channels against the oracle
    rows, cols, feats = sampled(rng, n, dx_form[0]), sampled(rng, c, dx_form[0]), sampled(rng, f, dw_side)
    wt = fo.dequantize(*codes(wt8[cols], wts.view(torch.uint8)[cols].view(torch.float8_e8m0fnu)))
    close_product("dx", dx[rows][:, cols], fo.round_trip(to_f64(tdy[rows])), wt)
    # dW: the bits of the bf16 gradient of the same values, and sampled entries against sums in 64 bits
    values = drawn_values(x8, xs)
    _, want = B.aeris_linear_bwd(values, tw, tdy, want_dx=False)
    assert torch.equal(dw, want)
    x, dy = to_f64(values[:, cols]), to_f64(tdy[:, feats])
    err = np.abs(to_f64(dw[feats][:, cols]) - dy.T @ x)
    assert (err <= max(1e-5, 4.0 * np.sqrt(n) * 2.0 ** -24) * (np.abs(dy).T @ np.abs(x))).all()
    # each alone and again: the same bits
    dx2, _ = B.aeris_linear_fp8_bwd(None, None, wt8, wts, tdy, want_dweight=False)
    _, dw2 = B.aeris_linear_fp8_bwd(x8, xs, None, None, tdy, want_dx=False)
    again = B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, tdy)
    assert same_bits(dx, dx2) and same_bits(dw, dw2) and same_bits((dx, dw), again)


@pytest.mark.parametrize("n,c,f,form", [
    (40, 1216, 192, (16, 8)), (1000, 64, 2048, (64, 1)), (200, 1344, 128, (64, 4)), (4100, 192, 1088, (128, 1)),
    (2500, 1600, 2112, (128, 1)), (1990, 1344, 1984, (128, 2)), (16310, 192, 832, (256, 1)), (8178, 320, 1920, (256, 1)),
    (8085, 576, 2048, (256, 1)), (24740, 512, 960, (256, 1))])
def test_linear_keeps_nan_to_itself_in_every_form(n, c, f, form):
    """Values that are not numbers at both ends of the channels, in rows and features where tiles end: their rows and
    features are, all others have the bits they have without them.  The largest scales of a row change no other."""
    assert (B.aeris_linear_fp8_plan(n, c, f)[0], B.aeris_linear_fp8_parts(n, c, f)) == form
    gen = torch.Generator(device="cuda").manual_seed(n + c)
    x8, xs = drawn_operand(gen, n, c)
    w8, ws = drawn_operand(gen, f, c)
    want = B.aeris_linear_fp8_fwd(x8, xs, w8, ws)
    assert torch.isfinite(want).all()
    raw = lambda t: t.view(torch.uint8)
    rows, feats, scaled = [(0, 0), (n // 2, c - 1), (n - 1, c // 2)], [(f // 3, 0), (f - 1, c - 1)], n // 4
    for row, channel in rows:
        raw(x8)[row, channel] = 0x7f
    for feature, channel in feats:
        raw(w8)[feature, channel] = 0xff
    raw(xs)[scaled, 0] = 227                              # 2^100
    y = B.aeris_linear_fp8_fwd(x8, xs, w8, ws)
    torch.cuda.synchronize()
    bad = torch.zeros(n, f, dtype=torch.bool, device="cuda")
    for row, _ in rows:
        bad[row] = True
    for feature, _ in feats:
        bad[:, feature] = True
    assert torch.equal(torch.isnan(y), bad)
    bad[scaled] = True
    assert torch.equal(y.view(torch.int16)[~bad], want.view(torch.int16)[~bad])


LARGE_GRADIENTS = [(20701, 448, 1472), (104617, 256, 832), (18569, 128, 2240), (2241, 2432, 1728)]


def gradient_operands(gen, n, c, f):
    x8, xs = drawn_operand(gen, n, c)
    w = torch.randn(f, c, device="cuda", generator=gen).bfloat16()
    w8, ws, wt8, wts = B.aeris_fp8_quantize(w, transposed=True)
    return [x8, xs, w8, ws, wt8, wts, torch.randn(n, f, device="cuda", generator=gen).bfloat16()]


@pytest.mark.parametrize("n,c,f", LARGE_GRADIENTS)
def test_linear_bwd_keeps_what_is_not_finite_to_itself(n, c, f):
    gen = torch.Generator(device="cuda").manual_seed(n)
    x8, xs, _, _, wt8, wts, dy = gradient_operands(gen, n, c, f)
    dx, dw = B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, dy)
    dy[n // 2, f - 1], dy[n - 1, 0] = float("inf"), float("nan")
    x8.view(torch.uint8)[n // 3, c - 1] = 0x7f
    dx2, dw2 = B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, dy)
    torch.cuda.synchronize()
    bad = torch.zeros(n, c, dtype=torch.bool, device="cuda")
    bad[n // 2], bad[n - 1] = True, True
    assert torch.equal(~torch.isfinite(dx2), bad) and torch.equal(dx[~bad], dx2[~bad])
    bad = torch.zeros(f, c, dtype=torch.bool, device="cuda")
    bad[f - 1], bad[0], bad[:, c - 1] = True, True, True
    assert torch.equal(~torch.isfinite(dw2), bad) and torch.equal(dw[~bad], dw2[~bad])


def test_captured_products_and_gradients_of_many_tiles():
    """The largest forms and both layouts of the gradients' workspace in one graph, replayed with new inputs in place."""
    gen = torch.Generator(device="cuda").manual_seed(71)

    def call(x8, xs, w8, ws, wt8, wts, dy):
        return (B.aeris_linear_fp8_fwd(x8, xs, w8, ws),) + B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, dy)
    held = [gradient_operands(gen, *size) for size in LARGE_GRADIENTS]
    assert {B.aeris_linear_fp8_plan(n, c, f)[0] for n, c, f in LARGE_GRADIENTS} == {128, 256}
    for v in held:
        call(*v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = [call(*v) for v in held]
    for _ in range(3):
        for v, size in zip(held, LARGE_GRADIENTS):
            for old, new in zip(v, gradient_operands(gen, *size)):
                old.view(torch.uint8).copy_(new.view(torch.uint8))
        want = [call(*v) for v in held]
        graph.replay()
        torch.cuda.synchronize()
        assert all(same_bits(a, b) for a, b in zip(outs, want))
        torch.randn(1000, 1000, device="cuda").sum().item()


# ------------------------------------------------------------------------------------- beyond 32 bits
def around(border, n):
    return np.unique(np.concatenate([[0, 1, 2 ** 31 // border, n - 257, n - 2, n - 1], np.arange(-2, 3) + 2 ** 32 // border]))


def test_offsets_beyond_32_bits():
    """Rows whose elements lie past 2^32 of each tensor: quantised, normalised, gated, multiplied, and their gradients."""
    n, c, f = 2 ** 21 + 70001, 2048, 64
    assert n * c > 2 ** 32 + 2 ** 27
    gen = torch.Generator(device="cuda").manual_seed(73)
    x = torch.empty(n, c, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    at = around(c, n)
    xf = to_f64(x[at])
    some = lambda q, scales, rows: codes(q[rows], scales.view(torch.uint8)[rows].view(torch.float8_e8m0fnu))

    def same(got, want):
        same_codes(got[0], want[0])
        assert (got[1] == want[1]).all()
    x8, xs, _, _ = B.aeris_fp8_quantize(x)
    same(some(x8, xs, at), fo.quantize(xf))
    # the norm without modulation
    one, zero = torch.ones(c, device="cuda"), torch.zeros(1, c, device="cuda")
    s, r, h8, hs = B.aeris_residual_norm_fp8_fwd(x, x, 1 + zero, one, zero, zero, 1e-6, n)
    sf = to_f64(s[at])
    assert (sf == 2 * xf).all()
    h = sf / np.sqrt((sf ** 2).mean(1) + 1e-6)[:, None]
    close_quantized("h", some(h8, hs, at), h, np.abs(h))
    del s, h8, hs
    # the gate of the rows as [u | v]
    g8, gs = B.aeris_swiglu_fp8_fwd(x[:n // 2 * 2].view(n // 2, 2 * c))
    half = around(2 * c, n // 2)
    uv = to_f64(x[:n // 2 * 2].view(n // 2, 2 * c)[half])
    g = bo.swiglu_fwd(uv)
    close_quantized("g", some(g8, gs, half), g, np.abs(g))
    del g8, gs
    # products: a large operand, a large result; gradients with a large dx
    w = torch.randn(f, c, device="cuda", generator=gen).bfloat16()
    w8, ws, wt8, wts = B.aeris_fp8_quantize(w, transposed=True)
    y = B.aeris_linear_fp8_fwd(x8, xs, w8, ws)
    close_product("y", y[at], fo.dequantize(*some(x8, xs, at)), fo.dequantize(*codes(w8, ws)))
    dx, dw = B.aeris_linear_fp8_bwd(x8, xs, wt8, wts, y)
    close_product("dx", dx[at], fo.round_trip(to_f64(y[at])), fo.dequantize(*codes(wt8, wts)))
    _, want = B.aeris_linear_bwd(drawn_values(x8, xs), w, y, want_dx=False)
    assert torch.equal(dw, want)


@pytest.mark.parametrize("c,f", [(2048, 320), (192, 2048)])
def test_largest_tiles_beyond_32_bits(c, f):
    """The 256 x 256 form on an operand and into a result of more than 2^32 elements."""
    n = 2 ** 21 + 70001
    assert n * max(c, f) > 2 ** 32 + 2 ** 27 and B.aeris_linear_fp8_plan(n, c, f)[0] == 256
    gen = torch.Generator(device="cuda").manual_seed(c)
    x8, xs, _, _ = B.aeris_fp8_quantize(torch.empty(n, c, dtype=torch.bfloat16, device="cuda").normal_(generator=gen))
    w8, ws = drawn_operand(gen, f, c)
    y = B.aeris_linear_fp8_fwd(x8, xs, w8, ws)
    torch.cuda.synchronize()
    at = around(max(c, f), n)
    x = fo.dequantize(*codes(x8[at], xs.view(torch.uint8)[at].view(torch.float8_e8m0fnu)))
    close_product("y", y[at], x, fo.dequantize(*codes(w8, ws)))


def test_transpose_of_the_most_rows_and_columns():
    """65,536 x 65,536: 2^32 elements, 512 blocks on either side."""
    n = 65536
    gen = torch.Generator(device="cuda").manual_seed(79)
    x = torch.empty(n, n, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    x8, xs, xt8, xts = B.aeris_fp8_quantize(x, transposed=True)
    torch.cuda.synchronize()
    at = np.array([0, 1, 127, 128, 32767, 32768, 65407, 65408, 65534, 65535])
    for (q, scales), part in (((x8, xs), x[at]), ((xt8, xts), x[:, at].t().contiguous())):
        got, want = codes(q[at], scales.view(torch.uint8)[at].view(torch.float8_e8m0fnu)), fo.quantize(to_f64(part))
        same_codes(got[0], want[0])
        assert (got[1] == want[1]).all()
