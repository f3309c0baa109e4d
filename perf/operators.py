"""The 8-bit path of a transformer layer's projections, as measured cases: rows and weights quantised
to e4m3 with a power-of-two scale per block of 128, the gated residual and RMSNorm with such an
output, the SwiGLU gate with such an output, the projection of such operands, and its gradients.

listed() are the fixed cases, draw() gives more of the same ranges; prepare() makes what a program holds
before the call, run() is one pass (of the plain form below, or where `own` is set through the
library's entry points), work() the bytes and operations it cannot do without, exact() the results in
64 bits.

The format: a block is 128 consecutive columns of one row (the last one of a row may be shorter). Its
scale is 2^e with the smallest integer e >= -126 for which the largest finite magnitude of the block is
at most 448 * 2^e; a value is held as x * 2^-e rounded to e4m3 (nearest even), a value that is not
finite as NaN. The scales of a row are padded with 1.0 to a multiple of four.
"""
import math

import torch

own = False

BLOCK, MOST, LEAST_EXPONENT = 128, 448.0, -126
EPS = 1e-6


# ------------------------------------------------------------------------------------- cases
def listed():
    cases = [
        # one layer's up-projection weights after a step of the optimiser: quantised for the forward
        # product and, transposed, for the gradient's
        ("quantize_weights", dict(kind="quantize", dtype="bf16", rows=11008, C=2048, transposed=True)),
        # the attention output of two coarse samples before the output projection; fp32 master copies
        # and odd sizes come in the drawn cases
        ("quantize_rows", dict(kind="quantize", dtype="bf16", rows=32400, C=1024, transposed=False)),
        # one 12 x 12 window of a small model: nothing but latency
        ("norm_window", dict(kind="norm", samples=1, rows=144, C=128, residual=True)),
        # channels that end inside a block, samples of odd length, first norm of a layer (no residual)
        ("norm_ragged", dict(kind="norm", samples=3, rows=5477, C=1600, residual=False)),
        # a latitude band of the 0.25-degree grid at the full width: memory traffic
        ("norm_band", dict(kind="norm", samples=1, rows=172800, C=2048, residual=True)),
        # the gate of a small model's layer, hidden width that ends inside a block
        ("swiglu_small", dict(kind="swiglu", rows=1728, H=576)),
        # the gate of the band at the full hidden width
        ("swiglu_band", dict(kind="swiglu", rows=172800, H=5504)),
        # the modulation values of one sample from its time embedding: a single row
        ("linear_one_row", dict(kind="linear", rows=1, C=2048, F=12288)),
        # a mid-sized model's QKV projection, rows that are no multiple of anything
        ("linear_ragged", dict(kind="linear", rows=20011, C=768, F=2304)),
        # the up-projection of the band
        ("linear_band", dict(kind="linear", rows=172800, C=2048, F=11008)),
        # gradients of the QKV projection above
        ("linear_bwd_ragged", dict(kind="linear_bwd", rows=20011, C=768, F=2304)),
        # gradients of the band's down-projection
        ("linear_bwd_band", dict(kind="linear_bwd", rows=172800, C=5504, F=2048)),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    kind = rng.choice(["quantize", "norm", "swiglu", "linear", "linear", "linear", "linear_bwd", "linear_bwd"])
    if kind == "quantize":
        transposed = rng.random() < 0.6
        C = 64 * _log(rng, 1, 86)
        rows = 64 * _log(rng, 1, 172) if transposed else _log(rng, 1, 100000)
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), rows=rows, C=C, transposed=transposed)
    if kind == "norm":
        samples = rng.randint(1, 4)
        return dict(kind=kind, samples=samples, rows=max(1, _log(rng, 1, 172800) // samples),
                    C=64 * _log(rng, 1, 32), residual=rng.random() < 0.7)
    if kind == "swiglu":
        return dict(kind=kind, rows=_log(rng, 1, 172800), H=64 * _log(rng, 1, 86))
    C, F = 64 * _log(rng, 1, 86), 64 * _log(rng, 1, 172)
    most = 172800 * 2048 * 11008 // (2 if kind == "linear_bwd" else 1)
    return dict(kind=kind, rows=min(_log(rng, 1, 172800), most // (C * F)), C=C, F=F)


# ------------------------------------------------------------------------------------- preparation
class _Inputs:
    """Device tensors drawn from one generator."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

    def f32(self, *shape, scale=1.0, mean=0.0):
        return mean + scale * torch.randn(*shape, device="cuda", generator=self.gen)

    def rows(self, n, c, scale=1.0):
        """Activations: normal, with channels of unlike size as a trained layer has them."""
        gain = torch.exp(0.7 * torch.randn(c, device="cuda", generator=self.gen)) * scale
        out = torch.empty(n, c, dtype=torch.bfloat16, device="cuda")
        step = max(1, (1 << 28) // c)
        for i in range(0, n, step):
            part = torch.randn(min(step, n - i), c, dtype=torch.bfloat16, device="cuda", generator=self.gen)
            out[i:i + step] = part * gain.bfloat16()
        return out


def prepare(case, seed):
    s = dict(case=case)
    inp = _Inputs(seed)
    kind = case["kind"]
    if kind == "quantize":
        s["x"] = inp.rows(case["rows"], case["C"])
        if case["dtype"] == "f32":
            s["x"] = s["x"].float() * (1.0 + 1e-3 * torch.rand(case["C"], device="cuda", generator=inp.gen))
    elif kind == "norm":
        n, C = case["samples"] * case["rows"], case["C"]
        s["x"] = inp.rows(n, C)
        s["w"] = inp.f32(C, scale=0.1, mean=1.0)
        s["gamma"], s["beta"] = inp.f32(case["samples"], C, scale=0.3), inp.f32(case["samples"], C, scale=0.5)
        s["y"] = inp.rows(n, C, scale=0.5) if case["residual"] else None
        s["alpha"] = inp.f32(case["samples"], C, scale=0.8) if case["residual"] else None
    elif kind == "swiglu":
        s["uv"] = inp.rows(case["rows"], 2 * case["H"])
    else:
        n, C, F = case["rows"], case["C"], case["F"]
        weight = inp.f32(F, C, scale=C ** -0.5).bfloat16()
        s["x8"], s["xs"] = _quantized(inp.rows(n, C))
        if kind == "linear":
            s["w8"], s["ws"] = _quantized(weight)
        else:
            s["wt8"], s["wts"] = _quantized(weight.t().contiguous())
            s["dy"] = inp.rows(n, F, scale=1e-3)
    return s


# ------------------------------------------------------------------------------------- plain form
def _power(e, dtype):
    """2^e from whole exponents of normal numbers, by their bits: exp2 and pow need not be exact."""
    if dtype == torch.float64:
        return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _blocks(x):
    """[n, c] -> [n, blocks, 128], the last block filled up with zeros."""
    n, c = x.shape
    more = -c % BLOCK
    if more:
        x = torch.nn.functional.pad(x, (0, more))
    return x.view(n, -1, BLOCK)


def _quantized(x):
    """(values as float8_e4m3fn [n, c], scales as float8_e8m0fnu [n, padded blocks]) of rows in 32 or 64 bits
    or bf16."""
    n, c = x.shape
    v = _blocks(x if x.dtype == torch.float64 else x.float())
    size = v.abs()
    size = torch.where(torch.isfinite(size), size, torch.zeros_like(size)).amax(-1)
    m, k = torch.frexp(size)                              # size = m 2^k, 1/2 <= m < 1; 448 = 7/8 2^9
    e = torch.where(m <= 0.875, k - 9, k - 8).clamp(min=LEAST_EXPONENT)
    e = torch.where(size == 0, torch.full_like(e, LEAST_EXPONENT), e)
    q = v * _power(-e, v.dtype)[..., None]
    q = torch.where(torch.isfinite(q), q, torch.full_like(q, float("nan"))).to(torch.float8_e4m3fn)
    scales = torch.full((n, -(-e.shape[1] // 4) * 4), 127, dtype=torch.uint8, device=x.device)
    scales[:, :e.shape[1]] = (e + 127).to(torch.uint8)
    return q.view(n, -1)[:, :c].contiguous(), scales.view(torch.float8_e8m0fnu)


def _values(x8, scales):
    """What quantised rows stand for, in 32 bits."""
    n, c = x8.shape
    v = _blocks(x8.float())
    scale = _power(scales.view(torch.uint8)[:, :v.shape[1]].to(torch.int32) - 127, torch.float32)
    return (v * scale[..., None]).view(n, -1)[:, :c]


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "quantize":
        out = dict(zip(("x8", "xs"), _quantized(s["x"])))
        if case["transposed"]:
            out.update(zip(("xt8", "xts"), _quantized(s["x"].t().contiguous())))
        return out
    if kind == "norm":
        # in 64 bits: results lie next to the borders of the 8-bit rounding
        x, rows = s["x"].double(), case["rows"]
        out = {}
        if case["residual"]:
            gated = torch.repeat_interleave(s["alpha"].double(), rows, 0) * s["y"].double()
            out["s"] = (x + gated).bfloat16()
            x = out["s"].double()
        r = (x.square().mean(-1) + EPS).rsqrt()
        gain = s["w"].double() * (1.0 + s["gamma"].double())
        h = x * r[:, None] * torch.repeat_interleave(gain, rows, 0)
        h = h + torch.repeat_interleave(s["beta"].double(), rows, 0)
        out["r"] = r.float()
        out.update(zip(("h8", "hs"), _quantized(h)))
        return out
    if kind == "swiglu":
        u, v = s["uv"][:, :case["H"]].double(), s["uv"][:, case["H"]:].double()
        return dict(zip(("g8", "gs"), _quantized(u / (1.0 + torch.exp(-u)) * v)))
    if kind == "linear":
        return dict(y=(_values(s["x8"], s["xs"]) @ _values(s["w8"], s["ws"]).t()).bfloat16())
    dx = _values(*_quantized(s["dy"])) @ _values(s["wt8"], s["wts"]).t()
    return dict(dx=dx.bfloat16(), dweight=s["dy"].float().t() @ _values(s["x8"], s["xs"]))


# ------------------------------------------------------------------------------------- one pass
def run(s):
    if not own:
        return _plain(s)
    from paper_2509_13523_amd import binding as B
    case = s["case"]
    kind = case["kind"]
    if kind == "quantize":
        x8, xs, xt8, xts = B.aeris_fp8_quantize(s["x"], transposed=case["transposed"])
        return dict(x8=x8, xs=xs, xt8=xt8, xts=xts) if case["transposed"] else dict(x8=x8, xs=xs)
    if kind == "norm":
        ss, r, h8, hs = B.aeris_residual_norm_fp8_fwd(s["x"], s["y"], s["alpha"], s["w"], s["gamma"], s["beta"],
                                                      EPS, case["rows"])
        return dict(s=ss, r=r, h8=h8, hs=hs) if case["residual"] else dict(r=r, h8=h8, hs=hs)
    if kind == "swiglu":
        return dict(zip(("g8", "gs"), B.aeris_swiglu_fp8_fwd(s["uv"])))
    if kind == "linear":
        return dict(y=B.aeris_linear_fp8_fwd(s["x8"], s["xs"], s["w8"], s["ws"]))
    dx, dweight = B.aeris_linear_fp8_bwd(s["x8"], s["xs"], s["wt8"], s["wts"], s["dy"])
    return dict(dx=dx, dweight=dweight)


# ------------------------------------------------------------------------------------- accounting
def work(case):
    kind = case["kind"]
    scales = lambda n, c: n * (-(-c // BLOCK))
    if kind == "quantize":
        n, C = case["rows"], case["C"]
        each = (4 if case["dtype"] == "f32" else 2) * n * C
        return dict(bytes=each + n * C + scales(n, C) + (n * C + scales(C, n) if case["transposed"] else 0),
                    flops=2 * n * C)
    if kind == "norm":
        n, C = case["samples"] * case["rows"], case["C"]
        return dict(bytes=(3 + 4 * case["residual"]) * n * C + scales(n, C) + 4 * n +
                    4 * C * (1 + (2 + case["residual"]) * case["samples"]), flops=8 * n * C)
    if kind == "swiglu":
        return dict(bytes=5 * case["rows"] * case["H"] + scales(case["rows"], case["H"]),
                    flops=6 * case["rows"] * case["H"])
    n, C, F = case["rows"], case["C"], case["F"]
    if kind == "linear":
        return dict(bytes=n * C + scales(n, C) + F * C + scales(F, C) + 2 * n * F, flops=2.0 * n * C * F)
    return dict(bytes=2 * n * F + n * C + scales(n, C) + C * F + scales(C, F) + 2 * n * C + 4 * C * F,
                flops=4.0 * n * C * F)


# ------------------------------------------------------------------------------------- in 64 bits
def _exact_exponent(size):
    """floor(log2(size)) of normal numbers in 64 bits, from their bits."""
    return ((size.view(torch.int64) >> 52) & 2047) - 1023


def _exact_scaled(x):
    """(values over their block's scale, not rounded, and the exponents of the scales) of rows in 64 bits."""
    n, c = x.shape
    count = -(-c // BLOCK)
    e = torch.empty(n, count, dtype=torch.int64, device=x.device)
    q = torch.empty_like(x)
    for b in range(count):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        most = part.abs().nan_to_num(nan=0.0, posinf=0.0).amax(1)
        at = _exact_exponent(most) - 8                      # most < 512 2^at
        over = most > MOST * _power(at, torch.float64)
        e[:, b] = torch.where(most > 0, at + over, LEAST_EXPONENT).clamp(min=LEAST_EXPONENT)
        q[:, b * BLOCK:(b + 1) * BLOCK] = part * _power(-e[:, b:b + 1], torch.float64)
    return q, e


def _exact_values(q, e):
    """q 2^e by blocks."""
    return q * torch.repeat_interleave(_power(e, torch.float64), BLOCK, 1)[:, :q.shape[1]]


def _exact_e4m3(q):
    """q rounded to e4m3: three bits behind the leading one, steps of 2^-9 at the least."""
    step = _power(_exact_exponent(q.abs().clamp(min=2.0 ** -6)) - 3, torch.float64)
    return torch.round(q / step) * step


def _held(x8, scales):
    return _exact_values(x8.double(), scales.view(torch.uint8).to(torch.int64) - 127)


def exact(case, seed):
    """8-bit results: the values over their scale before the rounding. A scale is a choice and has none."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        out = dict(x8=_exact_scaled(s["x"].double())[0], xs=None)
        if case["transposed"]:
            out.update(xt8=_exact_scaled(s["x"].double().t().contiguous())[0], xts=None)
        return out
    if kind == "norm":
        outs = []
        for b in range(case["samples"]):
            at = slice(b * case["rows"], (b + 1) * case["rows"])
            total = s["x"][at].double()
            part = {}
            if case["residual"]:
                part["s"] = total + s["alpha"][b].double() * s["y"][at].double()
                total = part["s"].bfloat16().double()
            part["r"] = 1.0 / torch.sqrt((total * total).sum(1) / case["C"] + EPS)
            h = total * part["r"][:, None] * s["w"].double()
            part["h8"] = _exact_scaled(h + h * s["gamma"][b].double() + s["beta"][b].double())[0]
            outs.append(part)
        return dict({k: torch.cat([p[k] for p in outs]) for k in outs[0]}, hs=None)
    if kind == "swiglu":
        uv = s["uv"].double()
        u, v = uv.chunk(2, 1)
        return dict(g8=_exact_scaled(u * torch.sigmoid(u) * v)[0], gs=None)
    x = _held(s["x8"], s["xs"])
    if kind == "linear":
        return dict(y=x @ _held(s["w8"], s["ws"]).t())
    dy = s["dy"].double()
    q, e = _exact_scaled(dy)
    return dict(dx=_exact_values(_exact_e4m3(q), e) @ _held(s["wt8"], s["wts"]).t(), dweight=dy.t() @ x)
