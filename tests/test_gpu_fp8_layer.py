"""The attention half of a transformer layer with 8-bit projections, forward and backward, as a training step runs it:

    s, h8 = x + alpha y, Q(RMSNorm(s; w) (1 + gamma) + beta)     aeris_residual_norm_fp8_fwd
    qkv   = h8 Wqkv8^T                                            aeris_linear_fp8_fwd, packed
    a     = window attention(rope(q), rope(k), v)                 aeris_winattn_rope_fwd on the packed qkv
    a8    = Q(a)                                                  aeris_fp8_quantize
    out   = a8 Wo8^T                                              aeris_linear_fp8_fwd

Each stage is held, from the operands that the stage before it left, to the bounds of its own tests (test_gpu_fp8.py,
test_gpu_layer_composition.py)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from oracle import fp8_oracle as fo
from oracle import rope_oracle as ro
from paper_2509_13523_amd import binding as B
from test_gpu_fp8 import bf16, close_product, close_quantized, codes, f32, rows_with_gain, same_codes, to_f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("samples,H,W,heads,d", [(2, 24, 36, 2, 64), (1, 12, 24, 6, 32)])
def test_attention_half_of_a_layer_in_8_bits(samples, H, W, heads, d):
    C, rows = heads * d, H * W
    n, eps, win, shift, mask, base = samples * rows, 1e-6, (12, 12), (6, 6), B.AERIS_MASK_SWIN, 100.0
    rng = np.random.default_rng(C + rows)
    (tx, x), (ty, y), (tdout, dout), (tds, ds) = [bf16(rows_with_gain(rng, n, C)) for _ in range(4)]
    (twqkv, _), (two, _) = [bf16(rng.standard_normal((f, C)) / np.sqrt(C)) for f in (3 * C, C)]
    (tw, w), (ta, _), (tg, g), (tb, b) = [f32(v) for v in (
        1 + 0.1 * rng.standard_normal(C), 0.8 * rng.standard_normal((samples, C)),
        0.3 * rng.standard_normal((samples, C)), 0.5 * rng.standard_normal((samples, C)))]
    wqkv8, wqkvs, wqkvt8, wqkvts = B.aeris_fp8_quantize(twqkv, transposed=True)
    wo8, wos, wot8, wots = B.aeris_fp8_quantize(two, transposed=True)

    # forward
    s, r, h8, hs = B.aeris_residual_norm_fp8_fwd(tx, ty, ta, tw, tg, tb, eps, rows)
    qkv = B.aeris_linear_fp8_fwd(h8, hs, wqkv8, wqkvs)                   # [n, 3C] = [B, H, W, 3, heads, d]
    p = B.make_params((samples, H, W, heads, d), win, shift, mask, qkv_strides=(3 * C, d))
    rope = B.aeris_rope_params(base, B.AERIS_ROPE_POS_WINDOW)
    lib, stream = B.load(), torch.cuda.current_stream().cuda_stream
    parts = lambda t: [t.data_ptr() + i * C * 2 for i in range(3)]
    attn = torch.empty(n, C, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(samples, heads, H, W, dtype=torch.float32, device="cuda")
    rotated = torch.empty(B.aeris_winattn_rope_fwd_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    space = torch.empty(B.aeris_winattn_bwd_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    assert lib.aeris_winattn_rope_fwd(ctypes.byref(p), ctypes.byref(rope), *parts(qkv), attn.data_ptr(), lse.data_ptr(),
                                      rotated.data_ptr(), rotated.numel(), stream) == 0
    a8, a_s, _, _ = B.aeris_fp8_quantize(attn)
    out = B.aeris_linear_fp8_fwd(a8, a_s, wo8, wos)
    # backward
    da, dwo = B.aeris_linear_fp8_bwd(a8, a_s, wot8, wots, tdout)
    dqkv = torch.empty_like(qkv)
    assert lib.aeris_winattn_rope_bwd(ctypes.byref(p), ctypes.byref(rope), *parts(qkv), attn.data_ptr(), lse.data_ptr(),
                                      da.data_ptr(), *parts(dqkv), rotated.data_ptr(), space.data_ptr(), space.numel(),
                                      stream) == 0
    dh, dwqkv = B.aeris_linear_fp8_bwd(h8, hs, wqkvt8, wqkvts, dqkv)
    dx, dw, dgamma, dbeta = B.aeris_rmsnorm_adaln_bwd(s, tw, tg, r, dh, rows, dres=tds)
    torch.cuda.synchronize()

    held = lambda q, scales: fo.dequantize(*codes(q, scales))
    h, _ = bo.rmsnorm_adaln_fwd(to_f64(s), w, g, b, eps, rows)
    close_quantized("h", codes(h8, hs), h, np.abs(h) + 2 * np.abs(np.repeat(b, rows, 0)))
    close_product("qkv", qkv, held(h8, hs), held(wqkv8, wqkvs))
    split = to_f64(qkv).reshape(samples, H, W, 3, heads, d)
    q, k, v = split[:, :, :, 0], split[:, :, :, 1], split[:, :, :, 2]
    rel = lambda got, want: np.linalg.norm(got - want) / np.linalg.norm(want)
    o, _ = ro.winattn_rope_fwd(q, k, v, win, shift, mask, base, ro.POS_WINDOW)
    assert rel(to_f64(attn), o.reshape(n, C)) <= 5e-3
    got, want = codes(a8, a_s), fo.quantize(to_f64(attn))
    same_codes(got[0], want[0])
    assert (got[1] == want[1]).all()
    close_product("out", out, held(a8, a_s), held(wo8, wos))
    close_product("da", da, fo.round_trip(dout), held(wot8, wots))
    grads = ro.winattn_rope_bwd(q, k, v, to_f64(da).reshape(samples, H, W, heads, d), win, shift, mask, base, ro.POS_WINDOW)
    assert rel(to_f64(dqkv), np.stack(grads, axis=3).reshape(n, 3 * C)) <= 8e-3
    close_product("dh", dh, fo.round_trip(to_f64(dqkv)), held(wqkvt8, wqkvts))
    for dweight, dy, x_of in ((dwo, dout, held(a8, a_s)), (dwqkv, to_f64(dqkv), held(h8, hs))):
        assert (np.abs(to_f64(dweight) - dy.T @ x_of) <= 1e-5 * np.abs(dy).T @ np.abs(x_of)).all()
    ref = bo.rmsnorm_adaln_bwd_residual(to_f64(s), w, g, b, eps, rows, to_f64(dh), ds)
    for got, want in zip((dx, dw, dgamma, dbeta), ref):
        assert rel(to_f64(got), want.reshape(got.shape)) <= 2e-3
