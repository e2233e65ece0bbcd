"""Tensors of more than 2^32 bytes: the rows at the far end, through every operator around the projections."""
import numpy as np
import pytest
import torch

from oracle import projection_oracle as po
from paper_2605_11354_amd import binding as B
from tests import gpu_util as G

pytestmark = pytest.mark.gpu
f64 = G.bf16_tensor_to_f64
bits = lambda t: t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def noise(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)


def test_heads():
    """6 000 000 tokens of 2 heads.  Tolerances as for 32 tokens: a row knows nothing of the others."""
    N, H, tail = 6_000_000, 2, 200
    qkv = noise((1, N, 3, H, 64), 1)
    q, k, v = qkv.unbind(2)
    p = B.make_heads_params(q, norm="layer", axes=1, base=1e4, layout="bhnd")
    pos = torch.arange(N, dtype=torch.int32, device="cuda").view(N, 1)
    w = 1 + 0.1 * torch.arange(64, device="cuda") / 64
    out = [torch.empty((1, H, N, 64), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    B.sla_qk_norm_rope(p, q, k, v, *out, pos=pos, q_weight=w)
    x, ps, wn = f64(q[:, -tail:]), pos[-tail:].view(1, tail, 1).cpu().numpy(), w.double().cpu().numpy()
    y = po.heads_forward(x, "layer", wn, None, 1e-5, 1, "halves", 1e4, ps)
    off = 64 * 2.0 ** -24 * 2 * np.abs(x).max(-1, keepdims=True) * 4
    assert (np.abs(f64(out[0][:, :, -tail:]).transpose(0, 2, 1, 3) - y) <= 2.0 ** -8 * np.abs(y) + off).all()
    assert torch.equal(out[2][0, -1, -tail:].view(torch.int16), v[0, -tail:, -1].contiguous().view(torch.int16))
    d = torch.empty_like(qkv)
    dq, dk, dv = d.unbind(2)
    B.sla_qk_norm_rope_grad(p, q, k, *out, dq, dk, dv, pos=pos, q_weight=w)
    gy = f64(out[0][:, :, -tail:]).transpose(0, 2, 1, 3)
    ref = po.heads_backward(x, "layer", wn, 1e-5, 1, "halves", 1e4, ps, gy)[0]
    # two sums more than the forward over products with |u| <= 8, r about 1
    assert (np.abs(f64(dq[:, -tail:]) - ref) <= 2.0 ** -8 * np.abs(ref) + 512 * 2.0 ** -24 * 2 * np.abs(gy).max(-1, keepdims=True) * 8).all()
    assert torch.equal(dv[0, -tail:, -1].contiguous().view(torch.int16), out[2][0, -1, -tail:].view(torch.int16))
    del out, d, dq, dk, dv
    codes = [torch.empty((1, H, N, 64), dtype=torch.uint8, device="cuda") for _ in range(3)]
    scales = [torch.empty((1, H, -(-N // b)), device="cuda") for b in (128, 64, 64)]
    B.sla_qk_norm_rope_e4m3(p, q, k, v, 128, *codes, *scales, pos=pos, q_weight=w)
    s = np.repeat(scales[0].double().cpu().numpy()[:, :, -3:].transpose(0, 2, 1), 128, 1)[:, :, :, None]
    last = N - (scales[0].shape[2] - 3) * 128
    s = s[:, last - tail:last]
    got = codes[0][:, :, -tail:].view(torch.float8_e4m3fn).float().cpu().numpy().astype(np.float64).transpose(0, 2, 1, 3) * s
    assert (np.abs(got - y) <= 2.0 ** -4 * np.abs(y) + 2.0 ** -10 * s + off).all()


def test_fp8_layer():
    N, d_in, d_out, tail = 1_050_003, 2048, 8, 100
    x, W, dy = noise((N, d_in), 2), noise((d_out, d_in), 3), noise((N, d_out), 4)
    y, ck = torch.empty((N, d_out), dtype=torch.bfloat16, device="cuda"), torch.empty(B.sla_fp8_checkpoint_bytes(N, d_in), dtype=torch.uint8, device="cuda")
    B.sla_fp8_linear_save(x, W, None, y, ck)
    xt, Wb, g = bits(x[-tail:]), bits(W), f64(dy[-tail:])
    (xc, xs), (wc, ws) = po.e4m3_rows(xt), po.e4m3_rows(Wb)
    xq, wq = xc * xs[:, None], wc * ws[:, None]
    ref = xq @ wq.T
    assert (np.abs(f64(y[-tail:]) - ref) <= 2.0 ** -8 * np.abs(ref) + (d_in + 4) * 2.0 ** -24 * (np.abs(xq) @ np.abs(wq).T)).all()
    dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty(d_out, dtype=torch.bfloat16, device="cuda")
    B.sla_fp8_linear_grad(dy, ck, W, dx, dW, db)
    ref, mag = g @ wq, np.abs(g) @ np.abs(wq)
    assert (np.abs(f64(dx[-tail:]) - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + (d_out + 20) * 2.0 ** -24) * mag).all()
    B.sla_fp8_checkpoint_restore(ck, x)
    assert (np.abs(f64(x[-tail:]) - xq) <= 2.0 ** -8 * np.abs(xq) * (1 + 2.0 ** -15)).all()
    ref = torch.zeros((d_out, d_in), dtype=torch.float64, device="cuda")
    for i in range(0, N, 100_000):
        ref += dy[i:i + 100_000].double().T @ x[i:i + 100_000].double()
    # the products are of the same rounded numbers: partial sums in fp32 (relative 2^-24 each, of random sign) and the store
    assert float(torch.linalg.norm(dW.double() - ref)) <= 2.0 ** -8 * float(torch.linalg.norm(ref))
    ref = dy.double().sum(0)
    assert bool(((db.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (N + 20) * 2.0 ** -24 * dy.double().abs().sum(0)).all())


def test_four_bits():
    N, d_in, d_out, tail = 1_050_003, 2048, 8, 100
    x, W = noise((N, d_in), 5), noise((d_out, d_in), 6)
    c, s = torch.empty((N, d_in // 2), dtype=torch.uint8, device="cuda"), torch.empty((N, d_in // 32), dtype=torch.uint8, device="cuda")
    B.sla_quantise_mxfp4(x, c, s)
    want = po.mxfp4_quantise(bits(x[-tail:]))
    assert (c[-tail:].cpu().numpy() == po.mxfp4_pack(want[0])).all() and (s[-tail:].cpu().numpy() == want[1]).all()
    back = torch.empty_like(x)
    B.sla_dequantise_mxfp4(c, s, back)
    xq = po.mxfp4_values(*want)
    assert (f64(back[-tail:]) == xq).all()
    Wc, Ws = torch.empty((d_out, d_in // 2), dtype=torch.uint8, device="cuda"), torch.empty((d_out, d_in // 32), dtype=torch.uint8, device="cuda")
    B.sla_quantise_mxfp4(W, Wc, Ws)
    y = torch.empty((N, d_out), dtype=torch.bfloat16, device="cuda")
    B.sla_mxfp4_linear(x, Wc, Ws, None, y)
    wq = po.mxfp4_values(*po.mxfp4_quantise(bits(W)))
    ref = xq @ wq.T
    assert (np.abs(f64(y[-tail:]) - ref) <= 2.0 ** -8 * np.abs(ref) + (d_in + 2) * 2.0 ** -24 * (np.abs(xq) @ np.abs(wq).T)).all()
