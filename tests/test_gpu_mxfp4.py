"""Microscaled 4-bit numbers and the linear layer on them, against the fp64 reference.

The quantiser and its inverse are defined bit for bit.  Products of two E2M1 numbers times two powers of two are exact; a sum of K of
them in fp32 is off by at most K 2^-24 of the sum of magnitudes (any order), the bias adds one rounding, the store half a bf16 step."""
import numpy as np
import pytest
import torch

from oracle import projection_oracle as po
from paper_2605_11354_amd import binding as B
from paper_2605_11354_amd import synth
from tests import gpu_util as G

pytestmark = pytest.mark.gpu
f64 = G.bf16_tensor_to_f64


def quantise(x):
    rows, cols = x.shape
    c, s = torch.full((rows, cols // 2), 0x77, dtype=torch.uint8, device="cuda"), torch.full((rows, cols // 32), 0x33, dtype=torch.uint8, device="cuda")
    B.sla_quantise_mxfp4(x, c, s)
    return c, s


def test_every_bf16_number_at_every_scale_it_can_have():
    """Row r holds all 32768 magnitudes behind one block maximum each; signs alternate."""
    mags = np.arange(0x7F80, dtype=np.uint16)
    tops = np.concatenate([np.arange(0, 0x180, 0x20), np.arange(0x180, 0x7F80, 0x80) + 0x55, [0x7F7F]]).astype(np.uint16)
    # values within 2^6 below the maximum meet every rounding; further down everything is 0 or a half
    rows = [np.minimum(np.where(np.arange(len(m)) % 31 == 0, t, m), t) for t in tops for m in (mags[max(0, int(t) - 0x380): int(t) + 1],)]
    rows = [np.concatenate([[t], np.resize(r, 1023)]).astype(np.uint16) for r, t in zip(rows, tops)]
    bits = np.stack(rows)
    bits[:, 1::2] |= 0x8000
    c, s = quantise(G.dev_bf16(bits))
    y = torch.empty(bits.shape, dtype=torch.bfloat16, device="cuda")
    B.sla_dequantise_mxfp4(c, s, y)
    torch.cuda.synchronize()
    wc, ws = po.mxfp4_quantise(bits)
    assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(c.cpu().numpy(), po.mxfp4_pack(wc))
    assert np.array_equal(f64(y), po.mxfp4_values(wc, ws))


def test_infinities_nan_and_zeros():
    bits = synth.to_bf16_bits(np.random.default_rng(0).standard_normal((3, 96)).astype(np.float32))
    bits[0, 5], bits[1, 64], bits[1, 0], bits[2, 32:64] = 0x7F80, 0xFFC1, 0x7F7F, 0x8000
    c, s = quantise(G.dev_bf16(bits))
    y = torch.empty((3, 96), dtype=torch.bfloat16, device="cuda")
    B.sla_dequantise_mxfp4(c, s, y)
    torch.cuda.synchronize()
    wc, ws = po.mxfp4_quantise(bits)
    assert ws[0, 0] == 255 and ws[1, 2] == 255 and ws[2, 1] == 0
    assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(c.cpu().numpy(), po.mxfp4_pack(wc))
    assert np.array_equal(f64(y), po.mxfp4_values(wc, ws), equal_nan=True)


def test_every_code_at_every_scale_comes_back():
    codes = np.tile(np.arange(16), 512).reshape(256, 32)
    scales = np.arange(256).reshape(256, 1)
    y = torch.empty((256, 32), dtype=torch.bfloat16, device="cuda")
    B.sla_dequantise_mxfp4(torch.from_numpy(po.mxfp4_pack(codes)).cuda(), torch.from_numpy(scales.astype(np.uint8)).cuda(), y)
    torch.cuda.synchronize()
    want = po.mxfp4_values(codes, scales)
    with np.errstate(invalid="ignore"):
        want = np.where(np.abs(want) > 3.39e38, np.sign(want) * np.inf, want)           # beyond bf16
    assert np.array_equal(f64(y), want, equal_nan=True)


def layer(N, d_in, d_out, seed=0):
    g = np.random.default_rng(seed)
    x = synth.to_bf16_bits((g.standard_normal((N, d_in)) * np.exp(g.uniform(-3, 3, (N, 1)))).astype(np.float32))
    W = synth.to_bf16_bits((g.standard_normal((d_out, d_in)) / np.sqrt(d_in) * np.exp(g.uniform(-3, 3, (d_out, 1)))).astype(np.float32))
    return x, W, synth.to_bf16_bits(g.standard_normal(d_out).astype(np.float32))


SIZES = [(1, 128, 8), (1, 4096, 520), (2, 256, 4096), (4, 640, 40), (5, 384, 264), (8, 1024, 24), (9, 128, 520), (15, 384, 136), (16, 1152, 16), (17, 128, 8200), (32, 2048, 264), (33, 128, 8), (64, 256, 72), (33, 512, 264), (48, 1024, 72), (49, 640, 520), (64, 2048, 4096), (60, 1024, 4104),
         (65, 384, 136), (197, 640, 1160), (1000, 128, 64), (2049, 256, 3080), (6500, 128, 1024), (8195, 384, 2056), (4100, 256, 4360)]


@pytest.mark.parametrize("N,d_in,d_out", SIZES)
@pytest.mark.parametrize("bias", [True, False])
def test_linear(N, d_in, d_out, bias):
    xb, Wb, bb = layer(N, d_in, d_out, N + d_out)
    Wc, Ws = quantise(G.dev_bf16(Wb))
    y = torch.full((N + 1, d_out), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.full((B.sla_mxfp4_linear_workspace_bytes(N, d_in, d_out) + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    call = lambda: B.sla_mxfp4_linear(G.dev_bf16(xb), Wc, Ws, G.dev_bf16(bb) if bias else None, y[:N], ws[:-256])
    call()
    torch.cuda.synchronize()
    first = y.clone()
    assert torch.isnan(y[N]).all() and bool((ws[-256:] == 0x5A).all())
    xq, wq = po.mxfp4_values(*po.mxfp4_quantise(xb)), po.mxfp4_values(*po.mxfp4_quantise(Wb))
    b = po.bf16_to_f64(bb) if bias else 0.0
    ref, mag = xq @ wq.T + b, np.abs(xq) @ np.abs(wq).T
    d = np.abs(f64(y[:N]) - ref)
    assert (d <= 2.0 ** -8 * np.abs(ref) + (d_in + 2) * 2.0 ** -24 * (mag + np.abs(b))).all(), d.max()
    call()
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), y.view(torch.int16))


@pytest.mark.parametrize("N", [7, 300])
def test_tokens_and_channels_that_are_not_finite_stay_by_themselves(N):
    xb, Wb, _ = layer(N, 256, 40)
    xb[3, 200], xb[5, 0] = 0x7F80, 0x7FC0
    Wb[9, 31] = 0xFF80
    Wc, Ws = quantise(G.dev_bf16(Wb))
    y = torch.empty((N, 40), dtype=torch.bfloat16, device="cuda")
    B.sla_mxfp4_linear(G.dev_bf16(xb), Wc, Ws, None, y)
    torch.cuda.synchronize()
    got, lost = f64(y), np.zeros((N, 40), bool)
    lost[[3, 5]], lost[:, 9] = True, True
    assert np.isnan(got[lost]).all()
    with np.errstate(invalid="ignore"):
        xq, wq = po.mxfp4_values(*po.mxfp4_quantise(xb)), po.mxfp4_values(*po.mxfp4_quantise(Wb))
        ref, mag = xq @ wq.T, np.abs(xq) @ np.abs(wq).T
    assert (np.abs(got - ref)[~lost] <= (2.0 ** -8 * np.abs(ref) + 258 * 2.0 ** -24 * mag)[~lost]).all()


@pytest.mark.parametrize("size_x,size_W", [(1e37, 1e-6), (1e-37, 1e30), (1e-39, 1.0)])
@pytest.mark.parametrize("N", [5, 70])
def test_operands_far_from_one(size_x, size_W, N):
    g = np.random.default_rng(1)
    bits = lambda a: (np.ascontiguousarray(a, np.float32).view(np.uint32) >> 16).astype(np.uint16)       # (truncated: nothing flushed)
    xb, Wb = bits(g.standard_normal((N, 128)) * size_x), bits(g.standard_normal((16, 128)) * size_W)
    Wc, Ws = quantise(G.dev_bf16(Wb))
    y = torch.empty((N, 16), dtype=torch.bfloat16, device="cuda")
    B.sla_mxfp4_linear(G.dev_bf16(xb), Wc, Ws, None, y)
    torch.cuda.synchronize()
    xq, wq = po.mxfp4_values(*po.mxfp4_quantise(xb)), po.mxfp4_values(*po.mxfp4_quantise(Wb))
    ref, mag = xq @ wq.T, np.abs(xq) @ np.abs(wq).T
    assert (np.abs(f64(y) - ref) <= 2.0 ** -8 * np.abs(ref) + 130 * 2.0 ** -24 * mag + 2.0 ** -126).all()       # results below the normal range may go to zero


def test_replays_from_a_graph():
    xb, Wb, bb = layer(100, 256, 72)
    x, W, b = map(G.dev_bf16, (xb, Wb, bb))
    Wc, Ws = quantise(W)
    y, z = torch.empty((100, 72), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 72), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.sla_mxfp4_linear_workspace_bytes(100, 256, 72), dtype=torch.uint8, device="cuda")

    def work():
        B.sla_quantise_mxfp4(W, Wc, Ws)
        B.sla_mxfp4_linear(x, Wc, Ws, b, y, ws)
        B.sla_mxfp4_linear(x[:3], Wc, Ws, b, z)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for k in range(3):
        x.mul_(1.5), W.add_(0.01)
        work()
        torch.cuda.synchronize()
        want = y.clone(), z.clone()
        y.zero_(), z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want[0].view(torch.int16), y.view(torch.int16)) and torch.equal(want[1].view(torch.int16), z.view(torch.int16)), k


def test_tensors_of_another_shape_type_or_place_are_refused():
    x, c, s = torch.empty((4, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((8, 64), dtype=torch.uint8, device="cuda"), torch.empty((8, 4), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="codes"):
        B.sla_quantise_mxfp4(x, c, s)
    with pytest.raises(ValueError, match="W_scales"):
        B.sla_mxfp4_linear(x, c, s[:, :2], None, x[:, :8].contiguous())
    with pytest.raises(ValueError, match="y: "):
        B.sla_mxfp4_linear(x, c, s, None, x[:, :8])
