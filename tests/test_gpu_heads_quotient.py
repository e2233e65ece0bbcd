"""The E4M3 form of heads divides by its scale as sla_quantise_e4m3 does: without norm and rotation queries and keys come out as
the stand-alone quantiser leaves them, bit for bit."""
import pytest
import torch

from paper_2605_11354_amd import binding as B

pytestmark = pytest.mark.gpu


def inputs(Bn, N, H):
    g = torch.Generator(device="cuda").manual_seed(N)
    qkv = torch.randn((Bn, N, 3, H, 64), generator=g, device="cuda").mul_(torch.exp(2 * torch.randn((Bn, N, 3, H, 1), generator=g, device="cuda"))).to(torch.bfloat16)
    qkv[:, ::3] = torch.randint(-127, 128, qkv[:, ::3].shape, generator=g, device="cuda").to(torch.bfloat16)          # many quotients half-way between two codes
    qkv[:, 1::7, :, :, ::5] = -0.0
    qkv[:, 2::7, :, :, ::5] = 0.0
    return qkv.unbind(2)


def run(p, qkv, bq, layout, **kw):
    Bn, N, H, _ = qkv[0].shape
    shape = (Bn, N, H, 64) if layout == "bnhd" else (Bn, H, N, 64)
    codes = [torch.full(shape, 0x55, dtype=torch.uint8, device="cuda") for _ in range(3)]
    scales = [torch.full((Bn, H, -(-N // b)), float("nan"), device="cuda") for b in (bq, 64, 64)]
    B.sla_qk_norm_rope_e4m3(p, *qkv, bq, *codes, *scales, **kw)
    return codes, scales


def quantiser(x, blk, layout):
    x = x.contiguous() if layout == "bnhd" else x.transpose(1, 2).contiguous()
    Bn, N, H = (x.shape[0], x.shape[1], x.shape[2]) if layout == "bnhd" else (x.shape[0], x.shape[2], x.shape[1])
    c, s = torch.empty(x.shape, dtype=torch.uint8, device="cuda"), torch.empty((Bn, H, -(-N // blk)), device="cuda")
    B.sla_quantise_e4m3(x, blk, c, s, layout=layout)
    return c, s


@pytest.mark.parametrize("bq", [64, 128])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("Bn,N,H", [(1, 1, 1), (2, 300, 3), (1, 4500, 16)])
def test_without_norm_and_rotation(Bn, N, H, layout, bq):
    qkv = inputs(Bn, N, H)
    codes, scales = run(B.make_heads_params(qkv[0], norm="none", axes=0, layout=layout), qkv, bq, layout)
    for c, s, x, blk in zip(codes, scales, qkv, (bq, 64, 64)):
        want = quantiser(x, blk, layout)
        torch.cuda.synchronize()
        assert torch.equal(s, want[1])
        assert torch.equal(c, want[0]), int((c != want[0]).sum())


@pytest.mark.parametrize("bq", [64, 128])
@pytest.mark.parametrize("axes,pairing", [(1, "halves"), (1, "adjacent"), (2, "halves")])
def test_rotation_by_nothing(axes, pairing, bq):
    """At position 0 the cosines are 1 and the sines 0: the values are the inputs, but for the sign of a zero."""
    qkv = inputs(2, 300, 3)
    pos = torch.zeros((300, axes), dtype=torch.int32, device="cuda")
    codes, scales = run(B.make_heads_params(qkv[0], norm="none", axes=axes, pairing=pairing), qkv, bq, "bhnd", pos=pos)
    for c, s, x, blk in zip(codes, scales, qkv, (bq, 64, 64)):
        want = quantiser(x, blk, "bhnd")
        torch.cuda.synchronize()
        assert torch.equal(s, want[1])
        assert torch.equal(c.view(torch.float8_e4m3fn).float(), want[0].view(torch.float8_e4m3fn).float())


@pytest.mark.parametrize("bq", [64, 128])
def test_infinities_and_nan(bq):
    q, k, v = inputs(2, 300, 3)
    for t in (q, k, v):
        t[0, 5, 0, 7], t[1, 70, 1, 0], t[1, 299, 2, 63] = float("inf"), float("nan"), float("-inf")
        t[0, 128:192, 2] = float("nan")
    codes, scales = run(B.make_heads_params(q, norm="none", axes=0), (q, k, v), bq, "bhnd")
    for c, s, x, blk in zip(codes, scales, (q, k, v), (bq, 64, 64)):
        want = quantiser(x, blk, "bhnd")
        torch.cuda.synchronize()
        assert torch.equal(s, want[1]) and torch.equal(c, want[0])
