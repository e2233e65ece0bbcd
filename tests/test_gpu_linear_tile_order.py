"""The FP8 layer's large tiles on both sides of the sizes at which they are taken in another order (24 channel tiles of 128, rows of 2048
elements, 3 MB of weights; longer rows: channel tiles a multiple of K / 128): every row right, and the same bits twice.

The products of the codes are exact and K of them are summed in fp32: an output is off by at most (K + 4) 2^-24 of the sum of magnitudes
(the sum, two scales, the bias), before half a bf16 step, 2^-8 relative."""
import pytest
import torch

from paper_2605_11354_amd import binding as B

pytestmark = pytest.mark.gpu


def quantised(x):
    """The values of the layer's E4M3 numbers, fp64: fp32 scale and quotient (true divisions), one rounding."""
    x = x.float()
    top = x.abs().amax(1, keepdim=True).clamp(min=1e-8)
    scale = top / torch.full_like(top, 448.0)
    return (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).double() * scale.double()


@pytest.mark.parametrize("N,d_in,d_out", [(10992, 1024, 2944), (10992, 1024, 2952), (10992, 2048, 3080), (10992, 2176, 3080), (4100, 4096, 4096), (4100, 4096, 4104), (8200, 896, 3200), (5000, 512, 6144), (4097, 512, 6152), (25601, 256, 1160)])
def test_every_tile_is_right(N, d_in, d_out):
    g = torch.Generator(device="cuda").manual_seed(d_in + d_out)
    x = torch.randn((N, d_in), generator=g, device="cuda").mul_(torch.exp(torch.randn((N, 1), generator=g, device="cuda"))).to(torch.bfloat16)
    W = torch.randn((d_out, d_in), generator=g, device="cuda").to(torch.bfloat16)
    b = torch.randn((d_out,), generator=g, device="cuda").to(torch.bfloat16)
    y, again = (torch.full((N, d_out), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.sla_fp8_linear(x, W, b, y)
    B.sla_fp8_linear(x, W, b, again)
    xq, wq = quantised(x), quantised(W)
    ref, mag = xq @ wq.t() + b.double(), xq.abs() @ wq.abs().t() + b.double().abs()
    assert bool(((y.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (d_in + 4) * 2.0 ** -24 * mag).all())
    assert torch.equal(y.view(torch.int16), again.view(torch.int16))
