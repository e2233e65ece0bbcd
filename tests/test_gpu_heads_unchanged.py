"""Without norm and rotation the bf16 form is a change of layout: every bit of q, k and v arrives, signs of zeros among them."""
import pytest
import torch

from paper_2605_11354_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Bn,N,H", [(1, 1, 1), (2, 130, 3), (1, 4500, 16)])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_every_bit(Bn, N, H, layout):
    g = torch.Generator(device="cuda").manual_seed(N)
    bits = torch.randint(-32768, 32768, (Bn, N, 3, H, 64), generator=g, device="cuda").to(torch.int16)
    bits = torch.where((bits & 0x7F80) == 0x7F80, bits & ~0x4000, bits)                      # every finite number
    bits[:, ::2, :, :, ::3] = -32768                                                         # -0
    bits[:, ::2, :, :, 1::3] = 0
    qkv = bits.view(torch.bfloat16).unbind(2)
    out = [torch.full((Bn, N, H, 64) if layout == "bnhd" else (Bn, H, N, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    B.sla_qk_norm_rope(B.make_heads_params(qkv[0], norm="none", axes=0, layout=layout), *qkv, *out)
    torch.cuda.synchronize()
    for x, y in zip(bits.unbind(2), out):
        y = y if layout == "bnhd" else y.transpose(1, 2)
        assert torch.equal(x, y.contiguous().view(torch.int16))
