"""dora_quantize and dora_dequantize take type and shape of the weight from the desc and nothing else."""
import pytest
import torch

import gpu_util as G
from paper_2603_22276_amd import binding as D

pytestmark = pytest.mark.gpu


def through(desc, W, group):
    d_out, d_in = W.shape
    q = torch.empty((d_out, d_in // 2), dtype=torch.uint8, device=G.DEV)
    scale, back = torch.empty((d_out, -(-d_in // group)), dtype=W.dtype, device=G.DEV), torch.empty_like(W)
    D.dora_quantize(desc, W, D.QUANT_INT4, group, q, scale, None)
    D.dora_dequantize(desc, D.make_quant(D.QUANT_INT4, group, q, scale), back)
    torch.cuda.synchronize()
    return q, scale, back


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("other", [dict(tokens=2 ** 31), dict(tokens=2 ** 62), dict(tokens=-1), dict(r=0), dict(r=-3), dict(r=2 ** 40), dict(s=float("nan")),
                                   dict(eps=float("nan"))], ids=str)
def test_only_type_and_shape_are_read(dtype, other):
    W = torch.randn((24, 72), device=G.DEV, generator=torch.Generator(device=G.DEV).manual_seed(1)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    make = lambda r=8, tokens=0, s=1.0, eps=0.0: D.make_desc(24, 72, r, tokens, G.dtype_code(dtype), s, eps)  # noqa: E731
    for a, b in zip(through(make(), W, 32), through(make(**other), W, 32)):
        assert torch.equal(a, b)
