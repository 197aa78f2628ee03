"""dora_quantize and dora_dequantize of narrow weights: rows shorter than their group, and so many of them that a wave to each would be more
threads than a launch takes."""
import numpy as np
import pytest
import torch

import gpu_util as G
import quant_util as U
from oracle import quant_oracle as Q
from paper_2603_22276_amd import binding as D
from test_gpu_quant import KINDS, quantize_on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d_in", [8, 40, 64, 136, 264, 520])
@pytest.mark.parametrize("group", [64, 512, 2 ** 20])
def test_rows_shorter_than_their_group(dtype, kind, d_in, group):
    # (weights of 16 bits in fp32 too: no quotient lies within rounding of a tie)
    W = U.stored(np.random.default_rng(d_in).standard_normal((40, d_in)), "bf16")
    code = "fp4" if kind == "fp4" else "int4"
    q, scale, zero = Q.quantize(W, code, kind == "zero", group, lambda v: U.stored(v, dtype))
    got_q, got_scale, got_zero, back = quantize_on_gpu(W, dtype, kind, group)
    want = Q.weight(q, scale, zero, code, group)
    assert np.array_equal(got_scale, scale) and (zero is None or np.array_equal(got_zero, zero))
    assert np.array_equal(Q.weight(got_q, scale, zero, code, group), want)
    assert np.all(np.abs(back - want) <= U.HALF_STEP[dtype] * np.abs(want))


def test_many_rows_of_eight():
    # 2^26 and a few rows that repeat 4096 others; a group of 2^20 is the row, as one of 32 is
    rows, d_in = 2 ** 26 + 4096, 8
    few = torch.randn((4096, d_in), device=G.DEV, generator=torch.Generator(device=G.DEV).manual_seed(2)).to(torch.bfloat16)
    W = few.repeat(rows // 4096, 1)

    def through(w, group):
        n = w.shape[0]
        q = torch.full((n, d_in // 2), 0xA5, dtype=torch.uint8, device=G.DEV)
        scale, zero = (torch.full((n, 1), float("nan"), dtype=w.dtype, device=G.DEV) for _ in range(2))
        desc = D.make_desc(n, d_in, 8, 0, D.DORA_BF16, 1.0)
        D.dora_quantize(desc, w, D.QUANT_INT4, group, q, scale, zero)
        back = torch.full_like(w, float("nan"))
        D.dora_dequantize(desc, D.make_quant(D.QUANT_INT4, group, q, scale, zero), back)
        torch.cuda.synchronize()
        return q, scale, zero, back

    for got, want in zip(through(W, 2 ** 20), through(few, 32)):
        assert torch.equal(got.view(rows // 4096, -1), want.view(1, -1).expand(rows // 4096, -1))
