"""Forwards over a 4-bit weight in exactly the scratch that their phase names, between bytes that have to stay as they are: the results are
those in the scratch that any forward takes."""
import pytest
import torch

import gpu_util as G
import quant_util as U
from paper_2603_22276_amd import binding as D

pytestmark = pytest.mark.gpu


def forward(mod, w_norm, phase, x_lora=None):
    cfg = mod.cfg
    y, c = G.empty((cfg.tokens, cfg.d_out), cfg.dtype), G.empty_f32(cfg.d_out)
    n = D.dora_workspace_bytes(mod.desc, phase)
    room = torch.full((n + 512,), 0xC3, dtype=torch.uint8, device=G.DEV)
    D.dora_forward_quant(mod.desc, mod.x, x_lora, mod.wq, mod.A, mod.B, mod.m_dev, w_norm, None, y, None, None, c, room[256:256 + n])
    torch.cuda.synchronize()
    assert bool((room[:256] == 0xC3).all()) and bool((room[256 + n:] == 0xC3).all())
    return y, c


@pytest.mark.parametrize("dtype,d_out,d_in,r,tokens,kind,group", [
    ("bf16", 264, 1056, 40, 1, "int4", 128), ("f16", 520, 544, 72, 32, "zero", 32), ("bf16", 136, 1032, 24, 7, "fp4", 64), ("bf16", 264, 544, 392, 20, "zero", 64),
    ("bf16", 264, 1024, 40, 33, "int4", 64), ("f16", 264, 1024, 72, 300, "fp4", 128), ("bf16", 136, 264, 24, 65, "int4", 32), ("f16", 200, 520, 40, 700, "zero", 64),
    ("f32", 100, 136, 12, 33, "zero", 32), ("bf16", 72, 8192, 16, 64, "int4", 128), ("bf16", 264, 544, 40, 0, "int4", 64)])
def test_in_the_scratch_of_the_phase(dtype, d_out, d_in, r, tokens, kind, group):
    mod = U.QuantModule(d_out, d_in, r, tokens, dtype, kind, group)
    want, c = forward(mod, None, D.PHASE_FORWARD_QUANT)
    for w_norm, phase, x_lora in ((None, D.PHASE_FORWARD_QUANT_PLAIN, None), (c, D.PHASE_FORWARD_QUANT_NORM_GIVEN, None),
                                  (c, D.PHASE_FORWARD_QUANT_NORM_GIVEN, mod.x)):
        got, cc = forward(mod, w_norm, phase, x_lora)
        assert torch.equal(got, want) and torch.equal(cc, c)
