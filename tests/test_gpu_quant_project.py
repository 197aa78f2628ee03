"""h = x A^T in front of the products over a 4-bit weight: one launch of 16 x 16 tiles and its neighbours, at the ends of tokens, ranks and
columns, and where the other launch takes over."""
import pytest
import torch

import gpu_util as G
import quant_util as U
from oracle import dora_oracle as O
from paper_2603_22276_amd import binding as D

pytestmark = pytest.mark.gpu


def h_of(mod, behind):
    cfg = mod.cfg
    y, h = G.empty((cfg.tokens, cfg.d_out), cfg.dtype), G.empty((cfg.tokens + behind, cfg.r), cfg.dtype)
    D.dora_forward_quant(mod.desc, mod.x, None, mod.wq, mod.A, mod.B, mod.m_dev, None, None, y, h, None, None,
                         G.workspace(mod.desc, D.PHASE_FORWARD_QUANT))
    torch.cuda.synchronize()
    assert bool(torch.isnan(h[cfg.tokens:]).all())
    return y, h[:cfg.tokens]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,d_in,r", [
    (33, 8, 8), (47, 56, 24), (48, 64, 16), (49, 72, 40), (64, 1016, 136), (65, 1024, 8), (300, 1032, 72), (333, 2056, 72), (340, 4096, 184),
    (341, 4104, 200), (4096, 264, 16), (4097, 264, 16), (35, 5120, 384), (36, 5128, 384), (100, 9000, 8)])
def test_h_and_what_comes_of_it(dtype, tokens, d_in, r):
    mod = U.QuantModule(264, d_in, r, tokens, dtype, "int4", 32, seed=tokens)
    y, h = h_of(mod, behind=3)
    f = O.forward(**mod.oracle_args())
    G.assert_close("h", G.to_f64(h), f["h"], G.TOL[dtype]["tensor"])
    G.assert_close("y", G.to_f64(y), f["y"], G.TOL[dtype]["tensor"])


def test_a_token_of_nan_stays_in_its_row():
    mod = U.QuantModule(136, 1032, 24, 90, "bf16", "fp4", 64)
    want, _ = h_of(mod, 1)
    mod.x[17, 1031] = float("nan")
    got, h = h_of(mod, 1)
    assert bool(torch.isnan(got[17]).all()) and bool(torch.isnan(h[17]).all())
    keep = [t for t in range(90) if t != 17]
    assert torch.equal(got[keep], want[keep])
