"""Forward over a 4-bit weight by tiles that decode in the product (33 to 320 tokens, rows of an even number of groups, eight at least),
against the fp64 oracle: edges of the tiles of 64 and 128 tokens and of 128 and 256 rows, columns that end inside a step, inside a chunk
of 32 and inside a group, ranks that end inside a low-rank step, slices of the columns, pieces of eight groups that the row ends
in; and which launches such a call makes."""
import numpy as np
import pytest
import torch

import gpu_util as G
import quant_util as U
from paper_2603_22276_amd import binding as D

pytestmark = pytest.mark.gpu

QUANT_TILE, DEQUANTIZE, REDUCE, QUANT_TOKENS = 24, 21, 19, 23


def launches(call):
    D.dora_trace_reset()
    D.dora_trace_select(~0)
    D.dora_trace_enable(True)
    try:
        call()
        torch.cuda.synchronize()
    finally:
        D.dora_trace_enable(False)
    D.dora_trace_collect()
    n = {k: D.dora_trace_get(k)[1] for k in (QUANT_TILE, DEQUANTIZE, REDUCE, QUANT_TOKENS)}
    D.dora_trace_reset()
    return n


CASES = [  # d_out, d_in, r, tokens, group
    (128, 256, 64, 64, 32), (8, 256, 8, 33, 32), (264, 488, 24, 65, 32), (136, 312, 72, 300, 32), (520, 1000, 40, 127, 64), (264, 1160, 136, 128, 128),
    (392, 2048, 8, 129, 256), (1160, 504, 200, 48, 32), (120, 4088, 64, 100, 512), (2056, 1096, 16, 320, 64), (72, 8200, 40, 36, 1024),
    (256, 4096, 128, 200, 128),
    # tiles of 256 rows and 128 tokens
    (16400, 1000, 72, 300, 64), (20488, 1160, 8, 257, 128), (33000, 512, 40, 130, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kind", ["int4", "zero", "fp4"])
@pytest.mark.parametrize("d_out,d_in,r,tokens,group", CASES)
def test_forward(dtype, kind, d_out, d_in, r, tokens, group):
    mod = U.QuantModule(d_out, d_in, r, tokens, dtype, kind, group, any_scale=(tokens % 2 == 1))
    tol = G.TOL[dtype]["tensor"]
    f, out = U.check_forward(mod, tol, rows_behind=3)                       # norm inside, everything saved
    bias = torch.linspace(-1, 1, d_out, device=G.DEV).to(mod.A.dtype)
    kept = {}
    n = launches(lambda: kept.update(mod.forward(w_norm=out["c"], save=False, bias=bias, rows_behind=1)))   # norm given, nothing saved
    G.assert_close("y+bias", G.to_f64(kept["y"]), f["y"] + G.to_f64(bias), tol)
    # (rows of nine groups: the weight is read back)
    groups = -(-d_in // group)
    tile = groups >= 8 and groups % 2 == 0
    assert (n[QUANT_TILE], n[DEQUANTIZE], n[QUANT_TOKENS]) == (int(tile), int(not tile), 0)


@pytest.mark.parametrize("d_out,d_in,tokens,group,tile,back,tokens_kernel", [
    (256, 1024, 32, 128, 0, 0, 1), (256, 1024, 33, 128, 1, 0, 0), (256, 1024, 320, 128, 1, 0, 0), (256, 1024, 321, 128, 0, 1, 0),
    (256, 896, 64, 128, 0, 1, 0), (256, 1152, 64, 128, 0, 1, 0), (256, 1280, 64, 128, 1, 0, 0)])
def test_route(d_out, d_in, tokens, group, tile, back, tokens_kernel):
    mod = U.QuantModule(d_out, d_in, 16, tokens, "bf16", "int4", group)
    c = mod.forward()["c"]
    n = launches(lambda: mod.forward(w_norm=c, save=False))
    assert (n[QUANT_TILE], n[DEQUANTIZE], n[QUANT_TOKENS]) == (tile, back, tokens_kernel)


def test_slices_and_whole_columns_agree():
    # one shape whose columns go in slices, beside the weight read back: the same sums in another order
    mod = U.QuantModule(264, 8192, 40, 64, "bf16", "zero", 64)
    c = mod.forward()["c"]
    out = {}
    n = launches(lambda: out.update(mod.forward(w_norm=c)))
    assert n[QUANT_TILE] == 1 and n[REDUCE] >= 1
    W = G.empty((264, 8192), "bf16")
    D.dora_dequantize(mod.desc, mod.wq, W)
    y, inner, h, cc = G.empty((64, 264), "bf16"), G.empty((64, 264), "bf16"), G.empty((64, 40), "bf16"), G.empty_f32(264)
    D.dora_forward(mod.desc, mod.x, W, mod.A, mod.B, mod.m_dev, c, None, y, h, inner, cc, G.workspace(mod.desc, D.PHASE_FORWARD))
    # y and inner rounded once each, s h rounded in one of the two (2^-8 of the low-rank branch): three half steps
    for a, b in ((out["y"], y), (out["inner"], inner)):
        assert G.rel_fro(G.to_f64(a), G.to_f64(b)) <= 3 * 2.0 ** -8


def test_a_row_of_nan_scales_stays_to_itself():
    mod = U.QuantModule(264, 1000, 24, 100, "bf16", "int4", 64)
    mod.scale[5, 3] = float("nan")
    c = torch.ones(264, device=G.DEV)
    y = mod.forward(w_norm=c, save=False)["y"]
    assert torch.isnan(y[:, 5]).all()
    keep = np.arange(264) != 5
    want = (mod.f64("x") @ mod.W.T + float(mod.inp["s"]) * (mod.f64("x") @ mod.f64("A").T) @ mod.f64("B").T) * mod.m
    G.assert_close("y", G.to_f64(y)[:, keep], want[:, keep], 2e-2)
