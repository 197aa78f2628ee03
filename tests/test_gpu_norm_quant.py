"""The row norm straight from 4-bit codes (rows of a multiple of 32 weights): ends inside a tile of 128 x 128, groups shorter and longer
than one, every rank the launch takes and the first past it, with and without zero points, beside a workspace that holds no weight."""
import numpy as np
import pytest
import torch

import gpu_util as G
import quant_util as U
from oracle import dora_oracle as O
from paper_2603_22276_amd import binding as D

pytestmark = pytest.mark.gpu


def norm_of(mod, behind=0):
    c = torch.full((mod.cfg.d_out + behind,), -7.0, device=G.DEV)
    D.dora_norm_quant(mod.desc, mod.wq, mod.A, mod.B, c, G.workspace(mod.desc, D.PHASE_NORM_QUANT))
    assert bool((c[mod.cfg.d_out:] == -7.0).all())
    return c[:mod.cfg.d_out]


def check(mod):
    U.assert_norm(mod, norm_of(mod, behind=5), O.dense_row_norm(mod.W, mod.f64("A"), mod.f64("B"), float(mod.inp["s"])))


@pytest.mark.parametrize("kind,dtype", [("int4", "bf16"), ("zero", "f16"), ("zero", "bf16"), ("fp4", "bf16"), ("fp4", "f16")])
@pytest.mark.parametrize("r", [8, 64, 72, 128, 136, 200, 256, 320, 384, 392])
def test_ranks(kind, dtype, r):
    check(U.QuantModule(136, 416, r, 0, dtype, kind, 64, any_scale=True, seed=r))


@pytest.mark.parametrize("r", [16, 384])
@pytest.mark.parametrize("group", [32, 64, 128, 256, 1024])
@pytest.mark.parametrize("d_in", [32, 64, 96, 160, 224, 288, 2080])
def test_ends_and_groups(d_in, group, r):
    kind = ("int4", "zero", "fp4")[(d_in // 32 + group // 32) % 3]
    check(U.QuantModule(24, d_in, r, 0, "bf16" if d_in % 64 else "f16", kind, group, any_scale=True, seed=d_in))


@pytest.mark.parametrize("d_out", [8, 56, 64, 72, 120, 128, 1032])
@pytest.mark.parametrize("r,kind", [(128, "zero"), (264, "fp4"), (384, "int4")])
def test_rows(d_out, r, kind):
    check(U.QuantModule(d_out, 1184, r, 0, "bf16", kind, 32, any_scale=True, seed=d_out))


@pytest.mark.parametrize("r", [128, 384])
def test_many_slices_and_repeats(r):
    mod = U.QuantModule(256, 8224, r, 0, "bf16", "zero", 128)
    check(mod)
    first = norm_of(mod)
    assert all(torch.equal(norm_of(mod), first) for _ in range(3))


@pytest.mark.parametrize("r", [40, 264])
def test_a_group_that_is_not_finite_stays_in_its_row(r):
    mod = U.QuantModule(136, 320, r, 0, "bf16", "int4", 64)
    mod.scale[5, 1] = float("nan")
    mod.scale[77, 4] = float("inf")
    c = G.to_f64(norm_of(mod))
    ref = O.dense_row_norm(mod.W, mod.f64("A"), mod.f64("B"), float(mod.inp["s"]))
    bad = [5, 77]
    assert not np.isfinite(c[bad]).any()
    G.assert_norm_close(np.delete(c, bad), np.delete(ref, bad), G.TOL["bf16"]["norm"])


@pytest.mark.parametrize("tokens", [0, 3, 40, 400])
def test_inside_the_forward(tokens):
    mod = U.QuantModule(264, 1056, 72, tokens, "bf16", "zero", 64)
    c = G.to_f64(mod.forward()["c"])
    U.assert_norm(mod, G.to_dev(c.astype(np.float32)), O.dense_row_norm(mod.W, mod.f64("A"), mod.f64("B"), float(mod.inp["s"])))


def test_no_weight_in_the_workspace():
    desc = G.desc_of(U.QuantModule(512, 1024, 64, 0, "bf16").cfg)
    assert D.dora_workspace_bytes(desc, D.PHASE_NORM_QUANT) == D.dora_workspace_bytes(desc, D.PHASE_NORM)
