"""4-bit frozen weights against the oracle: codes and scales value by value, the weight read back, norm, forward and backward of
the module over it, at the edges of groups, words, tiles and token blocks.

Bounds: codes, scales and zero points are equal; a weight read back is off by half a step of the storage type at most (nothing
for scales as dora_quantize chooses them); the module's outputs are held to the bounds of the 16-bit and fp32 module.
"""
import numpy as np
import pytest
import torch

import gpu_util as G
import quant_util as U
from oracle import dora_oracle as O
from oracle import quant_oracle as Q
from paper_2603_22276_amd import binding as D
from paper_2603_22276_amd import inputs as I

pytestmark = pytest.mark.gpu

KINDS = ["int4", "zero", "fp4"]


def quantize_on_gpu(W, dtype, kind, group):
    d_out, d_in = W.shape
    n = Q.groups_of(d_in, group)
    desc = D.make_desc(d_out, d_in, 8, 0, G.dtype_code(dtype), 1.0)
    Wd = G.to_dev(I.quantise(W, dtype))
    q = torch.full((d_out, d_in // 2), 0xA5, dtype=torch.uint8, device=G.DEV)
    scale, zero = G.empty((d_out, n), dtype), G.empty((d_out, n), dtype) if kind == "zero" else None
    D.dora_quantize(desc, Wd, U.CODE["fp4" if kind == "fp4" else "int4"], group, q, scale, zero)
    back = G.empty((d_out, d_in), dtype)
    D.dora_dequantize(desc, D.make_quant(U.CODE["fp4" if kind == "fp4" else "int4"], group, q, scale, zero), back)
    torch.cuda.synchronize()
    packed = q.cpu().numpy()
    codes = np.empty((d_out, d_in), dtype=np.uint8)
    codes[:, 0::2], codes[:, 1::2] = packed & 15, packed >> 4
    return codes, G.to_f64(scale), None if zero is None else G.to_f64(zero), G.to_f64(back)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d_out,d_in,group", [(4, 8, 32), (8, 40, 32), (24, 200, 64), (264, 1032, 128), (40, 2056, 256), (20, 4104, 1024),
                                              (12, 264, 2 ** 30), (1000, 776, 32)])
def test_codes_and_scales(dtype, kind, d_out, d_in, group):
    if dtype != "f32" and d_out % 8:
        d_out += 4
    rng = np.random.default_rng(d_out + d_in)
    W = U.stored(rng.standard_normal((d_out, d_in)) * 0.02 + (0.01 if kind == "zero" else 0.0), dtype)
    W[:, ::7] *= 2.0 ** rng.integers(-6, 3, size=W[:, ::7].shape)
    W = U.stored(W, dtype)
    # (fp32 is compared where the quotient is not within rounding of a tie: a weight of 16 bits in fp32 is that)
    W = U.stored(W, "bf16") if dtype == "f32" else W
    code = "fp4" if kind == "fp4" else "int4"
    q, scale, zero = Q.quantize(W, code, kind == "zero", group, lambda v: U.stored(v, dtype), 65504 if dtype == "f16" else np.inf)
    got_q, got_scale, got_zero, back = quantize_on_gpu(W, dtype, kind, group)
    assert np.array_equal(got_scale, scale)
    if zero is not None:
        assert np.array_equal(got_zero, zero)
    # the sign of a code that stands for 0 is free
    assert np.array_equal(Q.weight(got_q, scale, zero, code, group), Q.weight(q, scale, zero, code, group))
    want = Q.weight(q, scale, zero, code, group)
    assert np.all(np.abs(back - want) <= U.HALF_STEP[dtype] * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 0.0))
    if dtype == "bf16":
        assert np.array_equal(back, want)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_groups_of_zeros_infinities_and_tiny_weights(dtype, kind):
    W = np.zeros((8, 128))
    W[1, 3] = np.inf
    W[2, 40] = -np.inf
    W[3, 70] = np.nan
    W[4, :] = 2.0 ** -24 if dtype == "f16" else 2.0 ** -126
    W[5, :32], W[5, 32:] = -3.0, 3.0
    W[6, 5] = 65504.0 if dtype == "f16" else 2.0 ** 126
    W[7, 5], W[7, 6] = -1.0, 1.0
    code = "fp4" if kind == "fp4" else "int4"
    q, scale, zero = Q.quantize(W, code, kind == "zero", 32, lambda v: U.stored(v, dtype), 65504 if dtype == "f16" else np.inf)
    got_q, got_scale, got_zero, back = quantize_on_gpu(W, dtype, kind, 32)
    rows = [0, 1, 2, 3, 5, 7] + ([6] if kind != "zero" or dtype == "f16" else [])   # (row 4: scales in the subnormal range)
    assert np.array_equal(got_scale[rows], scale[rows], equal_nan=True)
    want = Q.weight(q, scale, zero, code, 32)
    assert np.array_equal(np.isnan(back[rows]), np.isnan(want[rows]))
    fine = ~np.isnan(want[rows])
    assert np.all(np.abs(back[rows] - want[rows])[fine] <= U.HALF_STEP[dtype] * np.abs(want[rows])[fine])
    assert np.isnan(back[1, :32]).all() and np.isnan(back[2, 32:64]).all() and np.isnan(back[3, 64:96]).all()
    assert not np.isnan(back[1, 32:]).any() and not back[0].any()
    assert np.isfinite(back[4]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("group", [32, 2048])
@pytest.mark.parametrize("exponent", [-126, -122, -116, -104, -96])
def test_tiny_weights_take_the_nearest_code(dtype, kind, group, exponent):
    W = U.stored(np.random.default_rng(-exponent).uniform(-1, 1, (8, 2048)) * 2.0 ** exponent, dtype)
    q, scale, zero, back = quantize_on_gpu(W, dtype, kind, group)
    s = np.repeat(scale, group, axis=1)[:, :2048]
    if kind == "fp4":
        values = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
        values = np.concatenate([values, -values])
    else:
        values = np.arange(16.0)
    off = 8.0 * (kind == "int4") if zero is None else np.repeat(zero, group, axis=1)[:, :2048]
    best = np.min([np.abs((v - off) * s - W) for v in values], axis=0)
    # (read back the product is rounded once: half a step of the smallest numbers)
    assert np.all(np.abs(back - W) <= best * (1 + 2.0 ** -20) + (2.0 ** -134 if dtype == "bf16" else 2.0 ** -150))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_any_scale_reads_back_within_half_a_step(dtype, kind):
    mod = U.QuantModule(40, 328, 8, 1, dtype, kind, 32, any_scale=True)
    back = G.empty((40, 328), dtype)
    D.dora_dequantize(mod.desc, mod.wq, back)
    # (a zero point that is no whole number: the difference is rounded to fp32 first, and the product once more)
    assert np.all(np.abs(G.to_f64(back) - mod.W) <= (U.HALF_STEP[dtype] + 2 * 2.0 ** -24) * np.abs(mod.W) + 2.0 ** -25)


@pytest.mark.parametrize("dtype,d_out,d_in,r,kind,group", [
    ("bf16", 264, 392, 40, "int4", 128), ("f16", 136, 1096, 128, "zero", 64), ("bf16", 520, 264, 384, "fp4", 32), ("bf16", 136, 200, 392, "int4", 32),
    ("f32", 100, 136, 12, "zero", 32), ("bf16", 8, 8, 8, "fp4", 32), ("f16", 72, 2056, 8, "int4", 256), ("bf16", 1032, 1160, 200, "zero", 128),
    ("f16", 264, 648, 320, "fp4", 64), ("bf16", 128, 128, 64, "int4", 64)])
def test_norm(dtype, d_out, d_in, r, kind, group):
    mod = U.QuantModule(d_out, d_in, r, 0, dtype, kind, group, any_scale=(r % 16 == 0))
    c = G.empty_f32(d_out)
    D.dora_norm_quant(mod.desc, mod.wq, mod.A, mod.B, c, G.workspace(mod.desc, D.PHASE_NORM_QUANT))
    U.assert_norm(mod, c, O.dense_row_norm(mod.W, mod.f64("A"), mod.f64("B"), float(mod.inp["s"])))


FORWARD = [  # d_out, d_in, r, tokens, group
    (8, 8, 8, 1, 32), (24, 40, 8, 2, 32), (264, 72, 24, 15, 64), (200, 1000, 40, 16, 128), (520, 392, 136, 17, 32), (72, 2312, 384, 31, 256),
    (1032, 520, 72, 32, 64), (136, 4104, 40, 33, 128), (520, 264, 392, 48, 32), (264, 1032, 8, 64, 512), (264, 392, 40, 65, 128),
    (8200, 72, 24, 1, 32), (8248, 136, 8, 17, 64), (72, 72, 1544, 3, 32), (136, 4096, 64, 4, 128), (16400, 264, 8, 9, 128),
    (264, 648, 72, 127, 64), (136, 1096, 200, 128, 128), (392, 520, 40, 129, 32), (1160, 264, 24, 300, 256), (520, 136, 392, 513, 64),
    (264, 2056, 16, 200, 1024),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d_out,d_in,r,tokens,group", FORWARD)
def test_forward(dtype, kind, d_out, d_in, r, tokens, group):
    mod = U.QuantModule(d_out, d_in, r, tokens, dtype, kind, group, any_scale=(tokens % 2 == 1))
    tol = G.TOL[dtype]["tensor"]
    f, out = U.check_forward(mod, tol, rows_behind=3)                       # norm inside, everything saved
    bias = torch.linspace(-1, 1, d_out, device=G.DEV).to(mod.A.dtype)
    kept = mod.forward(w_norm=out["c"], save=False, bias=bias, rows_behind=1)   # norm given, nothing saved
    G.assert_close("y+bias", G.to_f64(kept["y"]), f["y"] + G.to_f64(bias), tol)
    assert torch.equal(kept["c"], out["c"])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d_out,d_in,r,tokens,group", [(4, 8, 4, 1, 32), (100, 136, 12, 33, 32), (256, 512, 16, 64, 128), (1000, 776, 36, 150, 64)])
def test_f32_forward_and_backward(kind, d_out, d_in, r, tokens, group):
    mod = U.QuantModule(d_out, d_in, r, tokens, "f32", kind, group)
    _, out = U.check_forward(mod, G.TOL["f32"]["tensor"])
    want = O.backward(mod.f64("dy"), **mod.oracle_args())
    for kw in (dict(), dict(w_norm=out["c"], h=out["h"], inner=out["inner"])):
        got = mod.backward(**kw)
        for k in ("dx", "dA", "dB", "dm"):
            G.assert_close(k, G.to_f64(got[k]), want[k], G.TOL["f32"]["tensor"])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d_out,d_in,r,tokens,kind,group", [(8, 8, 8, 1, "int4", 32), (264, 392, 40, 65, "zero", 64), (520, 1032, 136, 300, "fp4", 32),
                                                            (200, 2056, 392, 129, "int4", 256)])
def test_backward(dtype, d_out, d_in, r, tokens, kind, group):
    mod = U.QuantModule(d_out, d_in, r, tokens, dtype, kind, group, any_scale=True)
    want = O.backward(mod.f64("dy"), **mod.oracle_args())
    out = mod.forward()
    tol = G.TOL[dtype]["tensor"]
    for kw in (dict(), dict(w_norm=out["c"], h=out["h"], inner=out["inner"]), dict(w_norm=out["c"], want_dm=False)):
        got = mod.backward(**kw)
        for k in ("dx", "dA", "dB", "dm"):
            if got[k] is not None:
                G.assert_close(k, G.to_f64(got[k]), want[k], tol)


def test_gradient_of_x_against_differences():
    # y is linear in x, so that a difference over a step of any size is the derivative: fp32, one element after another
    mod = U.QuantModule(24, 40, 8, 3, "f32", "zero", 32)
    dx = G.to_f64(mod.backward()["dx"])
    c = mod.forward()["c"]
    dy = mod.f64("dy")
    for t, k in ((0, 0), (1, 17), (2, 39)):
        x0 = mod.x[t, k].item()
        ys = []
        for x1 in (x0 + 4.0, x0 - 4.0):
            mod.x[t, k] = x1
            ys.append((G.to_f64(mod.forward(w_norm=c)["y"]) * dy).sum())
        mod.x[t, k] = x0
        # y of up to |y| ~ 20 in fp32 sums of 72 values: 2^-24 * 20 * 72 over a step of 8, with room for its accumulation
        assert abs((ys[0] - ys[1]) / 8.0 - dx[t, k]) <= 1e-4 * max(1.0, np.abs(dx).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_of_zero(dtype):
    mod = U.QuantModule(24, 40, 8, 0, dtype)
    c = G.empty_f32(24)
    D.dora_forward_quant(mod.desc, None, None, mod.wq, mod.A, mod.B, mod.m_dev, None, None, None, None, None, c,
                         G.workspace(mod.desc, D.PHASE_FORWARD_QUANT))
    G.assert_norm_close(G.to_f64(c), O.dense_row_norm(mod.W, mod.f64("A"), mod.f64("B"), float(mod.inp["s"])), G.TOL[dtype]["norm"])
    g = mod.backward()
    assert not g["dA"].any() and not g["dB"].any() and not g["dm"].any()


def test_zero_scaling_and_a_row_of_zeros():
    mod = U.QuantModule(24, 72, 8, 5, "bf16", "int4", 32)
    mod.q[3] = 0x88                                       # a row of zeros
    mod.W[3] = 0.0
    for s in (0.0, float(mod.inp["s"])):
        mod.desc.s = s
        mod.inp["s"] = np.float32(s)
        mod.B[3] = 0
        f = O.forward(**{**mod.oracle_args(), "B": G.to_f64(mod.B)})
        out = mod.forward()
        assert out["c"][3] == 0.0
        keep = np.arange(24) != 3
        G.assert_norm_close(G.to_f64(out["c"])[keep], f["c"][keep], 1e-3)
        G.assert_close("y", G.to_f64(out["y"])[:, keep], f["y"][:, keep], 2e-2)
        assert not out["y"][:, 3].any()


def test_token_rows_of_nan_stay_to_themselves():
    for T in (3, 20, 100):
        mod = U.QuantModule(136, 264, 24, T, "bf16", "zero", 32)
        mod.x[1] = float("nan")
        y = mod.forward()["y"]
        assert torch.isnan(y[1]).all()
        keep = torch.arange(T, device=G.DEV) != 1
        f = O.forward(**mod.oracle_args())
        G.assert_close("y", G.to_f64(y[keep]), f["y"][keep.cpu().numpy()], 2e-2)


def test_the_same_call_twice_and_on_another_stream_is_the_same():
    for T in (1, 27, 100, 400):
        mod = U.QuantModule(264, 1032, 40, T, "bf16", "int4", 128)
        a = mod.forward()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            b = mod.forward()
        torch.cuda.current_stream().wait_stream(side)
        for k in a:
            assert torch.equal(a[k], b[k]), (T, k)


def test_weights_unaligned_to_their_lines_and_misaligned_bases():
    # the tensors start 16 bytes into an allocation, as views of a larger one do
    mod = U.QuantModule(72, 264, 24, 20, "f16", "zero", 32)
    for name in ("q", "scale", "zero", "x", "A", "B"):
        t = getattr(mod, name)
        big = torch.empty(t.numel() + 16 // t.element_size(), dtype=t.dtype, device=G.DEV)
        view = big[16 // t.element_size():].view(t.shape)
        view.copy_(t)
        setattr(mod, name, view)
    mod.wq = D.make_quant(mod.wq.code, 32, mod.q, mod.scale, mod.zero)
    U.check_forward(mod, G.TOL["f16"]["tensor"])
