"""One module over a 4-bit weight, on the host (64 bits) and on the device, for the GPU tests."""
import numpy as np
import torch

import gpu_util as G
from oracle import dora_oracle as O
from oracle import quant_oracle as Q
from paper_2603_22276_amd import binding as D
from paper_2603_22276_amd import inputs as I

CODE = {"int4": D.QUANT_INT4, "fp4": D.QUANT_FP4}


def stored(a, dtype):
    """float64 rounded once to the storage type, as float64."""
    return I.to_f64(I.quantise(np.asarray(a), dtype))


class QuantModule:
    """`kind`: "int4", "zero" (int4 with zero points) or "fp4"; scales as dora_quantize chooses them, or (`any_scale`) with all
    the bits of the storage type and zero points that are no whole numbers."""

    def __init__(self, d_out, d_in, r, tokens, dtype, kind="int4", group=64, any_scale=False, seed=1):
        self.cfg = cfg = I.stress(I.DoraConfig("quant", d_out, d_in, r, tokens, dtype, 32.0, 1e-3, seed_offset=20000 + seed))
        inp = I.make_inputs(cfg)
        self.any_scale = any_scale
        self.inp, self.group, self.code = inp, group, "fp4" if kind == "fp4" else "int4"
        q, scale, zero = Q.quantize(I.to_f64(inp["W"]), self.code, kind == "zero", group, lambda v: stored(v, dtype))
        if any_scale:
            rng = np.random.default_rng(seed)
            scale = stored(scale * (1 + 0.3 * rng.standard_normal(scale.shape)), dtype)
            if zero is not None:
                zero = stored(zero + rng.standard_normal(zero.shape), dtype)
        self.W = Q.weight(q, scale, zero, self.code, group)
        self.m = (np.linalg.norm(self.W, axis=1) * (1 + 1e-3 * np.cos(np.arange(d_out)))).astype(np.float32)
        dev = lambda a: G.to_dev(I.quantise(a, dtype))  # noqa: E731
        self.q, self.scale, self.zero = torch.from_numpy(Q.pack(q)).to(G.DEV), dev(scale), None if zero is None else dev(zero)
        self.wq = D.make_quant(CODE[self.code], group, self.q, self.scale, self.zero)
        self.desc = G.desc_of(cfg)
        self.A, self.B, self.x, self.dy = (G.to_dev(inp[k]) for k in ("A", "B", "x", "dy"))
        self.m_dev = G.to_dev(self.m)

    def f64(self, k):
        return I.to_f64(self.inp[k])

    def oracle_args(self):
        return dict(x=self.f64("x"), W=self.W, A=self.f64("A"), B=self.f64("B"), m=self.m.astype(np.float64),
                    s=float(self.inp["s"]), eps=self.cfg.eps)

    def forward(self, w_norm=None, save=True, bias=None, x_lora=None, rows_behind=0):
        """Outputs of dora_forward_quant; `rows_behind` rows stand behind the last token and have to stay as they are."""
        cfg = self.cfg
        T = cfg.tokens
        y = G.empty((T + rows_behind, cfg.d_out), cfg.dtype)
        h = G.empty((T, cfg.r), cfg.dtype) if save else None
        inner = G.empty((T + rows_behind, cfg.d_out), cfg.dtype) if save else None
        c = G.empty_f32(cfg.d_out)
        D.dora_forward_quant(self.desc, self.x, x_lora, self.wq, self.A, self.B, self.m_dev, w_norm, bias, y, h, inner, c,
                             G.workspace(self.desc, D.PHASE_FORWARD_QUANT))
        if rows_behind:
            assert torch.isnan(y[T:]).all() and (inner is None or torch.isnan(inner[T:]).all())
        return {"y": y[:T], "h": h, "inner": None if inner is None else inner[:T], "c": c}

    def backward(self, w_norm=None, h=None, inner=None, x_lora=None, want_dm=True):
        cfg = self.cfg
        dx, dxl = G.empty((cfg.tokens, cfg.d_in), cfg.dtype), None if x_lora is None else G.empty((cfg.tokens, cfg.d_in), cfg.dtype)
        dA, dB, dm = G.empty_f32(cfg.r, cfg.d_in), G.empty_f32(cfg.d_out, cfg.r), G.empty_f32(cfg.d_out) if want_dm else None
        D.dora_backward_quant(self.desc, self.dy, self.x if x_lora is None else None, x_lora, self.wq, self.A, self.B, self.m_dev, w_norm, h,
                              inner, dx, dxl, dA, dB, dm, G.workspace(self.desc, D.PHASE_BACKWARD_QUANT))
        return {"dx": dx, "dx_lora": dxl, "dA": dA, "dB": dB, "dm": dm}


HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}   # relative


def assert_norm(mod, c, ref):
    """The module's bound on the norm, and where scales have all the bits of the storage type what reading the weight back may add:
    each weight is off by half a step at most, E = half step |W| element by element, and | ||D + E|| - ||D|| | <= ||E||."""
    c = G.to_f64(c)
    tol = G.TOL[mod.cfg.dtype]["norm"] * ref
    if mod.any_scale:
        tol = tol + HALF_STEP[mod.cfg.dtype] * np.linalg.norm(mod.W, axis=1)
    assert np.all(np.isfinite(c)) and np.all(np.abs(c - ref) <= tol), float(np.max(np.abs(c - ref) / ref))


def check_forward(mod, tol, **kw):
    f = O.forward(**mod.oracle_args())
    out = mod.forward(**kw)
    assert_norm(mod, out["c"], f["c"])
    for k in ("y", "h", "inner"):
        if out[k] is not None:
            G.assert_close(k, G.to_f64(out[k]), f[k], tol)
    return f, out
