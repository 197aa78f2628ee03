"""4-bit weights at the ends of what is allowed: 2^31 weights but a few, in many rows and in few, where offsets in bytes pass 32 bits;
and two captured graphs that share a workspace."""
import pytest
import torch

import gpu_util as G
import quant_util as U
from paper_2603_22276_amd import binding as D

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def rows_of(q, scale, zero, group, rows):
    """Some rows of the weight in float64, from codes of int4 with zero points."""
    packed = q[rows]
    codes = torch.stack([packed & 15, packed >> 4], dim=-1).reshape(len(rows), -1).double()
    over = lambda t: t[rows].double().repeat_interleave(group, dim=1)[:, :codes.shape[1]]  # noqa: E731
    return (codes - over(zero)) * over(scale)


def weight(d_out, d_in, group):
    gen = torch.Generator(device=G.DEV).manual_seed(d_out)
    n = -(-d_in // group)
    q = torch.randint(0, 256, (d_out, d_in // 2), dtype=torch.uint8, device=G.DEV, generator=gen)
    scale = (torch.randint(8, 16, (d_out, n), dtype=torch.int32, device=G.DEV, generator=gen).float() * 2.0 ** -12).to(BF16)
    zero = torch.randint(0, 16, (d_out, n), dtype=torch.int32, device=G.DEV, generator=gen).to(BF16)
    return q, scale, zero, D.make_quant(D.QUANT_INT4, group, q, scale, zero)


def close(got, ref, tol):
    got, ref = got.double(), ref.double()
    assert bool(torch.isfinite(got).all())
    assert float((got - ref).norm() / ref.norm()) <= tol


@pytest.mark.parametrize("d_out,d_in,group", [(65528, 32768, 64), (262136, 8184, 32)])
def test_many_rows(d_out, d_in, group):
    r, s = 8, 0.5
    rows = torch.tensor([0, 1, 32767, 32768, d_out // 2 + 5, d_out - 129, d_out - 2, d_out - 1], device=G.DEV)
    q, scale, zero, wq = weight(d_out, d_in, group)
    W = rows_of(q, scale, zero, group, rows)
    A = (torch.randn((r, d_in), device=G.DEV) / d_in ** 0.5).to(BF16)
    B = torch.randn((d_out, r), device=G.DEV).to(BF16)
    m = torch.rand(d_out, device=G.DEV) + 0.5
    for T in (0, 2, 40):
        desc = D.make_desc(d_out, d_in, r, T, D.DORA_BF16, s)
        x = torch.randn((T, d_in), device=G.DEV).to(BF16)
        y = torch.empty((T, d_out), device=G.DEV, dtype=BF16)
        c = torch.empty(d_out, device=G.DEV)
        D.dora_forward_quant(desc, x, None, wq, A, B, m, None, None, y, None, None, c, G.workspace(desc, D.PHASE_FORWARD_QUANT))
        norm = (W + s * B[rows].double() @ A.double()).norm(dim=1)
        assert float(((c[rows].double() - norm) / norm).abs().max()) <= G.TOL["bf16"]["norm"]
        if T:
            inner = x.double() @ W.t().contiguous() + s * (x.double() @ A.double().t().contiguous()) @ B[rows].double().t().contiguous()
            close(y[:, rows], inner * (m[rows].double() / norm), 2.0 ** -7)   # (y and h are each off by half a step, 2^-8, at most)
    # read back, and brought to codes again: the same weights, whose scale is theirs wherever code 0 and 15 both are in the group
    back = torch.empty((d_out, d_in), device=G.DEV, dtype=BF16)
    D.dora_dequantize(desc, wq, back)
    assert bool((back[rows].double() == W).all())
    q2, scale2, zero2 = torch.empty_like(q), torch.empty_like(scale), torch.empty_like(zero)
    D.dora_quantize(desc, back, D.QUANT_INT4, group, q2, scale2, zero2)
    again = rows_of(q2, scale2, zero2, group, rows)
    step = scale2[rows].double().repeat_interleave(group, dim=1)[:, :d_in]
    assert bool(((again - W).abs() <= step / 2 * (1 + 2.0 ** -20)).all())


def test_long_rows():
    d_out, d_in, group, r, s, T = 8, 2 ** 28 - 32, 32, 8, 0.5, 3
    q, scale, zero, wq = weight(d_out, d_in, group)
    A = torch.empty((r, d_in), device=G.DEV, dtype=BF16).normal_().mul_(2.0 ** -14)
    B = torch.randn((d_out, r), device=G.DEV).to(BF16)
    m = torch.rand(d_out, device=G.DEV) + 0.5
    x = torch.empty((T, d_in), device=G.DEV, dtype=BF16).normal_()
    desc = D.make_desc(d_out, d_in, r, T, D.DORA_BF16, s)
    y, h, c = torch.empty((T, d_out), device=G.DEV, dtype=BF16), torch.empty((T, r), device=G.DEV, dtype=BF16), torch.empty(d_out, device=G.DEV)
    D.dora_forward_quant(desc, x, None, wq, A, B, m, None, None, y, h, None, c, G.workspace(desc, D.PHASE_FORWARD_QUANT))
    square, base, lora, step = 0.0, 0.0, 0.0, 2 ** 23
    everything = torch.arange(d_out, device=G.DEV)
    for k in range(0, d_in, step):
        n = min(step, d_in - k)
        W = rows_of(q[:, k // 2:(k + n) // 2], scale[:, k // group:(k + n) // group], zero[:, k // group:(k + n) // group], group, everything)
        a, xs = A[:, k:k + n].double(), x[:, k:k + n].double()
        square = square + torch.stack([(w + s * (b.double()[:, None] * a).sum(dim=0)).square().sum() for w, b in zip(W, B)])
        base = base + torch.stack([(xs * w).sum(dim=1) for w in W], dim=1)
        lora = lora + torch.stack([(xs * v).sum(dim=1) for v in a], dim=1)
    norm = square.sqrt()
    assert float(((c.double() - norm) / norm).abs().max()) <= G.TOL["bf16"]["norm"]
    close(h, lora, 2.0 ** -8)
    close(y, (base + s * lora @ B.double().t().contiguous()) * (m.double() / norm), 2.0 ** -7)


def test_graphs_that_share_a_workspace():
    mods = [U.QuantModule(520, 776, 40, 3, "bf16", "zero", 64, seed=1), U.QuantModule(520, 800, 64, 40, "bf16", "int4", 32, seed=2),
            U.QuantModule(264, 1032, 24, 400, "f16", "fp4", 128, seed=3)]
    size = max(D.dora_workspace_bytes(m.desc, ph) for m in mods for ph in (D.PHASE_FORWARD_QUANT, D.PHASE_BACKWARD_QUANT))
    ws = torch.empty(size, dtype=torch.uint8, device=G.DEV)

    def step(mod, out):
        D.dora_forward_quant(mod.desc, mod.x, None, mod.wq, mod.A, mod.B, mod.m_dev, None, None, out["y"], None, None, out["c"], ws)
        D.dora_backward_quant(mod.desc, mod.dy, mod.x, None, mod.wq, mod.A, mod.B, mod.m_dev, None, None, None, out["dx"], None, out["dA"],
                              out["dB"], out["dm"], ws)

    def outputs(mod):
        cfg = mod.cfg
        return {"y": G.empty((cfg.tokens, cfg.d_out), cfg.dtype), "c": G.empty_f32(cfg.d_out), "dx": G.empty((cfg.tokens, cfg.d_in), cfg.dtype),
                "dA": torch.empty((cfg.r, cfg.d_in), device=G.DEV), "dB": torch.empty((cfg.d_out, cfg.r), device=G.DEV), "dm": G.empty_f32(cfg.d_out)}

    want, got, graphs = [outputs(m) for m in mods], [outputs(m) for m in mods], []
    for mod, out in zip(mods, want):
        step(mod, out)
    torch.cuda.synchronize()
    for mod, out in zip(mods, got):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(mod, out)
        graphs.append(graph)
    for order in ((0, 1, 2), (2, 0, 1), (1, 1, 0, 2)):
        for out in got:
            for t in out.values():
                t.fill_(float("nan"))
        ws.fill_(0xFF)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(a[k], b[k]) for k in a)
        step(mods[order[0]], want[order[0]])           # eager work between the replays
        torch.cuda.synchronize()
