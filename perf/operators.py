"""The operators of a DoRA module over a 4-bit frozen weight, and the dropout in front of its adapter, as cases that can be
timed and whose results can be compared.

A case is a dict of plain values.  `kind` says which operator one pass goes through:

  quantize  a weight to 4-bit codes with group scales (dora_quantize) and back (dora_dequantize)
  norm      the row norm of W + s B A with W in 4 bits (dora_norm_quant)
  forward   the module's forward over such a weight (dora_forward_quant), from one token to a long prompt
  backward  its backward, everything recomputed (dora_backward_quant)
  dropout   x_lora = dropout(x) with a mask that is drawn again wherever it is needed and never stored (dora_dropout)
  dropout_backward  dx + mask (.) dx_lora / (1 - p) with the same mask (dora_dropout_backward)

The 4-bit weight: W[j, k] = scale[j, k / group] * (value of code q[j, k]).  `code` "int4": the value is q - zero, zero being 8 or
(`zero` true) a number per group; "fp4": the value is that of the E2M1 float q.  Byte i of a row holds weights 2 i (low four
bits) and 2 i + 1 (high four bits).  The last group of a row may be short.

The mask: elements are numbered along the rows of x, eight of them share a block, block b takes the 128 bits of Philox 4x32-10
(Salmon et al. 2011) of counter (offset + b, 0) under key `seed`, element j of the block their bits 16 j .. 16 j + 15, and it is
kept if those are at least t = round(65536 p); what is kept is multiplied by 65536 / (65536 - t).

`own` false: elementary torch operations in 32 bits, rounded once.  `own` true: the framework's calls.
"""
import torch

own = False

DEV = "cuda:0"
TORCH_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BRANCH = 0.25   # s * sigma_B * sqrt(r): standard deviation of the low-rank branch against the frozen layer's
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # loading a base model: a key / value projection is brought to 4 bits, symmetric integers
        {"name": "quantize_projection", "kind": "quantize", "d_out": 1024, "d_in": 4096, "dtype": "bf16", "code": "int4",
         "zero": False, "group": 128},
        # the same for a wide MLP module in fp16, with zero points, rows that end inside a group
        {"name": "quantize_mlp_f16_zero", "kind": "quantize", "d_out": 14336, "d_in": 4104, "dtype": "f16", "code": "int4",
         "zero": True, "group": 64},
        # the norm after an optimiser step, a projection with a small adapter and short groups of 4-bit floats
        {"name": "norm_projection_fp4", "kind": "norm", "d_out": 4096, "d_in": 4096, "r": 64, "dtype": "bf16", "code": "fp4",
         "zero": False, "group": 32},
        # the same for the benchmark's largest module and rank
        {"name": "norm_8192", "kind": "norm", "d_out": 8192, "d_in": 8192, "r": 384, "dtype": "bf16", "code": "int4",
         "zero": False, "group": 128},
        # serving, one sequence: every token of the answer is such a call per adapted module; launches and latency count
        {"name": "decode_one_token", "kind": "forward", "d_out": 4096, "d_in": 4096, "r": 384, "tokens": 1, "dtype": "bf16",
         "code": "int4", "zero": False, "group": 128, "norm": "kept", "bias": False},
        # serving, a batch of sequences decoded together: fp16, zero points, a base layer with bias, a wide MLP module
        {"name": "decode_batch_f16", "kind": "forward", "d_out": 14336, "d_in": 4096, "r": 64, "tokens": 27, "dtype": "f16",
         "code": "int4", "zero": True, "group": 64, "norm": "kept", "bias": True},
        # serving, a short prompt, ragged everywhere, 4-bit floats
        {"name": "prefill_short_fp4", "kind": "forward", "d_out": 3000, "d_in": 2056, "r": 72, "tokens": 333, "dtype": "bf16",
         "code": "fp4", "zero": False, "group": 32, "norm": "kept", "bias": False},
        # serving, a long prompt through a wide MLP module
        {"name": "prefill_long", "kind": "forward", "d_out": 14336, "d_in": 4096, "r": 64, "tokens": 1999, "dtype": "bf16",
         "code": "int4", "zero": False, "group": 128, "norm": "kept", "bias": False},
        # fp32 fine-tuning of a small layer over a 4-bit base under gradient checkpointing: norm, h and inner recomputed
        {"name": "backward_f32_ragged", "kind": "backward", "d_out": 1000, "d_in": 776, "r": 36, "tokens": 1500, "dtype": "f32",
         "code": "int4", "zero": True, "group": 32, "frozen_m": False},
        # the headline module in 4 bits, gradients of the adapter and of x, magnitude frozen: the largest call
        {"name": "backward_8192", "kind": "backward", "d_out": 8192, "d_in": 8192, "r": 384, "tokens": 8192, "dtype": "bf16",
         "code": "int4", "zero": False, "group": 128, "frozen_m": True},
        # training with LoRA dropout: the adapter's input of a ragged batch
        {"name": "dropout_ragged_f16", "kind": "dropout", "tokens": 1501, "d_in": 3000, "dtype": "f16", "p": 0.1},
        # and the way back, at the headline batch
        {"name": "dropout_backward_8192", "kind": "dropout_backward", "tokens": 8192, "d_in": 8192, "dtype": "bf16", "p": 0.05},
    ]


def _log(rng, lo, hi, mult):
    """A multiple of `mult` between lo and hi, spread evenly over the logarithm."""
    v = lo * (hi / lo) ** rng.random()
    return max(mult, int(round(v / mult)) * mult)


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw(rng)
        if _cost(case) <= most:
            return case


def _draw(rng):
    kind = rng.choice(["quantize", "norm", "forward", "forward", "forward", "backward", "backward", "dropout", "dropout_backward"])
    half = rng.choice(["bf16", "bf16", "f16"])
    code = rng.choice(["int4", "int4", "fp4"])
    q = {"code": code, "zero": code == "int4" and rng.random() < 0.5, "group": rng.choice([32, 64, 128, 256])}
    if kind in ("dropout", "dropout_backward"):
        return {"kind": kind, "tokens": _log(rng, 64, 16384, 1), "d_in": _log(rng, 256, 8192, 8), "dtype": rng.choice([half, half, "f32"]),
                "p": rng.choice([0.01, 0.05, 0.1, 0.5])}
    if kind == "quantize":
        return {"kind": kind, "d_out": _log(rng, 512, 16384, 8), "d_in": _log(rng, 512, 16384, 8), "dtype": half, **q}
    if kind == "norm":
        return {"kind": kind, "d_out": _log(rng, 512, 16384, 8), "d_in": _log(rng, 512, 16384, 8), "r": _log(rng, 8, 768, 8),
                "dtype": half, **q}
    if kind == "forward":
        # decode (a few tokens) as often as prefill; the norm is inside the call now and then
        tokens = _log(rng, 1, 64, 1) if rng.random() < 0.5 else _log(rng, 65, 8192, 1)
        return {"kind": kind, "d_out": _log(rng, 512, 16384, 8), "d_in": _log(rng, 512, 16384, 8), "r": _log(rng, 8, 768, 8),
                "tokens": tokens, "dtype": half, **q, "norm": "kept" if rng.random() < 0.7 else "inside", "bias": rng.random() < 0.3}
    if rng.random() < 0.3:
        return {"kind": kind, "d_out": _log(rng, 64, 2048, 8), "d_in": _log(rng, 64, 2048, 8), "r": _log(rng, 8, 128, 4),
                "tokens": _log(rng, 16, 2048, 1), "dtype": "f32", **q, "frozen_m": rng.random() < 0.2}
    return {"kind": kind, "d_out": _log(rng, 512, 14336, 8), "d_in": _log(rng, 512, 14336, 8), "r": _log(rng, 8, 768, 8),
            "tokens": _log(rng, 128, 8192, 1), "dtype": half, **q, "frozen_m": True}


# ---- the 4-bit weight in plain form ------------------------------------------------------------------------------------
def _round_four_bits(v):
    """fp32 rounded to four significant bits, to nearest, ties to even."""
    u = v.view(torch.int32)
    return ((u + 0x7FFFF + ((u >> 20) & 1)) & ~0xFFFFF).view(torch.float32)


def _grouped(w, group):
    """[rows, d_in] with the last group filled up with zeros, as [rows, groups, group]."""
    rows, d_in = w.shape
    n = -(-d_in // group)
    if n * group != d_in:
        w = torch.cat([w, w.new_zeros(rows, n * group - d_in)], dim=1)
    return w.view(rows, n, group)


def _quantize(W, code, with_zero, group):
    """Codes [d_out, d_in] (uint8), scale and zero (or None) [d_out, groups] of W.

    int4: scale = largest magnitude / 7 (four significant bits, to nearest), q = 8 + round(w / scale); with zero points scale =
    (max - min) / 15 over the group and 0 (four significant bits, upwards), zero = round(-min / scale), q = zero + round(w /
    scale) kept within 0 .. 15.  fp4: scale = largest magnitude / 6 (four significant bits, to nearest), q the nearest E2M1 float
    (halfway: the even code), its sign in bit 3 where w < 0.  A scale of 0 gives the code of 0 everywhere.
    """
    w = _grouped(W.float(), group)
    zero = None
    steps = w.new_full((), 15 if with_zero else 7 if code == "int4" else 6)   # (a tensor: a division, not a product with 1 / steps)
    if with_zero:
        lo, hi = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
        raw = (hi - lo) / steps
        near = _round_four_bits(raw)
        step = torch.ldexp(torch.ones_like(near), torch.frexp(near).exponent - 4)   # one unit of the fourth bit
        scale = torch.where(near < raw, near + step, near).to(W.dtype)
    else:
        scale = _round_four_bits(w.abs().amax(2) / steps).to(W.dtype)
    s = scale.float()
    some = s > 0
    safe = torch.where(some, s, torch.ones_like(s))
    if with_zero:
        z = torch.where(some, (-lo / safe).round().clamp(0, 15), torch.zeros_like(s))
        zero = z.to(W.dtype)
        q = (z[..., None] + (w / safe[..., None]).round()).clamp(0, 15)
        q = torch.where(some[..., None], q, z[..., None])
    elif code == "int4":
        q = (8 + (w / safe[..., None]).round()).clamp(0, 15)
        q = torch.where(some[..., None], q, torch.full_like(q, 8))
    else:
        a = w.abs()
        q = torch.zeros_like(w)
        for i, mid in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
            edge = (mid * safe)[..., None]
            q += (a > edge) if i % 2 == 0 else (a >= edge)
        q = torch.where(some[..., None], q + 8 * (w < 0), torch.zeros_like(q))
    q = q.to(torch.uint8).reshape(W.shape[0], -1)[:, : W.shape[1]]
    return q, scale, zero


def _pack(q):
    return (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous()


def _weight(packed, scale, zero, code, group, dtype=torch.float32):
    """The weight that codes and scales stand for, [d_out, d_in]."""
    rows, half = packed.shape
    q = torch.stack([packed & 15, packed >> 4], dim=2).view(rows, 2 * half)
    if code == "int4":
        v = _grouped(q.to(dtype), group)
        v = v - (8 if zero is None else zero.to(dtype)[..., None])
    else:
        v = torch.tensor(E2M1 + tuple(-x for x in E2M1), dtype=dtype, device=q.device)[q.int()]
        v = _grouped(v, group)
    return (v * scale.to(dtype)[..., None]).reshape(rows, -1)[:, : 2 * half]


# ---- the mask in plain form --------------------------------------------------------------------------------------------
def _mul32(a, m):
    """High and low 32 bits of the product of 32-bit numbers held in int64."""
    p = a * m                      # (wraps past 63 bits: the bits are right)
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _draws(seed, offset, n):
    """n numbers of 16 bits (int64)."""
    b = torch.arange((n + 7) // 8, dtype=torch.int64, device=DEV) + offset
    c0, c1 = b & 0xFFFFFFFF, (b >> 32) & 0xFFFFFFFF
    c2 = torch.zeros_like(b)
    c3 = torch.zeros_like(b)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        h0, l0 = _mul32(c0, 0xD2511F53)
        h1, l1 = _mul32(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], dim=1)
    return torch.stack([words & 0xFFFF, words >> 16], dim=2).view(-1)[:n]


def _dropped(v, case, state):
    """v (fp32) under the mask, scaled."""
    t = int(round(case["p"] * 65536))
    keep = _draws(state["seed"], state["offset"], v.numel()).view(v.shape) >= t
    return torch.where(keep, v * (65536 / (65536 - t)), torch.zeros_like(v))


# ---- inputs --------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt = TORCH_TYPE[case["dtype"]]
    kind, d_in = case["kind"], case["d_in"]

    def normal(*shape, std=1.0, dtype=dt):
        v = torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)
        return (v * std if std != 1.0 else v).to(dtype)

    s = {"case": case}
    if kind in ("dropout", "dropout_backward"):
        # the key and the place in the stream of random numbers, as a training step hands them on
        s["seed"], s["offset"] = (seed * 0x9E3779B97F4A7C15 + 1) % (1 << 63), (seed * 7919) % (1 << 40)
        s["x"] = normal(case["tokens"], d_in)
        if kind == "dropout_backward":
            s["dx"] = normal(case["tokens"], d_in)
        if own:
            _handles(case, s)
        return s
    W = normal(case["d_out"], d_in, std=d_in ** -0.5)
    if kind == "quantize":
        s["W"] = W
        if own:
            _handles(case, s)
        return s
    codes, s["scale"], s["zero"] = _quantize(W, case["code"], case["zero"], case["group"])
    s["q"] = _pack(codes)
    del W, codes
    r = case["r"]
    s["s"] = (16.0 if case["dtype"] == "f32" else 32.0) / r ** 0.5
    s["A"] = normal(r, d_in, std=d_in ** -0.5)
    s["B"] = normal(case["d_out"], r, std=BRANCH / (s["s"] * r ** 0.5))
    if kind != "norm":
        T = case["tokens"]
        W = _weight(s["q"], s["scale"], s["zero"], case["code"], case["group"])
        s["m"] = torch.linalg.vector_norm(W, dim=1) * (1 + 1e-3 * normal(case["d_out"], dtype=torch.float32))
        s["x"] = normal(T, d_in)
        if kind == "backward":
            s["dy"] = normal(T, case["d_out"])
        else:
            s["bias"] = normal(case["d_out"]) if case["bias"] else None
            # a serving program has the norm from when it loaded the adapter
            s["w_norm"] = torch.linalg.vector_norm(W.add_(s["B"].float() @ s["A"].float(), alpha=s["s"]), dim=1) if case["norm"] == "kept" else None
        del W
    if own:
        _handles(case, s)
    return s


def _handles(case, s):
    """What a program keeps between calls: descriptor, outputs, workspace."""
    from paper_2603_22276_amd import binding as D

    kind, d_in, T, r = case["kind"], case["d_in"], case.get("tokens", 0), case.get("r", 8)
    d_out, dt = case.get("d_out", 8), TORCH_TYPE[case["dtype"]]

    def out(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device=DEV)

    def scratch(phase):
        return torch.empty(D.dora_workspace_bytes(s["desc"], phase), dtype=torch.uint8, device=DEV)

    s["desc"] = D.make_desc(d_out, d_in, r, T, {"f32": D.DORA_F32, "bf16": D.DORA_BF16, "f16": D.DORA_F16}[case["dtype"]], s.get("s", 1.0))
    if kind == "dropout":
        s["x_lora"] = out(T, d_in)
    if kind == "dropout_backward":
        s["dx_sum"] = out(T, d_in)
    if "code" not in case:
        return
    code = D.QUANT_INT4 if case["code"] == "int4" else D.QUANT_FP4
    if kind == "quantize":
        groups = -(-d_in // case["group"])
        s["code"] = code
        s["q"], s["scale"] = out(d_out, d_in // 2, dtype=torch.uint8), out(d_out, groups)
        s["zero"] = out(d_out, groups) if case["zero"] else None
        s["W_out"] = out(d_out, d_in)
    s["wq"] = D.make_quant(code, case["group"], s["q"], s["scale"], s["zero"])
    if kind == "norm":
        s["c"], s["ws"] = out(d_out, dtype=torch.float32), scratch(D.PHASE_NORM_QUANT)
    if kind == "forward":
        s["y"], s["ws"] = out(T, d_out), scratch(D.PHASE_FORWARD_QUANT)
    if kind == "backward":
        s["dx"], s["ws"] = out(T, d_in), scratch(D.PHASE_BACKWARD_QUANT)
        s["dA"], s["dB"] = out(r, d_in, dtype=torch.float32), out(d_out, r, dtype=torch.float32)
        s["dm"] = None if case["frozen_m"] else out(d_out, dtype=torch.float32)


# ---- one pass ------------------------------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2603_22276_amd import binding as D

    case = s["case"]
    kind = case["kind"]
    if kind == "quantize":
        D.dora_quantize(s["desc"], s["W"], s["code"], case["group"], s["q"], s["scale"], s["zero"])
        D.dora_dequantize(s["desc"], s["wq"], s["W_out"])
        return {"W": s["W_out"], "scale": s["scale"], "zero": s["zero"]}
    if kind == "norm":
        D.dora_norm_quant(s["desc"], s["wq"], s["A"], s["B"], s["c"], s["ws"])
        return {"w_norm": s["c"]}
    if kind == "forward":
        D.dora_forward_quant(s["desc"], s["x"], None, s["wq"], s["A"], s["B"], s["m"], s["w_norm"], s["bias"], s["y"], None, None, None, s["ws"])
        return {"y": s["y"]}
    if kind == "backward":
        D.dora_backward_quant(s["desc"], s["dy"], s["x"], None, s["wq"], s["A"], s["B"], s["m"], None, None, None, s["dx"], None, s["dA"],
                              s["dB"], s["dm"], s["ws"])
        # a parameter's gradient has the parameter's type
        return {"dx": s["dx"], "dA": s["dA"].to(s["A"].dtype), "dB": s["dB"].to(s["B"].dtype), "dm": s["dm"]}
    if kind == "dropout":
        D.dora_dropout(s["desc"], s["x"], case["p"], s["seed"], s["offset"], None, s["x_lora"])
        return {"x_lora": s["x_lora"]}
    D.dora_dropout_backward(s["desc"], s["x"], case["p"], s["seed"], s["offset"], None, s["dx"], s["dx_sum"])
    return {"dx": s["dx_sum"]}


def _run_plain(s):
    case = s["case"]
    kind, dt = case["kind"], TORCH_TYPE[case["dtype"]]
    if kind == "quantize":
        q, scale, zero = _quantize(s["W"], case["code"], case["zero"], case["group"])
        return {"W": _weight(_pack(q), scale, zero, case["code"], case["group"]).to(dt), "scale": scale, "zero": zero}
    if kind == "dropout":
        return {"x_lora": _dropped(s["x"].float(), case, s).to(dt)}
    if kind == "dropout_backward":
        return {"dx": (s["dx"].float() + _dropped(s["x"].float(), case, s)).to(dt)}
    W = _weight(s["q"], s["scale"], s["zero"], case["code"], case["group"])
    A, B = s["A"].float(), s["B"].float()
    c = s.get("w_norm")
    if c is None:
        c = (W + s["s"] * (B @ A)).square().sum(1).sqrt()
    if kind == "norm":
        return {"w_norm": c}
    c = c.clamp(min=1e-12 if case["dtype"] == "f32" else 1e-6)
    g = s["m"] / c
    x = s["x"].float()
    h = x @ A.T
    if kind == "forward":
        y = g * (x @ W.T + s["s"] * (h @ B.T))
        return {"y": (y if s["bias"] is None else y + s["bias"].float()).to(dt)}
    dy = s["dy"].float()
    dm = None if case["frozen_m"] else (dy * (x @ W.T + s["s"] * (h @ B.T))).sum(0) / c
    dz = g * dy
    dh = s["s"] * (dz @ B)
    return {"dx": (dz @ W + dh @ A).to(dt), "dA": (dh.T @ x).to(dt), "dB": (s["s"] * (dz.T @ h)).to(dt), "dm": dm}


# ---- work ----------------------------------------------------------------------------------------------------------------
def work(case):
    kind, d_in = case["kind"], case["d_in"]
    e = 4 if case["dtype"] == "f32" else 2
    if kind in ("dropout", "dropout_backward"):
        n = case["tokens"] * d_in
        return {"bytes": (2 if kind == "dropout" else 3) * e * n, "flops": 2 * n}
    d_out = case["d_out"]
    packed = d_out * d_in // 2 + d_out * -(-d_in // case["group"]) * e * (2 if case["zero"] else 1)
    if kind == "quantize":   # W in, codes and scales out; the same in, W out
        return {"bytes": 2 * (e * d_out * d_in + packed), "flops": 6 * d_out * d_in}
    r = case["r"]
    weights = packed + e * (r * d_in + d_out * r)
    norm = 2 * d_out * d_in * (r + 1) + 2 * r * r * d_in + 2 * d_out * r * (r + 1)   # cross and base term, Gram matrix, B G
    if kind == "norm":
        return {"bytes": weights + 4 * d_out, "flops": norm}
    T = case["tokens"]
    big, low = 2 * T * d_out * d_in, 2 * T * r * (d_out + d_in)
    if kind == "forward":
        return {"bytes": weights + 8 * d_out + e * T * (d_in + d_out) + (e * d_out if case["bias"] else 0),
                "flops": big + low + (0 if case["norm"] == "kept" else norm)}
    # x, dy and the weights in, dx, dA, dB (and dm) out; norm and h again, and inner for dm; dz B, dz W + dh A, dh^T x, dz^T h
    grads = 4 * (r * d_in + d_out * r) + (0 if case["frozen_m"] else 4 * d_out)
    return {"bytes": weights + 4 * d_out + e * T * (2 * d_in + d_out) + grads,
            "flops": norm + big + 2 * low + (2 * T * r * d_in if case["frozen_m"] else big + low + 2 * T * d_out)}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    if kind == "quantize":
        return _exact_quantize(s["W"], case)
    if kind in ("dropout", "dropout_backward"):
        return _exact_dropout(case, s)
    # the frozen weight row by row of groups, then the adapted weight of the definition
    low, high = s["q"].long() % 16, s["q"].long() // 16
    q = torch.empty(case["d_out"], case["d_in"], dtype=torch.int64, device=DEV)
    q[:, 0::2], q[:, 1::2] = low, high
    at = torch.arange(case["d_in"], device=DEV) // case["group"]
    if case["code"] == "fp4":
        man, ex = q % 2, q // 2 % 4
        v = torch.where(ex == 0, man.double() / 2, (1 + man.double() / 2) * 2.0 ** (ex - 1).double()) * torch.where(q >= 8, -1.0, 1.0).double()
    elif case["zero"]:
        v = q.double() - s["zero"].double()[:, at]
    else:
        v = q.double() - 8
    frozen = v * s["scale"].double()[:, at]
    del q, v, low, high
    A, B, sc = s["A"].double(), s["B"].double(), s["s"]
    sc = float(torch.tensor(sc, dtype=torch.float32))       # the scaling is held in 32 bits
    full = frozen + sc * (B @ A)
    c = torch.linalg.vector_norm(full, dim=1)
    if kind == "norm":
        return {"w_norm": c}
    if s.get("w_norm") is not None:
        c = s["w_norm"].double()
    c = torch.clamp(c, min=1e-12 if case["dtype"] == "f32" else 1e-6)
    g = s["m"].double() / c
    x = s["x"].double()
    if kind == "forward":
        y = x @ (g[:, None] * full).T
        return {"y": y if s["bias"] is None else y + s["bias"].double()}
    dy = s["dy"].double()
    dfull = (dy * g).T @ x                                   # gradient of the composed weight, the norm held constant
    dm = None if case["frozen_m"] else (dy * (x @ full.T)).sum(0) / c
    return {"dx": dy @ (g[:, None] * full), "dA": sc * (B.T @ dfull), "dB": sc * (dfull @ A.T), "dm": dm}


def _exact_quantize(W, case):
    group = case["group"]
    n = -(-W.shape[1] // group)
    w = torch.zeros(W.shape[0], n * group, dtype=torch.float64, device=DEV)
    w[:, : W.shape[1]] = W.double()
    w = w.view(W.shape[0], n, group)

    def bits(v, up):
        man, ex = torch.frexp(v)                             # v = man 2^ex, man in [1/2, 1)
        man = torch.ceil(man * 16) if up else torch.round(man * 16)
        return torch.ldexp(man / 16, ex).to(W.dtype).double()   # (held in the storage type)

    if case["zero"]:
        lo, hi = torch.minimum(w.min(2).values, torch.zeros((), dtype=torch.float64, device=DEV)), torch.maximum(w.max(2).values, torch.zeros((), dtype=torch.float64, device=DEV))
        scale = bits((hi - lo) / 15, True)
        zero = torch.round(-lo / scale).clamp(0, 15)
        v = (torch.round(w / scale[..., None]) + zero[..., None]).clamp(0, 15) - zero[..., None]
    else:
        scale = bits(w.abs().max(2).values / (7 if case["code"] == "int4" else 6), False)
        zero = None
        t = w / scale[..., None]
        if case["code"] == "int4":
            v = torch.round(t).clamp(-8, 7)
        else:
            # steps of 1/2 up to 2, of 1 up to 4, of 2 up to 6
            a = t.abs()
            v = torch.where(a < 2, torch.round(2 * a) / 2, torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2))).clamp(max=6) * torch.sign(t)
    return {"W": (v * scale[..., None]).reshape(W.shape[0], -1)[:, : W.shape[1]], "scale": scale, "zero": zero}


def _exact_dropout(case, s):
    import numpy as np

    T, d_in = case["tokens"], case["d_in"]
    n = T * d_in
    mask = np.uint64(0xFFFFFFFF)
    b = np.arange(-(-n // 8), dtype=np.uint64) + np.uint64(s["offset"])
    ctr = [b & mask, b >> np.uint64(32), np.zeros_like(b), np.zeros_like(b)]
    key = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32]
    for i in range(10):
        k = [np.uint64((key[0] + i * 0x9E3779B9) % 2 ** 32), np.uint64((key[1] + i * 0xBB67AE85) % 2 ** 32)]
        p, q = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ctr = [(q >> np.uint64(32)) ^ ctr[1] ^ k[0], q & mask, (p >> np.uint64(32)) ^ ctr[3] ^ k[1], p & mask]
    u = np.stack(ctr, axis=1).astype("<u4").view("<u2").reshape(-1)[:n].astype(np.int32)
    t = round(case["p"] * 65536)
    keep = torch.from_numpy(u >= t).to(DEV).view(T, d_in)
    v = s["x"].double() * keep / (1 - t / 65536)
    return {"x_lora": v} if case["kind"] == "dropout" else {"dx": s["dx"].double() + v}
