"""dora_quantize where weights come near the largest number of their type: scales, zero points and codes against the oracle, and what
is read back is finite."""
import numpy as np
import pytest

import quant_util as U
from oracle import quant_oracle as Q
from test_gpu_quant import KINDS, quantize_on_gpu

pytestmark = pytest.mark.gpu

LARGEST = {"bf16": (2.0 - 2.0 ** -7) * 2.0 ** 127, "f16": 65504.0, "f32": (2.0 - 2.0 ** -23) * 2.0 ** 127}


def check(W, dtype, kind, group, largest):
    code = "fp4" if kind == "fp4" else "int4"
    q, scale, zero = Q.quantize(W, code, kind == "zero", group, lambda v: U.stored(v, dtype), largest)
    want = Q.weight(q, scale, zero, code, group)
    assert np.all(np.abs(want) <= LARGEST[dtype])           # (the oracle's own)
    got_q, got_scale, got_zero, back = quantize_on_gpu(W, dtype, kind, group)
    assert np.array_equal(got_scale, scale)
    assert zero is None or np.array_equal(got_zero, zero)
    assert np.array_equal(Q.weight(got_q, scale, zero, code, group), want)
    assert np.all(np.abs(back - want) <= U.HALF_STEP[dtype] * np.abs(want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [32, 1024])
def test_a_span_past_the_largest_float(dtype, group):
    # (weights of 16 bits in either type: the span is a sum of few bits, exact where it does not overflow)
    W = U.stored(np.random.default_rng(3).uniform(-2, 2, (8, 1024)) * 2.0 ** 126, "bf16")
    top = U.stored(3e38, "bf16")
    W[0, ::32], W[0, 1::32] = -top, top
    W[1] = 0.0
    W[1, 5] = 2.0 ** 126                                    # (no overflow)
    W[2, ::32], W[2, 7::32] = -2.0 ** 127, 2.0 ** 127       # (the span is 2^128)
    W[3] = U.stored(np.random.default_rng(4).standard_normal(1024), "bf16")
    check(W, dtype, "zero", group, np.inf)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("group", [32, 1024])
def test_the_largest_weights_read_back_finite(dtype, kind, group):
    # (16-bit weights in fp32 too, as above; beside them the largest float itself)
    M = LARGEST["bf16" if dtype == "f32" else dtype]
    stored = lambda a: U.stored(a, "bf16" if dtype == "f32" else dtype)  # noqa: E731
    W = stored(np.random.default_rng(5).uniform(-1, 1, (16, 1024)) * M)
    W[0], W[1] = M, -M
    W[2, ::32], W[2, 1::32] = -M, M
    W[3:8] = stored(np.random.default_rng(6).uniform(0, 1, (5, 1024)) * M)
    for row, share in zip(range(3, 8), (0.05, 0.1, 0.15, 0.2, 0.3)):
        W[row, ::32], W[row, 1::32] = M, stored(-share * M)
        W[row + 5] = -W[row]
    W[13, 4:] = 0.0
    if dtype == "f32":
        W[14] = LARGEST["f32"]
    check(W, dtype, kind, group, LARGEST[dtype])
