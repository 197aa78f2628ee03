"""Dimensions whose products wrap past 64 bits are refused before anything is enqueued (no GPU needed)."""
import ctypes

import pytest

from paper_2603_22276_amd import binding as D

FAKE = 0x10000   # a 256-byte aligned, never dereferenced "device pointer"


# (d_out d_in is 0 and 64 modulo 2^64)
@pytest.mark.parametrize("d_out,d_in", [(8, 2 ** 61), (8, 2 ** 61 + 8), (2 ** 61, 8), (2 ** 61 + 8, 8), (2 ** 32, 2 ** 32)])
@pytest.mark.parametrize("dtype", [D.DORA_BF16, D.DORA_F16, D.DORA_F32])
def test_a_weight_whose_size_wraps_is_not_quantized(dtype, d_out, d_in):
    L, b = D.lib(), ctypes.byref
    d, wq = D.make_desc(d_out, d_in, 8, 0, dtype, 1.0), D.make_quant(D.QUANT_INT4, 64, FAKE, FAKE)
    assert L.dora_quantize(b(d), FAKE, D.QUANT_INT4, 64, FAKE, FAKE, None, None) == 2
    assert L.dora_dequantize(b(d), b(wq), FAKE, None) == 2


# one dimension at a time whose product with 8, 16, 64 or 512 of the others is a small number modulo 2^64
WRAPPING = [dict(d_out=2 ** 61 + 8, d_in=8, r=8), dict(d_in=2 ** 61 + 8, d_out=8, r=8), dict(r=2 ** 61 + 8, d_in=8, d_out=8, tokens=8),
            dict(tokens=2 ** 61, d_in=8, d_out=8, r=8), dict(tokens=2 ** 58 + 1), dict(tokens=2 ** 62)]


@pytest.mark.parametrize("dtype", [D.DORA_BF16, D.DORA_F16, D.DORA_F32])
@pytest.mark.parametrize("dims", WRAPPING, ids=str)
def test_a_module_whose_sizes_wrap_is_refused(dtype, dims):
    L, b, big = D.lib(), ctypes.byref, (1 << 64) - 1
    d = D.make_desc(**{**dict(d_out=64, d_in=512, r=16, tokens=64), **dims}, dtype=dtype, s=1.0)
    wq = D.make_quant(D.QUANT_INT4, 64, FAKE, FAKE)
    for phase in set(range(10)) - {D.PHASE_COMPOSE_BACKWARD}:   # (that one reads neither d_in nor r)
        assert D.dora_workspace_bytes(d, phase) == 0, phase
    assert L.dora_norm(b(d), FAKE, FAKE, FAKE, FAKE, FAKE, big, None) == 2
    assert L.dora_forward(b(d), FAKE, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, None, None, None, FAKE, big, None) == 2
    assert L.dora_backward(b(d), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, None, FAKE, FAKE, FAKE, FAKE, FAKE, big, None) == 2
    assert L.dora_norm_quant(b(d), b(wq), FAKE, FAKE, FAKE, FAKE, big, None) == 2
    assert L.dora_forward_quant(b(d), FAKE, None, b(wq), FAKE, FAKE, FAKE, None, None, FAKE, None, None, None, FAKE, big, None) == 2
    assert L.dora_backward_quant(b(d), FAKE, FAKE, None, b(wq), FAKE, FAKE, FAKE, None, None, None, FAKE, None, FAKE, FAKE, FAKE, FAKE, big, None) == 2
