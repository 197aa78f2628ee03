"""4-bit frozen weights and the drawn dropout mask on the CPU: what pins the oracle, and what the entry points refuse before
anything is enqueued."""
import ctypes

import numpy as np
import pytest

from oracle import quant_oracle as Q
from paper_2603_22276_amd import binding as D

FAKE = 0x10000   # a 256-byte aligned, never dereferenced "device pointer"


def desc(**kw):
    base = dict(d_out=256, d_in=512, r=16, tokens=64, dtype=D.DORA_BF16, s=4.0)
    base.update(kw)
    return D.make_desc(**base)


def quant(code=D.QUANT_INT4, group=64, q=FAKE, scale=FAKE, zero=None):
    return D.make_quant(code, group, q, scale, zero)


# ---- the oracle ----------------------------------------------------------------------------------------------------------
def test_philox_known_answers():
    # the published test vectors of Philox 4x32-10
    assert Q.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert Q.philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_four_significant_bits():
    assert Q.four_bits(np.array([1.0, 1.0625, 1.1875, 15.5, 16.5, 0.0])).tolist() == [1.0, 1.0, 1.25, 16.0, 16.0, 0.0]
    assert Q.four_bits(np.array([1.0, 1.0001, 15.0, 15.1]), up=True).tolist() == [1.0, 1.125, 15.0, 16.0]


@pytest.mark.parametrize("code,zero", [("int4", False), ("int4", True), ("fp4", False)])
def test_quantized_weight_is_within_half_a_step_and_a_bf16_number(code, zero):
    rng = np.random.default_rng(5)
    W = (rng.standard_normal((40, 200)) + (0.7 if zero else 0.0)).astype(np.float32).astype(np.float64)
    q, scale, z = Q.quantize(W, code, zero, 64)
    back = Q.weight(q, scale, z, code, 64)
    at = np.arange(200) // 64
    # the widest gap between E2M1 values is 2; the largest magnitude lies at most 6 (1 + 1/16) steps out
    assert np.all(np.abs(back - W) <= (1.0 if code == "fp4" else 0.5) * scale[:, at] * (1 + 1e-12))
    bits = back.astype(np.float32).view(np.uint32)
    assert np.all(bits & 0xFFFF == 0) and np.array_equal(bits.view(np.float32).astype(np.float64), back)


def test_quantize_by_hand():
    W = np.array([[-7.0, 3.5, 0.49, 2.5, 0.0, 1.5, -0.5, 7.0]])
    q, scale, _ = Q.quantize(W, "int4", False, 32)
    assert scale.tolist() == [[1.0]] and (q.astype(int) - 8).tolist() == [[-7, 4, 0, 2, 0, 2, 0, 7]]
    q, scale, zero = Q.quantize(np.array([[-3.0, 12.0, 0.0, 5.0]]), "int4", True, 32)
    assert scale.tolist() == [[1.0]] and zero.tolist() == [[3.0]] and q.tolist() == [[0, 15, 3, 8]]
    q, scale, _ = Q.quantize(np.array([[-6.0, 2.5, 3.5, 5.0, 0.25, -0.75]]), "fp4", False, 32)
    assert scale.tolist() == [[1.0]] and Q.E2M1[q].tolist() == [[-6.0, 2.0, 4.0, 4.0, 0.0, -1.0]]


def test_mask_of_later_rows_and_its_share():
    whole = Q.keep(11, 2 ** 33, 4096, 0.25)
    assert np.array_equal(Q.keep(11, 2 ** 33 + 64, 4096 - 512, 0.25), whole[512:])
    assert abs(whole.mean() - 0.75) < 5 * np.sqrt(0.25 * 0.75 / 4096)
    assert Q.keep(1, 0, 64, 0.0).all() and not Q.keep(1, 0, 64, 65535 / 65536).any()


# ---- refusals ------------------------------------------------------------------------------------------------------------
def calls(d, wq, big=1 << 40):
    L, b = D.lib(), ctypes.byref
    w = b(wq) if wq is not None else None
    return {
        "dora_dequantize": lambda: L.dora_dequantize(b(d), w, FAKE, None),
        "dora_norm_quant": lambda: L.dora_norm_quant(b(d), w, FAKE, FAKE, FAKE, FAKE, big, None),
        "dora_forward_quant": lambda: L.dora_forward_quant(b(d), FAKE, None, w, FAKE, FAKE, FAKE, None, None, FAKE, None, None, None, FAKE, big, None),
        "dora_backward_quant": lambda: L.dora_backward_quant(b(d), FAKE, FAKE, None, w, FAKE, FAKE, FAKE, None, None, None, FAKE, None, FAKE, FAKE,
                                                             FAKE, FAKE, big, None),
    }


BAD = [  # what is wrong, status
    (dict(), dict(code=2), 2), (dict(), dict(code=-1), 2), (dict(), dict(group=16), 2), (dict(), dict(group=96), 2), (dict(), dict(group=0), 2),
    (dict(), dict(group=-64), 2), (dict(), dict(group=-2 ** 31), 2), (dict(), dict(code=D.QUANT_FP4, zero=FAKE), 2), (dict(), dict(q=None), 1),
    (dict(), dict(scale=None), 1), (dict(), dict(q=FAKE + 4), 3), (dict(), dict(scale=FAKE + 2), 3), (dict(), dict(zero=FAKE + 8), 3),
    (dict(d_in=516, dtype=D.DORA_F32), dict(), 2), (dict(d_in=508), dict(), 2), (dict(d_in=0), dict(), 2), (dict(dtype=3), dict(), 4),
    (dict(d_out=65536, d_in=32768), dict(), 2),
]


@pytest.mark.parametrize("dkw,qkw,status", BAD)
def test_bad_quant_is_refused(dkw, qkw, status):
    for name, call in calls(desc(**dkw), quant(**qkw)).items():
        assert call() == status, name


def test_null_quant_and_small_workspace_are_refused():
    for name, call in calls(desc(), None).items():
        assert call() == 1, name
    for name, call in calls(desc(), quant(), big=255).items():
        if name != "dora_dequantize":   # (it takes no workspace)
            assert call() == 5, name
    L, b = D.lib(), ctypes.byref
    # a rank whose Gram matrix cannot be an operand
    d, wq = desc(d_out=8, d_in=8, r=46344, tokens=0), quant()
    assert L.dora_norm_quant(b(d), b(wq), FAKE, FAKE, FAKE, FAKE, 1 << 50, None) == 2
    assert L.dora_forward_quant(b(d), FAKE, None, b(wq), FAKE, FAKE, FAKE, None, None, FAKE, None, None, None, FAKE, 1 << 50, None) == 2
    assert L.dora_backward_quant(b(d), FAKE, FAKE, None, b(wq), FAKE, FAKE, FAKE, None, None, None, FAKE, None, FAKE, FAKE, FAKE, FAKE,
                                 1 << 50, None) == 2


def test_quantize_refusals():
    L, b = D.lib(), ctypes.byref
    d = desc()
    assert L.dora_quantize(b(d), FAKE, 5, 64, FAKE, FAKE, None, None) == 2
    assert L.dora_quantize(b(d), FAKE, 0, 48, FAKE, FAKE, None, None) == 2
    assert L.dora_quantize(b(d), FAKE, 1, 64, FAKE, FAKE, FAKE, None) == 2
    assert L.dora_quantize(b(d), None, 0, 64, FAKE, FAKE, None, None) == 1
    assert L.dora_quantize(b(d), FAKE, 0, 64, None, FAKE, None, None) == 1
    assert L.dora_quantize(b(d), FAKE, 0, 64, FAKE, None, None, None) == 1
    assert L.dora_quantize(b(d), FAKE + 8, 0, 64, FAKE, FAKE, None, None) == 3
    assert L.dora_quantize(None, FAKE, 0, 64, FAKE, FAKE, None, None) == 1


def test_dropout_refusals():
    L, b = D.lib(), ctypes.byref
    for p, st in ((1.0, 2), (-0.1, 2), (float("nan"), 2), (1.5, 2), (float("inf"), 2)):
        assert L.dora_dropout(b(desc()), FAKE, p, 1, 0, None, FAKE, None) == st
        assert L.dora_dropout_backward(b(desc()), FAKE, p, 1, 0, None, None, FAKE, None) == st
    assert L.dora_dropout(b(desc()), None, 0.1, 1, 0, None, FAKE, None) == 1
    assert L.dora_dropout(b(desc()), FAKE, 0.1, 1, 0, None, None, None) == 1
    assert L.dora_dropout(b(desc()), FAKE + 8, 0.1, 1, 0, None, FAKE, None) == 3
    assert L.dora_dropout(b(desc()), FAKE, 0.1, 1, 0, FAKE + 4, FAKE, None) == 3
    assert L.dora_dropout_backward(b(desc()), FAKE, 0.1, 1, 0, None, FAKE + 8, FAKE, None) == 3
    assert L.dora_dropout(b(desc(d_in=516)), FAKE, 0.1, 1, 0, None, FAKE, None) == 2
    assert L.dora_dropout(b(desc(tokens=2 ** 40)), FAKE, 0.1, 1, 0, None, FAKE, None) == 2
    assert L.dora_dropout(b(desc(tokens=-1)), FAKE, 0.1, 1, 0, None, FAKE, None) == 2
    assert L.dora_dropout(b(desc(dtype=9)), FAKE, 0.1, 1, 0, None, FAKE, None) == 4
    assert L.dora_dropout(b(desc(tokens=0)), None, 0.1, 1, 0, None, None, None) == 0


def test_workspaces_of_a_quantized_module():
    for dtype, e in ((D.DORA_BF16, 2), (D.DORA_F16, 2), (D.DORA_F32, 4)):
        d = desc(d_out=1000, d_in=2056, r=40, tokens=300, dtype=dtype)
        w = -(-1000 * 2056 * e // 256) * 256
        for phase, plain in ((D.PHASE_NORM_QUANT, D.PHASE_NORM), (D.PHASE_FORWARD_QUANT, D.PHASE_FORWARD_DROPOUT),
                             (D.PHASE_BACKWARD_QUANT, D.PHASE_BACKWARD_DROPOUT)):
            assert D.dora_workspace_bytes(d, phase) >= D.dora_workspace_bytes(d, plain) + w
    assert D.dora_workspace_bytes(desc(d_in=516, dtype=D.DORA_F32), D.PHASE_FORWARD_QUANT) == 0
