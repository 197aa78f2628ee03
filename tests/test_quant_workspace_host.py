"""Scratch of forwards over a 4-bit weight (no GPU needed): those that take the codes as they are ask for no room for the weight, and no call
takes less than its phase says."""
import ctypes

import pytest

from paper_2603_22276_amd import binding as D

FAKE = 0x10000   # a 256-byte aligned, never dereferenced "device pointer"
PLAIN, GIVEN, ANY = D.PHASE_FORWARD_QUANT_PLAIN, D.PHASE_FORWARD_QUANT_NORM_GIVEN, D.PHASE_FORWARD_QUANT


def desc(**kw):
    return D.make_desc(**{**dict(d_out=8192, d_in=8192, r=384, tokens=1, dtype=D.DORA_BF16, s=1.0), **kw})


CASES = [  # the desc, whether the weight is read back with the norm formed in the call, and with the norm given
    (dict(), False, False), (dict(tokens=32), False, False), (dict(tokens=0), False, False), (dict(dtype=D.DORA_F16, tokens=17), False, False),
    (dict(r=392), True, False), (dict(d_in=8200), True, False), (dict(s=0.0), True, False), (dict(s=0.0, tokens=0), True, False),
    (dict(tokens=33), True, True), (dict(tokens=2000), True, True), (dict(dtype=D.DORA_F32), True, True), (dict(dtype=D.DORA_F32, tokens=0), True, False),
]


@pytest.mark.parametrize("dims,with_norm,without", CASES, ids=str)
def test_room_for_the_weight(dims, with_norm, without):
    d = desc(**dims)
    weight = d.d_out * d.d_in * (4 if d.dtype == D.DORA_F32 else 2)
    for phase, reads in ((PLAIN, with_norm), (GIVEN, without)):
        n, all_of_it = D.dora_workspace_bytes(d, phase), D.dora_workspace_bytes(d, ANY)
        assert 0 < n <= all_of_it
        # beside the weight stand h, s h, lora and K slices of [tokens, d_out] at most, and the norm's sums
        assert weight <= n if reads else n < weight // 8
    assert D.dora_workspace_bytes(d, GIVEN) <= D.dora_workspace_bytes(d, PLAIN)


@pytest.mark.parametrize("dims,with_norm,without", CASES, ids=str)
def test_less_is_refused(dims, with_norm, without):
    L, b, d = D.lib(), ctypes.byref, desc(**dims)
    wq = D.make_quant(D.QUANT_INT4, 2 ** 20, FAKE, FAKE)    # (one group to a row: none of the tiles that decode)
    for phase, w_norm in ((PLAIN, None), (GIVEN, FAKE)):
        n = D.dora_workspace_bytes(d, phase)
        assert L.dora_forward_quant(b(d), FAKE, None, b(wq), FAKE, FAKE, FAKE, w_norm, None, FAKE, None, None, None, FAKE, n - 1, None) == 5
        assert L.dora_forward_quant(b(d), FAKE, FAKE, b(wq), FAKE, FAKE, FAKE, w_norm, None, FAKE, None, None, None, FAKE, n - 1, None) == 5


def test_a_desc_that_no_forward_takes_has_none():
    for phase in (PLAIN, GIVEN):
        for bad in (desc(d_in=8196, dtype=D.DORA_F32), desc(d_out=8196), desc(tokens=-1), desc(dtype=7)):
            assert D.dora_workspace_bytes(bad, phase) == 0
