"""The drawn dropout mask: every decision against the oracle's Philox, values to the rounding of the storage type, the way back,
places in the stream, and what is dropped staying out of the result."""
import numpy as np
import pytest
import torch

import gpu_util as G
from oracle import quant_oracle as Q
from paper_2603_22276_amd import binding as D
from paper_2603_22276_amd import inputs as I

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}   # relative
# fp16 below 2^-14 has steps of 2^-24, so half a step is 2^-25 there whatever the value
SMALLEST_HALF_STEP = {"bf16": 0.0, "f16": 2.0 ** -25, "f32": 0.0}


def desc(tokens, d_in, dtype):
    return D.make_desc(8, d_in, 8, tokens, G.dtype_code(dtype), 1.0)


def draw(shape, dtype, seed):
    a = I.quantise(np.random.default_rng(seed).standard_normal(shape), dtype)
    return G.to_dev(a), I.to_f64(a)


def call(x, p, seed, offset, dtype, counter=None, dx=None, backward=False):
    out = G.empty(tuple(x.shape), dtype)
    d = desc(x.shape[0], x.shape[1], dtype)
    if backward:
        D.dora_dropout_backward(d, x, p, seed, offset, counter, dx, out)
    else:
        D.dora_dropout(d, x, p, seed, offset, counter, out)
    return out


CASES = [  # tokens, d_in, p, seed, offset
    (1, 8, 0.5, 0, 0), (3, 40, 0.1, 1, 7), (17, 264, 0.25, 2 ** 63 + 5, 2 ** 32 - 3), (1, 2056, 0.9, 12345678901234567, 2 ** 64 - 2),
    (5, 72, 0.0, 3, 0), (4, 64, 0.999999, 9, 1), (129, 128, 1 / 3, 77, 2 ** 40),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,d_in,p,seed,offset", CASES + [(3, 12, 0.4, 5, 6), (1, 4, 0.5, 8, 0)])
def test_forward_and_backward(dtype, tokens, d_in, p, seed, offset):
    if dtype != "f32" and d_in % 8:
        d_in += 4
    x, x64 = draw((tokens, d_in), dtype, 1)
    want = Q.dropout(x64, seed, offset, p)
    got = G.to_f64(call(x, p, seed, offset, dtype))
    t = min(65535, int(np.rint(p * 65536)))
    if dtype != "f16" or t < 65000:                        # (fp16: 65536 times a value is an infinity)
        # one rounding to fp32 of the scale, one of the product, one to the storage type
        assert np.all(np.abs(got - want) <= (HALF_STEP[dtype] + 2 * 2.0 ** -24) * np.abs(want) + SMALLEST_HALF_STEP[dtype])
    assert np.array_equal(got != 0, want != 0)
    dx, dx64 = draw((tokens, d_in), dtype, 2)
    back = G.to_f64(call(x, p, seed, offset, dtype, dx=dx, backward=True))
    if dtype != "f16" or t < 65000:
        assert np.all(np.abs(back - (dx64 + want)) <= HALF_STEP[dtype] * np.abs(dx64 + want) + 3 * 2.0 ** -24 * (np.abs(dx64) + np.abs(want)) +
                      SMALLEST_HALF_STEP[dtype])
    alone = call(x, p, seed, offset, dtype, backward=True)   # dx == NULL counts as 0
    assert torch.equal(alone, call(x, p, seed, offset, dtype))


def test_gradient_against_differences():
    # the map is linear: a step of one element moves the output by that element's factor and nothing else
    x, _ = draw((3, 16), "f32", 4)
    one = torch.zeros_like(x)
    base = call(x, 0.4, 5, 6, "f32")
    factor = call(torch.ones_like(x), 0.4, 5, 6, "f32", backward=True)
    for at in ((0, 0), (1, 7), (2, 15)):
        one.zero_()
        one[at] = 4.0
        moved = call(x + one, 0.4, 5, 6, "f32") - base
        assert abs(moved[at].item() / 4.0 - factor[at].item()) <= 1e-5
        moved[at] = 0.0
        assert not moved.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_a_batch_by_offset_and_by_counter(dtype):
    x, _ = draw((48, 200), dtype, 5)
    whole = call(x, 0.3, 99, 2 ** 33, dtype)
    assert torch.equal(whole[16:], call(x[16:].contiguous(), 0.3, 99, 2 ** 33 + 16 * 200 // 8, dtype))
    counter = torch.tensor([2 ** 33 - 11], dtype=torch.int64, device=G.DEV)
    assert torch.equal(whole, call(x, 0.3, 99, 11, dtype, counter=counter))


def test_the_mask_is_that_of_every_dtype():
    ones = torch.ones((33, 264), device=G.DEV)
    masks = [call(ones.to(t), 0.2, 4, 5, n) != 0 for t, n in ((torch.float32, "f32"), (torch.bfloat16, "bf16"), (torch.float16, "f16"))]
    assert torch.equal(masks[0], masks[1]) and torch.equal(masks[0], masks[2])


def test_in_place_and_what_is_dropped_stays_out():
    x, _ = draw((40, 136), "bf16", 6)
    want = call(x, 0.5, 1, 2, "bf16")
    dropped = want == 0
    x[dropped] = float("nan")
    y = x.clone()
    D.dora_dropout(desc(40, 136, "bf16"), y, 0.5, 1, 2, None, y)
    assert torch.equal(y, want)
    dx, _ = draw((40, 136), "bf16", 7)
    sum1 = call(x, 0.5, 1, 2, "bf16", dx=dx, backward=True)
    over_dx, over_dxl = dx.clone(), x.clone()
    D.dora_dropout_backward(desc(40, 136, "bf16"), x, 0.5, 1, 2, None, over_dx, over_dx)
    D.dora_dropout_backward(desc(40, 136, "bf16"), over_dxl, 0.5, 1, 2, None, dx, over_dxl)
    assert torch.equal(sum1, over_dx) and torch.equal(sum1, over_dxl)
    assert torch.equal(sum1[dropped], dx[dropped])


def test_rows_behind_the_last_token_stay():
    for dtype, d_in in (("bf16", 40), ("f32", 12)):
        x, _ = draw((3, d_in), dtype, 8)
        out = G.empty((5, d_in), dtype)
        D.dora_dropout(desc(3, d_in, dtype), x, 0.1, 1, 0, None, out)
        assert torch.isnan(out[3:]).all() and not torch.isnan(out[:3]).any()


def test_large_batch_draws_to_its_last_block():
    # 2^27 elements and a ragged rest: the places near the end against the oracle
    tokens, d_in = 65537, 2056
    x = torch.ones((tokens, d_in), dtype=torch.bfloat16, device=G.DEV)
    out = call(x, 0.25, 21, 2 ** 45, "bf16").view(-1)
    n = tokens * d_in
    for first in (0, 2 ** 26, n - 4096):
        first -= first % 8
        want = Q.keep(21, 2 ** 45 + first // 8, min(4096, n - first), 0.25)
        assert np.array_equal((out[first:first + want.size] != 0).cpu().numpy(), want)
    # five standard deviations of the share kept
    assert abs((out != 0).float().mean().item() - 0.75) < 5 * (0.25 * 0.75 / n) ** 0.5 + 2 ** -17


def test_captured_with_a_counter_on_the_device_draws_anew():
    x, _ = draw((24, 72), "bf16", 9)
    counter = torch.zeros(1, dtype=torch.int64, device=G.DEV)
    out = G.empty((24, 72), "bf16")
    d = desc(24, 72, "bf16")
    D.dora_dropout(d, x, 0.5, 3, 0, counter, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.dora_dropout(d, x, 0.5, 3, 0, counter, out)
        counter += 24 * 72 // 8
    counter.zero_()
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call(x, 0.5, 3, i * 24 * 72 // 8, "bf16"))
