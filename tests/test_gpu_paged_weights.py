"""GPU tests of the weights with which attention over a paged cache takes its values: how many bits they are held in."""
import copy
import math

import pytest
import torch

from tests.paged_plain import HALF_STEP, Step, inside

pytestmark = pytest.mark.gpu

af = pytest.importorskip("paper_2512_20276_amd")

BF16 = torch.bfloat16


def attend(s: Step, window=0, sinks=0):
    kv = s.to_gpu(af)
    o = torch.full((s.M, s.Hq, s.hd), 7.0, dtype=s.dtype, device="cuda")
    workspace = torch.full((af.attention_paged_workspace(kv, s.M, s.Hq),), 255, dtype=torch.uint8, device="cuda")
    af.op_attention_paged(kv, s.g["q"], o, 1.0 / math.sqrt(s.hd), workspace, window, sinks)
    return o


def held_to_16_bits(s: Step, window, sinks):
    """(o, its bound) in 64 bits, where a weight of any row is held to 2^-16, as those of single rows are.

    ``attended`` gives r = sum of w v and a bound e + h (|r| + e), h half a step, e = (2 worst + held) sum of w |v| with a held of
    2^-8 for bf16 rows beside others; the sum of w |v| is what it gives for the values' magnitudes.  A weight is a bf16 number cut to
    8 bits and the rest of it, below 2^-7 of the power of two under the weight, to half of its step: 2^-16 of the weight at
    most.  The rest is taken of the weight times 1 + 2^-23, 2^-23 more of it, which the additions counted in ``worst``
    cover: n for n terms, in the numerator and in the denominator, are one more than there are, 2^-24 each."""
    scale = 1.0 / math.sqrt(s.hd)
    r, bound, _, _ = s.attended(scale, window, sinks)
    t = copy.copy(s)
    t.v_cache = s.v_cache.abs()
    total = t.attended(scale, window, sinks)[0]
    h = HALF_STEP[s.dtype]
    several = torch.zeros(s.M, 1, 1, dtype=torch.float64)
    for row, b, _ in s.rows():
        several[row] = s.requests[b][0] > 1
    err = (bound - h * r.abs()) / (1 + h) - several * (2.0 ** -8 - 2.0 ** -16) * total
    return r, err + h * (r.abs() + err)


@pytest.mark.parametrize("hd,Hkv,group,page", [(128, 2, 4, 16), (64, 2, 2, 8)])
@pytest.mark.parametrize("requests,window,sinks", [
    ([(2, 2), (3, 40), (1, 30)], 0, 0),
    ([(150, 150), (70, 400), (3, 90)], 0, 0),
    ([(150, 150), (70, 400), (3, 90)], 50, 4),
    ([(40, 3000), (1, 2500), (3, 700)], 0, 0),  # split over the keys
])
def test_rows_beside_others_hold_their_weights_as_single_rows_do(hd, Hkv, group, page, requests, window, sinks):
    s = Step(requests, Hkv, group, hd, page, BF16)
    inside(attend(s, window, sinks), *held_to_16_bits(s, window, sinks))


def test_a_row_is_as_exact_beside_another_as_alone():
    """The last row of a chunk of two, and the same row in a step of its own."""
    s = Step([(2, 300)], 2, 4, 128, 16, BF16)
    t = Step([(1, 300)], 2, 4, 128, 16, BF16, single=True)
    t.k_cache, t.v_cache, t.table, t.q = s.k_cache, s.v_cache, s.table, s.q[1:]
    r, bound = held_to_16_bits(t, 0, 0)
    inside(attend(t), r, bound)
    inside(attend(s)[1:], r, bound)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("hd,Hkv,group,page", [(128, 2, 4, 16), (64, 1, 17, 8)])
@pytest.mark.parametrize("requests,single", [
    ([(1, 41), (1, 64), (1, 1)], True),
    ([(1, 700), (1, 64), (1, 2500)], True),  # split over the keys
    ([(70, 100), (1, 64), (2, 130)], False),
    ([(20, 700), (1, 2500), (3, 64)], False),  # split
])
def test_infinite_values_that_are_seen(dtype, hd, Hkv, group, page, requests, single):
    """softmax . V gives the infinity to the rows that see it, NaN where both are seen, and to other dimensions what they had."""
    for window in (0, 30):
        s = Step(requests, Hkv, group, hd, page, dtype, single)
        for b, (n, length) in enumerate(requests):
            for j, d, worst in ((0, 0, math.inf), (length // 2, 5, -math.inf), (length - 1, 33, math.inf), (length - 1, 40, -math.inf),
                                (max(length - 3, 0), 41, math.inf), (length - 1, 41, -math.inf)):
                page_of, at = s.cell(b, j)
                s.v_cache[page_of, :, at, d] = worst
        got = attend(s, window)
        want, bound, _, _ = s.attended(1.0 / math.sqrt(hd), window)
        inside(got, want, bound, window)
        mine = [row for row, _, _ in s.rows()]
        assert torch.equal(got.cpu()[mine].isnan(), want[mine].isnan()), window
