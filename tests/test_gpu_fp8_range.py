"""The 8-bit norm of rows whose squares leave fp32's range: the norm is that of the formula all the same."""
import numpy as np
import pytest
import torch

import workload as wl
from tests.helpers import to_np
from tests.plain_ops import FP8, U32, blocks, check_fp8, norm_rel, rmsnorm

pytestmark = pytest.mark.gpu

af = pytest.importorskip("paper_2512_20276_amd")

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
INF, NAN = float("inf"), float("nan")


def norm(x, resid, g, eps):
    M, D = x.shape
    q = torch.empty((M, D), dtype=torch.uint8, device="cuda").view(FP8)
    s = torch.empty((M, blocks(D)), device="cuda")
    h = None if resid is None else torch.empty_like(x)
    af.op_add_rmsnorm_fp8(x, resid, g, h, q, s, eps)
    return x if h is None else h, q, s


def rows(D, scales, storage):
    x = wl.draw(("range_x", D), (len(scales), D), dtype=torch.float32).clamp_(-3.0, 3.0).double()
    x = (x * torch.tensor(scales, dtype=torch.float64)[:, None]).to(DT[storage])
    x[1::2, D // 2:] = x[1::2, D // 2:] * 2.0 ** -12  # blocks far below the row's mean
    return x.cuda()


# Against norm_rel's roundings: the reciprocal of a root mean square past 2^126 is a subnormal number of at least 22
# bits (half a step is 2 U32 at most, and so is 1 / 2 of the step that its root and the product by 2^-84 add to it): 4 U32.
@pytest.mark.parametrize("resid", [False, True])
@pytest.mark.parametrize("storage", ["bf16", "f32"])
@pytest.mark.parametrize("D", [1, 130, 256, 4096, 11008, 20001])
def test_squares_past_the_largest_number(D, storage, resid):
    scales = [1e18, 1.0, 3e19, 1e25, 3e33, 1e38, 1e17, 0.0]
    x = rows(D, scales, storage)
    g = wl.draw(("range_g", D), (D,), std=0.3, mean=1.0, dtype=DT[storage], device="cuda")
    h, q, s = norm(x * 0.25, x * 0.75, g, 1e-6) if resid else norm(x, None, g, 1e-6)
    check_fp8(q, s, rmsnorm(to_np(h), to_np(g), 1e-6), 1, norm_rel(D) + 4 * U32)


@pytest.mark.parametrize("storage", ["bf16", "f32"])
@pytest.mark.parametrize("eps", [0.0, 1e-42, 1e-34])
@pytest.mark.parametrize("D", [1, 130, 256, 4096, 11008, 20001])
def test_squares_below_the_smallest_number(D, storage, eps):
    x = rows(D, [1e-18, 1e-15, 3e-20, 1e-25, 1e-31, 1e-36, 1e-14, 1.0], storage)
    if D == 1:
        x[1::2] = x[1::2] * 2.0 ** 12
    g = wl.draw(("range_g", D), (D,), std=0.3, mean=1.0, dtype=DT[storage], device="cuda")
    h, q, s = norm(x, None, g, eps)
    check_fp8(q, s, rmsnorm(to_np(h), to_np(g), float(np.float32(eps))), 1, norm_rel(D) + 4 * U32)  # eps as it is passed


@pytest.mark.parametrize("D", [256, 4096, 11008, 20001])
def test_what_is_not_finite_stays_so(D):
    x = rows(D, [1e25, 1e25, 1e25, 1.0, 1e-30], "f32")
    x[0, 3], x[1, 5], x[3, 7] = INF, NAN, -INF
    x[4] = 0.0
    g = torch.ones(D, device="cuda")
    _, q, s = norm(x, None, g, 1e-6)
    v, s = q.float().cpu(), s.cpu()
    assert bool(v[1].isnan().all()) and bool(s[1].isnan().all())
    for r in (0, 3):  # its own block, the rest is divided by an infinite norm
        assert bool(v[r, :128].isnan().all()) and bool(s[r, 0].isnan()) and bool((v[r, 128:] == 0).all())
    assert bool((v[4] == 0).all()) and bool((s[4] == 2.0 ** -126).all())
    check_fp8(q[2:3], s[2:3], rmsnorm(to_np(x[2:3]), to_np(g), 1e-6), 1, norm_rel(D) + 4 * U32)
