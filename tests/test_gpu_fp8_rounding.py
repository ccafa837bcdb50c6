"""The 8-bit form bit for bit: v over the scale, rounded to fp32 and then to the nearest e4m3 value, ties to even.
bf16 elements over a bf16 maximum often lie midway between two e4m3 values."""
import pytest
import torch

import workload as wl
from tests.plain_ops import FP8, blocks

pytestmark = pytest.mark.gpu

af = pytest.importorskip("paper_2512_20276_amd")

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def eight_bits(v, block_rows):
    """(codes, scales) of an fp32 CPU matrix of whole blocks of columns, with fp32 divisions."""
    M, K = v.shape
    full = torch.zeros(-(-M // block_rows) * block_rows, K)
    full[:M] = v
    t = full.view(-1, block_rows, K // 128, 128)
    s = (t.abs().amax(dim=(1, 3)) / 448.0).clamp_min(2.0 ** -126)
    q = (t / s[:, None, :, None]).reshape(full.shape)[:M]
    return q.to(FP8).view(torch.uint8), s


@pytest.mark.parametrize("storage", ["bf16", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("M,K", [(1, 128), (37, 4096), (300, 1152)])
def test_codes_are_those_of_the_division(storage, block_rows, M, K):
    x = wl.draw(("r8_x", M, K), (M, K), dtype=DT[storage], device="cuda")
    # blocks of every magnitude, subnormal ones among them, and zeros of either sign
    at = torch.arange(M)[:, None] // block_rows * 5 + torch.arange(K)[None, :] // 128
    e = torch.tensor([0, 0, -6, 40, -80, -93, -100, -118, -124, -130, -140, 110])[at % 12].double()
    x = (x.double().cpu() * torch.pow(2.0, e)).to(DT[storage])
    x[:, 3::17] = 0.0
    x[:, 5::17] = -0.0
    want_q, want_s = eight_bits(x.float(), block_rows)
    q = torch.empty((M, K), dtype=torch.uint8, device="cuda")
    s = torch.empty(want_s.shape, device="cuda")
    af.op_quantize_fp8(x.cuda(), q.view(FP8), s, block_rows)
    assert torch.equal(s.cpu(), want_s)
    assert torch.equal(q.cpu(), want_q), int((q.cpu() != want_q).sum())


@pytest.mark.parametrize("storage", ["bf16", "f32"])
@pytest.mark.parametrize("M,D", [(9, 256), (5, 4096), (3, 8192), (2, 16384)])
def test_codes_of_a_norm_are_those_of_the_division(storage, M, D):
    """Whole numbers of up to 8 whose mean square and eps add up to 64: the norm is h g / 8, exactly."""
    gen = torch.Generator().manual_seed(D)
    row = torch.randint(-8, 9, (D,), generator=gen).float()
    x = torch.stack([row[torch.randperm(D, generator=gen)] for _ in range(M)])
    eps = 64.0 - float((row * row).mean())  # a multiple of 1 / D
    g = wl.draw(("r8_g", D), (D,), std=0.3, mean=1.0, dtype=torch.bfloat16).float()
    want_q, want_s = eight_bits(x / 8 * g, 1)
    q = torch.empty((M, D), dtype=torch.uint8, device="cuda")
    s = torch.empty((M, blocks(D)), device="cuda")
    af.op_add_rmsnorm_fp8(x.to(DT[storage]).cuda(), None, g.to(DT[storage]).cuda(), None, q.view(FP8), s, eps)
    assert torch.equal(s.cpu(), want_s)
    assert torch.equal(q.cpu(), want_q), int((q.cpu() != want_q).sum())


@pytest.mark.parametrize("exponent", [0, -60, -112, 100])
def test_quotients_next_to_the_middle_between_two_values(exponent):
    """Elements within two ulps of the scale times a midpoint, over scales of any significand, the last one before a
    power of two among them (a maximum of 896 - 2^-14)."""
    gen = torch.Generator().manual_seed(exponent + 200)
    M = 600
    top = torch.rand(M, generator=gen) * 448 + 448
    top[::7] = 896.0 - 2.0 ** -14
    s = top / 448.0
    codes = torch.arange(0, 127, dtype=torch.uint8).view(FP8).double()
    mid = (codes[1:] + codes[:-1]) / 2
    x = (s.double()[:, None] * mid[torch.randint(0, 126, (M, 128), generator=gen)]).float()
    step = torch.randint(-2, 3, (M, 128), generator=gen, dtype=torch.int32)
    x = (x.view(torch.int32) + step).view(torch.float32).minimum(top[:, None])
    x[:, 17] = top
    x[:, ::2] *= -1.0
    x[::7, 20:60] = torch.pow(2.0, torch.arange(40) - 33.0)  # quotients one step above a power of two
    x = x * 2.0 ** exponent
    want_q, want_s = eight_bits(x, 1)
    q, got_s = torch.empty((M, 128), dtype=torch.uint8, device="cuda"), torch.empty((M, 1), device="cuda")
    af.op_quantize_fp8(x.cuda(), q.view(FP8), got_s)
    assert torch.equal(got_s.cpu(), want_s)
    assert torch.equal(q.cpu(), want_q), int((q.cpu() != want_q).sum())
