"""GPU parity of the 8-bit norm, quantisation and projection with their plain 64-bit forms."""
import numpy as np
import pytest
import torch

import workload as wl
from tests.helpers import to_np
from tests.plain_ops import FP8, U32, blocks, check_fp8, linear_fp8, norm_rel, rmsnorm

pytestmark = pytest.mark.gpu

af = pytest.importorskip("paper_2512_20276_amd")

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NORM_SHAPES = [(1, 1), (2, 7), (3, 127), (5, 128), (4, 129), (34, 256), (7, 513), (1, 4096), (33, 4096), (282, 4096),
               (1024, 4096), (1031, 520), (2264, 4096), (9, 4104), (3, 11008), (2, 12287), (2, 20001)]


def outputs(M, K, mb=None):
    """q and scales with a row of canaries behind them."""
    q = torch.full((M + 1, K), 3, dtype=torch.uint8, device="cuda")
    s = torch.full(((M if mb is None else mb) + 1, blocks(K)), -7.0, device="cuda")
    return q, s


def untouched(q, s):
    return bool((q[-1] == 3).all()) and bool((s[-1] == -7.0).all())


# ----------------------------------------------------------------------------- norm
def run_norm(x, r, g, eps=1e-6, out=None):
    M, D = x.shape
    q, s = outputs(M, D)
    h = None if r is None else (torch.empty_like(x) if out is None else out)
    af.op_add_rmsnorm_fp8(x, r, g, h, q[:M].view(FP8), s[:M], eps)
    torch.cuda.synchronize()
    assert untouched(q, s)
    return h, q[:M].view(FP8), s[:M]


@pytest.mark.parametrize("storage", ["bf16", "f32"])
@pytest.mark.parametrize("M,D", NORM_SHAPES)
def test_add_rmsnorm_fp8(storage, M, D):
    dt = DT[storage]
    x = wl.draw(("f8_x", M, D), (M, D), std=0.5, dtype=dt, device="cuda")
    r = wl.draw(("f8_r", M, D), (M, D), dtype=dt, device="cuda")
    g = wl.draw(("f8_g", D), (D,), std=0.3, mean=1.0, dtype=dt, device="cuda")
    h, q, s = run_norm(x, r, g)
    assert torch.equal(h.cpu(), (x.cpu().float() + r.cpu().float()).to(dt))  # one fp32 sum, rounded as stored
    check_fp8(q, s, rmsnorm(to_np(h), to_np(g), 1e-6), 1, norm_rel(D))
    _, q0, s0 = run_norm(h, None, g)  # the norm alone, of the same rows
    assert torch.equal(q0.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s0, s)


@pytest.mark.parametrize("M,D", [(1031, 4096), (1100, 264), (3, 9000)])
def test_a_row_does_not_depend_on_the_others(M, D):
    x = wl.draw(("f8_x", M, D), (M, D), device="cuda")
    r = wl.draw(("f8_r", M, D), (M, D), device="cuda")
    g = wl.draw(("f8_g", D), (D,), std=0.3, mean=1.0, device="cuda")
    h, q, s = run_norm(x, r, g)
    for m in (0, M // 2, M - 1):
        h1, q1, s1 = run_norm(x[m:m + 1], r[m:m + 1], g)
        assert torch.equal(h1, h[m:m + 1]) and torch.equal(s1, s[m:m + 1])
        assert torch.equal(q1.view(torch.uint8), q[m:m + 1].view(torch.uint8))


@pytest.mark.parametrize("M,D", [(5, 255), (1100, 4096), (2, 11008)])
@pytest.mark.parametrize("over", ["resid", "x"])
def test_norm_in_place(M, D, over):
    x = wl.draw(("f8_x", M, D), (M, D), device="cuda")
    r = wl.draw(("f8_r", M, D), (M, D), device="cuda")
    g = wl.draw(("f8_g", D), (D,), std=0.3, mean=1.0, device="cuda")
    h, q, s = run_norm(x, r, g)
    h2, q2, s2 = run_norm(x, r, g, out=r if over == "resid" else x)
    assert torch.equal(h2, h) and torch.equal(s2, s) and torch.equal(q2.view(torch.uint8), q.view(torch.uint8))


@pytest.mark.parametrize("storage", ["bf16", "f32"])
@pytest.mark.parametrize("off", [1, 3, 8])
def test_norm_at_any_alignment(storage, off):
    """Rows that start at odd elements of a larger allocation; odd widths move every further row."""
    M, D, dt = 6, 391, DT[storage]
    flat = lambda key: wl.draw((key, off), (M * D + off,), dtype=dt, device="cuda")[off:].view(M, D)  # noqa: E731
    x, r = flat("f8_xa"), flat("f8_ra")
    g = wl.draw(("f8_ga", off), (D + off,), std=0.3, mean=1.0, dtype=dt, device="cuda")[off:]
    q = torch.full((M * D + 16,), 3, dtype=torch.uint8, device="cuda")
    s = torch.empty((M, blocks(D)), device="cuda")
    h = torch.empty(M * D + off, dtype=dt, device="cuda")[off:].view(M, D)
    af.op_add_rmsnorm_fp8(x, r, g, h, q[off:off + M * D].view(M, D).view(FP8), s, 1e-6)
    check_fp8(q[off:off + M * D].view(M, D).view(FP8), s, rmsnorm(to_np(h), to_np(g), 1e-6), 1, norm_rel(D))
    assert bool((q[:off] == 3).all()) and bool((q[off + M * D:] == 3).all())


def test_norm_of_zeros_and_of_what_is_not_finite():
    D = 384
    x = torch.zeros((5, D), device="cuda")
    x[1, 5], x[2, 5], x[3] = float("nan"), float("inf"), 1e-30
    x[4, 200] = 2.0
    g = torch.ones(D, device="cuda")
    _, q, s = run_norm(x, None, g)
    v = q.float().cpu()
    assert bool((v[0] == 0).all()) and bool((s[0] == 2.0 ** -126).all())
    assert bool(v[1].isnan().all()) and bool(s[1].isnan().all())      # a NaN reaches the whole row
    # infinity: its own block is not finite, the rest of the row is divided by an infinite norm
    assert bool(v[2, :128].isnan().all()) and bool(s[2, 0].isnan()) and bool((v[2, 128:] == 0).all())
    check_fp8(q[3:], s[3:], rmsnorm(to_np(x[3:]), to_np(g), 1e-6), 1, norm_rel(D))


# ----------------------------------------------------------------------------- quantisation
@pytest.mark.parametrize("storage", ["bf16", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 128), (3, 130), (127, 129), (128, 256), (129, 391), (282, 11008), (257, 4096)])
def test_quantize(storage, block_rows, M, K):
    x = wl.draw(("f8_q", M, K), (M, K), std=0.02, dtype=DT[storage], device="cuda")
    mb = M if block_rows == 1 else blocks(M)
    q, s = outputs(M, K, mb)
    af.op_quantize_fp8(x, q[:M].view(FP8), s[:mb], block_rows)
    torch.cuda.synchronize()
    assert untouched(q, s)
    check_fp8(q[:M].view(FP8), s[:mb], to_np(x), block_rows, 0.0)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_at_any_alignment_and_extremes(block_rows):
    M, K, off = 131, 135, 1
    x = wl.draw(("f8_qa",), (M * K + off,), device="cuda")[off:].view(M, K)
    x[0, 0], x[1, 1], x[5] = 3e38, -1e-38, 0.0
    q = torch.full((M * K + 8,), 3, dtype=torch.uint8, device="cuda")
    mb = M if block_rows == 1 else blocks(M)
    s = torch.empty((mb, 2), device="cuda")
    v = q[off:off + M * K].view(M, K).view(FP8)
    af.op_quantize_fp8(x, v, s, block_rows)
    check_fp8(v, s, to_np(x), block_rows, 0.0)
    assert bool((q[:off] == 3).all()) and bool((q[off + M * K:] == 3).all())
    x[130, 134], x[2, 3] = float("-inf"), float("nan")
    af.op_quantize_fp8(x, v, s, block_rows)
    torch.cuda.synchronize()
    nan_s, nan_v = s.isnan().cpu(), v.float().isnan().cpu()
    want = torch.zeros_like(nan_s)
    want[-1, 1] = True
    want[2 if block_rows == 1 else 0, 0] = True
    assert torch.equal(nan_s, want)
    wide = want.repeat_interleave(block_rows, 0)[:M].repeat_interleave(128, 1)[:, :K]
    assert torch.equal(nan_v, wide)


def test_e4m3_rounding_is_to_nearest_even():
    """Every midpoint between two e4m3 values, and its neighbours in fp32, in a block whose scale is 1."""
    codes = torch.arange(0, 127, dtype=torch.uint8).view(FP8).double().numpy()
    mid = (codes[1:] + codes[:-1]) / 2
    vals = np.concatenate([mid, np.nextafter(mid.astype(np.float32), np.float32(0)), np.nextafter(mid.astype(np.float32), np.float32(1e9)), codes])
    vals = np.concatenate([vals, -vals]).astype(np.float32)
    rows = -(-vals.size // 127)
    x = np.zeros((rows, 128), np.float32)
    x[:, 127] = 448.0
    x[:, :127].reshape(-1)[:] = 0
    flat = np.zeros(rows * 127, np.float32)
    flat[:vals.size] = vals
    x[:, :127] = flat.reshape(rows, 127)
    q, s = torch.empty((rows, 128), dtype=torch.uint8, device="cuda").view(FP8), torch.empty((rows, 1), device="cuda")
    af.op_quantize_fp8(torch.from_numpy(x).cuda(), q, s)
    assert bool((s == 1).all())
    assert torch.equal(q.cpu().float(), torch.from_numpy(x).to(FP8).float())


# ----------------------------------------------------------------------------- projection
LINEAR_SHAPES = [(1, 1, 16), (1, 16, 128), (3, 17, 144), (7, 130, 256), (16, 128, 272), (17, 4096, 4096),
                 (31, 1000, 1040), (33, 515, 11008), (64, 257, 640), (65, 129, 384), (100, 640, 1024), (130, 384, 512),
                 (161, 1376, 688), (282, 4096, 1152), (300, 1111, 2064), (513, 771, 400), (1040, 1300, 256)]


# One shape or two for every kernel of the choice (see test_shapes_reach_every_kernel), with rows, columns and
# blocks of K left over, K below one block, and stages that the groups of waves do not share evenly.
KERNEL_SHAPES = [(1, 14, 32), (9, 300, 1936), (5, 9973, 48), (16, 9000, 400), (18, 3887, 32), (32, 5000, 1168),
                 (34, 15, 32), (35, 33, 2704), (60, 300, 1168), (17, 13982, 32), (33, 681, 32), (100, 7000, 656),
                 (21, 16361, 32), (1, 15761, 8416), (90, 5000, 1552), (72, 8606, 32), (95, 9001, 272),
                 (235, 14083, 32), (250, 4000, 912), (130, 15289, 32), (389, 7740, 144), (155, 17000, 656),
                 (374, 13191, 32), (162, 17029, 48), (250, 16200, 1040), (587, 8197, 32), (500, 8100, 528),
                 (507, 19667, 32), (510, 19667, 272), (515, 18548, 160), (570, 17900, 1040)]


def exact_inputs(M, N, K, seed):
    """Small whole numbers and scales that are powers of two: every sum is exact in fp32."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    pick = lambda shape, vals: torch.tensor(vals, device="cuda")[torch.randint(0, len(vals), shape, generator=gen, device="cuda")]  # noqa: E731
    xq, wq = (pick(s, [-2.0, -1.0, 0.0, 1.0, 2.0]).to(FP8) for s in ((M, K), (N, K)))
    xs, ws = pick((M, blocks(K)), [0.5, 1.0, 2.0]), pick((blocks(N), blocks(K)), [0.25, 1.0, 2.0])
    return xq, xs, wq, ws


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", LINEAR_SHAPES + KERNEL_SHAPES)
def test_linear_of_whole_numbers_is_exact(out, M, N, K):
    """Terms of up to 16 in steps of 1/8: sums below 11008 * 16 = 2^17.5, 21 bits in all, so every order of
    summation gives the same fp32 value; bf16 rounds it once."""
    args = exact_inputs(M, N, K, M + 3 * N + 7 * K)
    y = torch.full((M + 1, N), -3.0, dtype=DT[out], device="cuda")
    af.op_linear_fp8(*args, y[:M])
    torch.cuda.synchronize()
    want, _ = linear_fp8(*args)
    assert torch.equal(y[:M].cpu(), torch.from_numpy(want).float().to(DT[out]))
    assert bool((y[M] == -3.0).all())


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (7, 3200, 4096), (40, 1000, 2064), (282, 1024, 11008), (500, 640, 4096)])
def test_linear_of_real_values(out, M, N, K):
    """Against float64.  fp32 results: exact products, added in some order with roundings of at most 2^-23 of
    the partial sum (allowing for truncation), then one product of scales, one with the sum and one
    addition per block: at most (128 + 3 + blocks) 2^-23 of the sum of the absolute terms.  bf16 results may
    come from the 8-bit matrix instruction, which cuts each of eight neighbouring products at 2^-13 of the
    largest: at most 8 * 2^-13 of that, so of the group's absolute sum; then comes bf16's half step, 2^-8.
    As a whole such a result is within 2^-8 of the norm: the cuts are 1e-5 of it, a rounding 2^-8 at the
    most and less on the mean."""
    x = wl.draw(("f8_lx", M, K), (M, K), device="cuda")
    w = wl.draw(("f8_lw", N, K), (N, K), std=0.02, device="cuda")
    xq, xs = torch.empty((M, K), dtype=torch.uint8, device="cuda").view(FP8), torch.empty((M, blocks(K)), device="cuda")
    wq, ws = torch.empty((N, K), dtype=torch.uint8, device="cuda").view(FP8), torch.empty((blocks(N), blocks(K)), device="cuda")
    af.op_quantize_fp8(x, xq, xs)
    af.op_quantize_fp8(w, wq, ws, 128)
    y = torch.empty((M, N), dtype=DT[out], device="cuda")
    af.op_linear_fp8(xq, xs, wq, ws, y)
    want, terms = linear_fp8(xq, xs, wq, ws)
    err = np.abs(to_np(y) - want)
    bound = (131 + blocks(K)) * 2.0 ** -23 * terms
    if out == "bf16":
        bound = bound + 2.0 ** -10 * terms
        bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
        assert np.linalg.norm(err) <= 2.0 ** -8 * np.linalg.norm(want)
    else:  # no worse than an fp32 chain over blocks: 2-norm within 2 U32 sqrt(blocks + 8) of the terms'
        assert np.linalg.norm(err) <= 2 * U32 * np.sqrt(blocks(K) + 8) * np.linalg.norm(terms)
    assert np.all(err <= bound), float((err / bound).max())


@pytest.mark.parametrize("M,N,K", [(3, 100, 272), (70, 300, 400), (300, 520, 1040)])
def test_linear_reads_no_neighbour(M, N, K):
    """NaN in the row behind the activations, the weights and the scales never reaches the result, and a NaN scale
    or value reaches exactly its own row or columns."""
    xq, xs, wq, ws = exact_inputs(M, N, K, 5)
    nan = lambda t, n: torch.cat([t.float(), torch.full((n, t.shape[1]), float("nan"), device="cuda")]).to(t.dtype)  # noqa: E731
    y = torch.empty((M, N), device="cuda")
    af.op_linear_fp8(nan(xq, 130)[:M], nan(xs, 130)[:M], nan(wq, 130)[:N], nan(ws, 1)[:blocks(N)], y)
    want = torch.from_numpy(linear_fp8(xq, xs, wq, ws)[0]).float()
    assert torch.equal(y.cpu(), want)
    xs2, wq2 = xs.clone(), wq.clone().float()
    xs2[1, -1] = float("nan")
    wq2[N - 1, K - 1] = float("nan")
    af.op_linear_fp8(xq, xs2, wq2.to(FP8), ws, y)
    bad = torch.zeros((M, N), dtype=torch.bool)
    bad[1], bad[:, N - 1] = True, True
    assert torch.equal(y.isnan().cpu(), bad)
    assert torch.equal(y.cpu()[~bad], want[~bad])


def test_linear_same_rows_twice_give_the_same_bits():
    args = list(exact_inputs(64, 512, 2048, 9))
    args[1] = args[1] * 0.3
    y1, y2 = (torch.empty((64, 512), device="cuda") for _ in range(2))
    af.op_linear_fp8(*args, y1)
    af.op_linear_fp8(*args, y2)
    assert torch.equal(y1, y2)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(5, 48, 128), (64, 512, 272), (282, 1024, 128), (300, 2048, 400), (1030, 777, 144), (2264, 4096, 128)])
def test_linear_stores_at_any_alignment(out, M, N, K):
    """The same bits wherever the results begin, and nothing before or behind them."""
    xq, xs, wq, ws = exact_inputs(M, N, K, 7)[:4]
    dt = DT[out]
    want = torch.empty(M, N, dtype=dt, device="cuda")
    af.op_linear_fp8(xq, xs, wq, ws, want)
    for off in (1, 3, 4, 8):
        room = torch.full((M * N + 32,), -3.0, dtype=dt, device="cuda")
        y = room[off:off + M * N].view(M, N)
        af.op_linear_fp8(xq, xs, wq, ws, y)
        assert torch.equal(y, want) and bool((room[:off] == -3.0).all()) and bool((room[off + M * N:] == -3.0).all()), off
