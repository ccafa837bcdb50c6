"""GPU tests of the operators over a paged key-value cache: append with the rotation, and attention over the pages."""
import math

import pytest
import torch

from tests.paged_plain import Step, inside

pytestmark = pytest.mark.gpu

af = pytest.importorskip("paper_2512_20276_amd")

F32, BF16 = torch.float32, torch.bfloat16
THETA = 10000.0


def append(s: Step, positions=None, sections=None, theta=THETA, q_out=None, stream=None):
    kv = s.kv if hasattr(s, "kv") else s.to_gpu(af)
    q_out = torch.full_like(s.g["q"], 7.0) if q_out is None else q_out
    af.op_rope_append_paged(kv, s.g["q"], s.g["k"], s.g["v"], q_out, theta,
                            None if positions is None else positions.cuda(), sections, stream)
    return q_out


def check_append(s: Step, q_out, positions=None, sections=None, theta=THETA):
    (q, q_bound), (k, k_bound) = s.rotated(theta, positions, sections)
    want_q = torch.full_like(q, 7.0)
    bound = torch.zeros_like(q)
    want_k, want_v = s.k_cache.double().clone(), s.v_cache.clone()
    bound_k = torch.zeros_like(want_k)
    for row, b, p in s.rows():
        want_q[row], bound[row] = q[row], q_bound[row]
        at = s.cell(b, p)
        if at is not None:
            want_k[at[0], :, at[1]], bound_k[at[0], :, at[1]], want_v[at[0], :, at[1]] = k[row], k_bound[row], s.v[row]
    inside(q_out, want_q, bound, "q")
    inside(s.g["k_cache"], want_k, bound_k, "k")
    assert torch.equal(s.g["v_cache"].cpu(), want_v)


def attend(s: Step, scale=None, window=0, sinks=0, lse=True, workspace=None):
    kv = s.kv if hasattr(s, "kv") else s.to_gpu(af)
    scale = 1.0 / math.sqrt(s.hd) if scale is None else scale
    o = torch.full((s.M, s.Hq, s.hd), 7.0, dtype=s.dtype, device="cuda")
    out = torch.full((s.M, s.Hq), 7.0, device="cuda") if lse else None
    if workspace is None:  # what a workspace holds does not matter
        workspace = torch.full((af.attention_paged_workspace(kv, s.M, s.Hq),), 255, dtype=torch.uint8, device="cuda")
    af.op_attention_paged(kv, s.g["q"], o, scale, workspace, window, sinks, out)
    return o, out


def check_attend(s: Step, scale=None, window=0, sinks=0, lse=True):
    o, got_lse = attend(s, scale, window, sinks, lse)
    want, bound, want_lse, lse_bound = s.attended(1.0 / math.sqrt(s.hd) if scale is None else scale, window, sinks)
    inside(o, want, bound, "o")
    mine = torch.tensor([r for r, _, _ in s.rows()], dtype=torch.long)
    others = torch.ones(s.M, dtype=torch.bool)
    others[mine] = False
    assert bool((o.cpu()[others] == 7.0).all())
    if lse:
        inside(got_lse, want_lse, lse_bound, "lse")
        assert bool((got_lse.cpu()[others] == 7.0).all())
    return o


# ----------------------------------------------------------------------------- append
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,Hkv,group,page", [(64, 4, 1, 16), (128, 2, 4, 8), (128, 1, 8, 64), (64, 3, 5, 32)])
@pytest.mark.parametrize("requests,single,before,behind", [
    ([(1, 1)], True, 0, 0),
    ([(1, 36), (1, 8), (1, 17), (1, 9)], True, 0, 0),
    ([(5, 5), (1, 40), (0, 9), (33, 50), (1, 1)], False, 0, 0),
    ([(0, 0), (2, 70), (0, 3)], False, 3, 4),
])
def test_append(dtype, hd, Hkv, group, page, requests, single, before, behind):
    s = Step(requests, Hkv, group, hd, page, dtype, single, before, behind)
    check_append(s, append(s))


@pytest.mark.parametrize("n_axes,sections", [(1, None), (1, [32]), (2, [10, 22]), (3, [8, 12, 12]), (3, [0, 31, 1]), (2, [32, 0])])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_positions_of_several_axes(dtype, n_axes, sections):
    s = Step([(20, 25), (1, 9), (6, 6)], 2, 3, 64, 8, dtype, behind=2)
    pos = torch.randint(-5, 5000, (s.M, n_axes), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    check_append(s, append(s, pos if n_axes > 1 else pos[:, 0].contiguous(), sections), pos, sections)


@pytest.mark.parametrize("theta", [10000.0, 500000.0, 1.0, 0.5])
def test_append_far_positions(theta):
    far = torch.tensor([0, 1, 100003, 10 ** 6, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, -77], dtype=torch.int32)
    s = Step([(8, 8)], 2, 2, 128, 16, F32)
    check_append(s, append(s, far, theta=theta), far, theta=theta)


def test_append_of_a_projection_s_rows_and_in_place():
    """q, k and v as parts of one projection's rows; the rotated queries where the queries were."""
    s = Step([(7, 20), (3, 3)], 2, 3, 128, 16, BF16)
    s.to_gpu(af)
    qkv = torch.cat([s.g["q"], s.g["k"], s.g["v"]], dim=1)
    s.g["q"], s.g["k"], s.g["v"] = qkv[:, :6], qkv[:, 6:8], qkv[:, 8:]
    q = append(s, q_out=s.g["q"])
    check_append(s, q)
    assert torch.equal(qkv[:, 6:8].cpu(), s.k) and torch.equal(qkv[:, 8:].cpu(), s.v)


def test_append_of_rows_without_a_cell():
    """Pages that do not exist, positions past the table and before 0: the row is rotated and not written."""
    s = Step([(4, 30), (3, 40), (5, 2), (2, 1000), (1, 12)], 2, 2, 64, 8)
    s.table[0, 3] = -1
    s.table[1, 4] = s.k_cache.shape[0]
    s.table[4, 1] = 2 ** 31 - 1
    check_append(s, append(s))


# ----------------------------------------------------------------------------- attention: single rows
LENGTHS = [1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 100, 129, 250]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,Hkv,group,page", [(64, 4, 1, 16), (128, 2, 4, 8), (128, 1, 16, 64), (64, 1, 17, 32), (128, 1, 35, 256),
                                               (64, 3, 5, 128)])
@pytest.mark.parametrize("split", [False, True])
def test_single_rows(dtype, hd, Hkv, group, page, split):
    """Short tables take a workgroup a request, long ones shares of all requests' keys."""
    s = Step([(1, n) for n in LENGTHS], Hkv, group, hd, page, dtype, single=True, extra_table=(640 // page + 1) if split else 0)
    check_attend(s)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("requests", [[(1, 5000)], [(1, 1), (1, 3000), (1, 0), (1, 2), (1, 2047), (1, 129)],
                                      [(1, 40 * i) for i in range(70)], [(1, 0)] * 3, [(1, 700)] + [(1, 0)] * 70 + [(1, 33)]])
def test_single_rows_of_long_caches(dtype, requests):
    check_attend(Step(requests, 2, 4, 128, 32, dtype, single=True))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 0), (32, 4), (33, 32), (64, 33), (100, 70), (1000, 20), (5000, 3)])
@pytest.mark.parametrize("long_table", [False, True])
def test_single_rows_with_a_window(window, sinks, long_table):
    s = Step([(1, n) for n in [0] + LENGTHS + [300, 411] + ([1500] if long_table else [])], 2, 2, 64, 16, single=True)
    check_attend(s, window=window, sinks=sinks)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_scales(scale):
    check_attend(Step([(1, 90), (1, 5), (1, 700)], 2, 2, 64, 16, single=True), scale=scale)
    check_attend(Step([(9, 90), (5, 5)], 2, 2, 64, 16), scale=scale)


# ----------------------------------------------------------------------------- attention: several rows
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,Hkv,group,page", [(64, 4, 1, 16), (128, 2, 4, 8), (128, 1, 7, 64), (64, 2, 8, 32), (128, 1, 40, 16)])
@pytest.mark.parametrize("requests", [[(2, 2)], [(33, 33)], [(65, 65), (2, 100)], [(5, 5), (1, 40), (0, 9), (33, 150), (1, 1)],
                                      [(130, 131)], [(1, 30), (1, 8)]])
def test_several_rows(dtype, hd, Hkv, group, page, requests):
    check_attend(Step(requests, Hkv, group, hd, page, dtype, before=1, behind=3))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("requests", [[(2, 4000)], [(40, 3000), (1, 2500), (3, 700)], [(17, 2100)] * 3, [(700, 1500), (1, 3000)],
                                      [(2, 2100), (2, 40)]])
def test_chunks_on_long_caches(dtype, requests):
    """Few rows and many keys: the keys are split and joined."""
    check_attend(Step(requests, 2, 4, 128, 32, dtype))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (16, 0), (50, 4), (64, 64), (200, 33)])
@pytest.mark.parametrize("hd,group,dtype", [(64, 2, F32), (128, 4, BF16), (64, 1, BF16)])
def test_several_rows_with_a_window(window, sinks, hd, group, dtype):
    check_attend(Step([(150, 150), (70, 400), (1, 200), (3, 90)], 2, group, hd, 16, dtype), window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_one_request_of_a_packed_step(dtype):
    """A prompt, and a single row with rows of nobody around it, on a long cache."""
    check_attend(Step([(50, 1900)], 2, 4, 64, 16, dtype, before=1, behind=2))
    check_attend(Step([(1, 1900)], 2, 4, 64, 16, dtype, before=1, behind=2))
    check_attend(Step([(1, 1900)], 2, 4, 64, 16, dtype))
    check_attend(Step([(0, 1900)], 2, 4, 64, 16, dtype, behind=2))


@pytest.mark.parametrize("requests,dtype", [([(600, 600), (500, 700)], BF16), ([(300, 300), (1, 90), (260, 400)], F32)])
def test_prompts_that_fill_the_gpu_once(requests, dtype):
    """Tiles of rows for more than half of the workgroups that the GPU holds, and no more than all of them."""
    check_attend(Step(requests, 4, 8, 64, 16, dtype, before=1, behind=2))


def test_window_over_chunks_that_are_split():
    check_attend(Step([(20, 3000), (1, 2900)], 1, 4, 128, 16), window=1700, sinks=40)


@pytest.mark.parametrize("n_seq,Hkv,group,hd,dtype", [(701, 3, 2, 64, BF16), (351, 3, 4, 128, F32), (2101, 1, 1, 64, F32)])
@pytest.mark.parametrize("single", [True, False])
def test_short_caches_of_many_requests(n_seq, Hkv, group, hd, dtype, single):
    """A request's key head on one, two or four waves, with waves left over in the last workgroup."""
    requests = [(1 if single else (1, 1, 0, 2)[i % 4], 1 + (i * 31) % (100 if i % 9 else 3)) for i in range(n_seq)]
    requests = [(n, max(n, length)) for n, length in requests]
    check_attend(Step(requests, Hkv, group, hd, 16, dtype, single=single))


def test_many_requests_of_long_caches():
    """More requests than a wave has lanes, whose keys are split: single rows, chunks, rows of nobody."""
    requests = [((0, 1, 1, 2, 9)[i % 5], 9 + (i * 37) % 90 + (1500 if i % 23 == 0 else 0)) for i in range(131)]
    check_attend(Step(requests, 1, 4, 64, 16, before=2, behind=5))
    check_attend(Step(requests, 1, 4, 64, 16, before=2, behind=5), window=700, sinks=9)


@pytest.mark.parametrize("requests,Hkv,dtype", [([(2, 1100)] * 700, 1, BF16),
                                                ([(2, 1100)] * 380 + [(9, 4000)] * 3 + [(1, 700)] * 4 + [(3, 40)] * 30, 1, BF16),
                                                ([(3, 700), (1, 30)] * 60 + [(3, 5000)], 4, F32)])
def test_many_requests_of_equal_long_caches(requests, Hkv, dtype):
    """Tiles of rows that fill the GPU without a split, or nearly, beside longer ones."""
    check_attend(Step(requests, Hkv, 1, 64, 64, dtype))


def test_starts_that_are_not_ascending():
    """No result means anything then, and nothing but the rows and the workspace is written."""
    for n_seq, rows in ((200, 24), (40, 2), (900, 9)):
        s = Step([(rows, 1200)] + [(0, 1200)] * 2, 1, 2, 64, 64)
        s.to_gpu(af)
        table = s.g["table"][:1].expand(n_seq, -1).contiguous()
        lens = torch.full((n_seq,), 1200, dtype=torch.int32, device="cuda")
        starts = torch.tensor([0, rows] * (n_seq // 2) + [0], dtype=torch.int32, device="cuda")
        kv = af.PagedKV(s.g["k_cache"], s.g["v_cache"], table, lens, starts)
        n = af.attention_paged_workspace(kv, rows, s.Hq)
        around = torch.full((n + 8192,), 7, dtype=torch.uint8, device="cuda")
        o = torch.full((rows + 20, s.Hq, s.hd), 7.0, dtype=BF16, device="cuda")
        af.op_attention_paged(kv, s.g["q"], o[10:10 + rows], 0.125, around[4096:4096 + n])
        torch.cuda.synchronize()
        assert (around[:4096] == 7).all() and (around[4096 + n:] == 7).all()
        assert (o[:10] == 7).all() and (o[10 + rows:] == 7).all()


def test_the_same_inputs_give_the_same_bits():
    for requests, single in (([(1, 2000), (1, 5), (1, 900)], True), ([(30, 2000), (1, 1500), (9, 60)], False)):
        s = Step(requests, 2, 4, 128, 16, single=single)
        first, lse = attend(s)
        for _ in range(3):
            again, more = attend(s)
            assert torch.equal(first, again) and torch.equal(lse, more)


def test_many_requests():
    """More requests than a wave has lanes, some without rows or keys."""
    requests = [((0, 1, 2, 3, 9)[i % 5], (0, 1, 2, 3, 9)[i % 5] + (i * 37) % 90) for i in range(150)]
    check_attend(Step(requests, 2, 2, 64, 16, before=2, behind=5))


# ----------------------------------------------------------------------------- what nobody sees
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("worst", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 5)])
def test_cells_that_no_row_sees_do_not_matter(dtype, worst, window, sinks):
    """Stale cells behind a request's length, pages of nobody and keys left of the window."""
    for requests, single in (([(1, 41), (1, 8), (1, 600), (1, 97)], True), ([(5, 41), (1, 8), (70, 90), (3, 700)], False)):
        s = Step(requests, 2, 2, 128, 16, dtype, single=single)
        seen = torch.zeros(s.k_cache.shape[0], s.page, dtype=torch.bool)
        for _, b, p in s.rows():
            for j in range(p + 1):
                if not window or j > p - window or j < sinks:
                    seen[s.cell(b, j)] = True
        for c in (s.k_cache, s.v_cache):
            c.permute(0, 2, 1, 3)[~seen] = worst
        check_attend(s, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("worst", [math.nan, math.inf])
def test_a_row_does_not_see_a_later_row_s_values(dtype, worst):
    """A value that is not finite changes the rows that see it and no others, in either cache, also at a window's edge."""
    for window in (0, 30):
        for which, at in (("v_cache", 37), ("k_cache", 37), ("v_cache", 3), ("v_cache", 69)):
            s = Step([(60, 70), (4, 20)], 2, 2, 64, 16, dtype)
            clean, _ = attend(s, window=window)
            s2 = Step([(60, 70), (4, 20)], 2, 2, 64, 16, dtype)
            page, off = s2.cell(0, at)
            getattr(s2, which)[page, :, off] = worst
            got, _ = attend(s2, window=window)
            for row, b, p in s.rows():
                sees = b == 0 and at <= p and (not window or at > p - window)
                if not sees:  # sums of 70 products below 1 in another order, 2 x 70 U32, and a bf16 step
                    assert torch.allclose(got[row].float(), clean[row].float(), rtol=2.0 ** -7 if dtype is BF16 else 0, atol=1e-5), (which, at, row)
                elif which == "v_cache":
                    assert not torch.isfinite(got[row]).any(), (which, at, row)


def test_pages_that_do_not_exist_and_lengths_past_the_table():
    for single in (True, False):
        requests = [(1, 60), (1, 45), (1, 90), (1, 30)] if single else [(20, 60), (5, 45), (1, 90), (40, 30)]
        s = Step(requests, 2, 2, 64, 8, single=single)
        s.table[0, 2] = -1
        s.table[1, 0] = s.k_cache.shape[0]
        s.table[2, :] = -5
        s.table[3, 3] = 2 ** 31 - 1
        check_attend(s)
        s = Step([(1, 60), (1, 45)] if single else [(20, 60), (5, 45)], 2, 2, 64, 8, single=single)
        s.requests = [(n, length + 37) for n, length in s.requests]
        s.lens += 37
        check_attend(s)
        check_attend(s, window=50, sinks=3)
        check_attend(s, window=20, sinks=0)


def test_lengths_below_the_rows_and_below_zero():
    """Rows at positions below 0 see nothing: zeros, and -inf."""
    s = Step([(6, 4), (1, 0), (3, 0), (2, 9)], 2, 2, 64, 8)
    check_attend(s)
    s = Step([(1, 5), (1, 0), (1, 9)], 2, 2, 64, 8, single=True)
    s.lens[1] = -3
    check_attend(s)
    for big in (2 ** 31 - 1, 2 ** 30):
        s = Step([(1, 30), (1, 9)], 2, 2, 64, 8, single=True)
        s.lens[0] = big
        s.to_gpu(af)
        o, _ = attend(s)  # all its keys
        t = Step([(1, 30), (1, 9)], 2, 2, 64, 8, single=True)
        t.requests[0] = (1, 32)
        t.lens[0] = 32
        assert torch.equal(o, attend(t)[0])


def test_starts_that_pass_the_rows_stay_inside():
    """q_starts past M, below 0 and descending: rows are cut to the packed ones, nothing else is touched."""
    s = Step([(4, 20), (3, 9)], 2, 2, 64, 8)
    for starts in ([-5, 4, 900], [2, 1, 7], [0, 2 ** 31 - 1, 7], [7, 7, 7]):
        s.to_gpu(af)
        s.kv.q_starts.copy_(torch.tensor(starts, dtype=torch.int32))
        append(s)
        attend(s)
    torch.cuda.synchronize()
