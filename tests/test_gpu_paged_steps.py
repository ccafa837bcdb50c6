"""GPU tests of attention over a paged cache at pools, steps and replays that a program meets beside the usual ones."""
import math

import pytest
import torch

from tests.paged_plain import Step, inside

pytestmark = pytest.mark.gpu

af = pytest.importorskip("paper_2512_20276_amd")

F32, BF16 = torch.float32, torch.bfloat16


def attend(s: Step, kv=None, window=0, sinks=0):
    kv = kv or s.to_gpu(af)
    o = torch.full((s.M, s.Hq, s.hd), 7.0, dtype=s.dtype, device="cuda")
    lse = torch.full((s.M, s.Hq), 7.0, device="cuda")
    workspace = torch.full((af.attention_paged_workspace(kv, s.M, s.Hq),), 255, dtype=torch.uint8, device="cuda")
    af.op_attention_paged(kv, s.g["q"], o, 1.0 / math.sqrt(s.hd), workspace, window, sinks, lse)
    return o, lse


def check(s: Step, o, lse, window=0, sinks=0):
    want, bound, want_lse, lse_bound = s.attended(1.0 / math.sqrt(s.hd), window, sinks)
    inside(o, want, bound, "o")
    inside(lse, want_lse, lse_bound, "lse")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("requests,single", [([(1, 41), (1, 900), (1, 8)], True), ([(70, 100), (1, 64), (2, 900)], False)])
def test_pools_aligned_to_16_bytes_alone(dtype, hd, requests, single):
    """The header promises no more than 16: pools that begin 16 bytes behind a multiple of 256."""
    s = Step(requests, 2, 4, hd, 16, dtype, single)
    s.to_gpu(af)
    for name in ("k_cache", "v_cache"):
        c = s.g[name]
        wide = torch.empty(c.numel() + 256, dtype=dtype, device="cuda")
        off = (16 - wide.data_ptr() % 256) % 256 // dtype.itemsize
        s.g[name] = wide[off:off + c.numel()].view(c.shape).copy_(c)
        assert s.g[name].data_ptr() % 32 == 16
    kv = af.PagedKV(s.g["k_cache"], s.g["v_cache"], s.g["table"], s.g["lens"], s.kv.q_starts)
    check(s, *attend(s, kv))
    q_out = torch.empty_like(s.g["q"])
    af.op_rope_append_paged(s.kv, s.g["q"], s.g["k"], s.g["v"], q_out, 1e4)
    usual = s.kv.k.clone(), s.kv.v.clone()
    af.op_rope_append_paged(kv, s.g["q"], s.g["k"], s.g["v"], q_out, 1e4)
    assert torch.equal(kv.k, usual[0]) and torch.equal(kv.v, usual[1])


def _with(s: Step, counts, lens):
    """The step's pool, table and rows with other counts of rows and lengths."""
    s.requests = list(zip(counts, lens))
    s.starts = [sum(counts[:i]) for i in range(len(counts) + 1)]
    s.lens = torch.tensor(lens, dtype=torch.int32)
    return torch.tensor(s.starts, dtype=torch.int32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hkv,group,past", [(1, 4, 1500), (4, 8, 300)])
def test_replays_of_packed_rows_against_64_bits(dtype, hkv, group, past):
    """One captured step whose rows change hands: prompts, chunks, single rows, requests without rows, a padded batch."""
    s = Step([(40, 40 + past)] * 4, hkv, group, 64, 16, dtype)
    kv = s.to_gpu(af)
    o, lse = torch.zeros_like(s.g["q"]), torch.zeros(s.M, s.Hq, device="cuda")
    ws = torch.empty(af.attention_paged_workspace(kv, s.M, s.Hq), dtype=torch.uint8, device="cuda")
    step = lambda: af.op_attention_paged(kv, s.g["q"], o, 0.125, ws, 0, 0, lse)  # noqa: E731
    step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step()
    for counts in ([160, 0, 0, 0], [1, 1, 150, 1], [2, 155, 1, 2], [40, 40, 40, 40], [0, 0, 1, 4], [0, 1, 0, 0], [1, 1, 1, 1]):
        lens = [min(max(n, (37 * i + 11 * n + past) % (40 + past)), 40 + past) for i, n in enumerate(counts)]
        kv.q_starts.copy_(_with(s, counts, lens))
        s.g["lens"].copy_(s.lens)
        o.fill_(7.0), lse.fill_(7.0), ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        check(s, o, lse)
        assert (o[sum(counts):] == 7).all() and (lse[sum(counts):] == 7).all()


@pytest.mark.parametrize("dtype,rows", [(BF16, 520), (BF16, 600), (F32, 250), (F32, 300)])
def test_a_chunk_on_a_long_cache_beside_many_rows(dtype, rows):
    """Either side of the number of rows from which tiles are not split."""
    check(*(lambda s: (s, *attend(s)))(Step([(rows, rows), (9, 6000), (1, 3000)], 8, 8, 64, 16, dtype)))


def test_one_request_of_a_padded_step():
    """A step of one request with places for many rows, of which it has one, many or none."""
    s = Step([(60, 3000)], 2, 4, 128, 16, BF16)
    kv = s.to_gpu(af)
    for n, length in ((60, 3000), (1, 2999), (0, 77), (2, 2), (1, 1)):
        kv.q_starts.copy_(_with(s, [n], [length]))
        s.g["lens"].copy_(s.lens)
        o, lse = attend(s, kv)
        check(s, o, lse)
        assert (o[n:] == 7).all()


def test_one_workspace_for_every_step():
    """Asked for the largest step, it serves the smaller ones, with q_starts and without."""
    s = Step([(300, 1500)] * 4, 4, 8, 64, 16, BF16)
    kv = s.to_gpu(af)
    n = af.attention_paged_workspace(kv, s.M, s.Hq)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    seen = []
    for counts, single in (([300] * 4, False), ([60] * 4, False), ([20, 1, 0, 1], False), ([1] * 4, False), ([1] * 4, True)):
        starts = _with(s, counts, [1500, 900, 40, 700])
        M = sum(counts)
        part = af.PagedKV(kv.k, kv.v, kv.page_table, s.lens.cuda(), None if single else starts.cuda())
        o = torch.full((M, s.Hq, s.hd), 7.0, dtype=BF16, device="cuda")
        af.op_attention_paged(part, s.g["q"][:M], o, 0.125, ws)
        if counts[0] < 300:
            t = Step(s.requests, 4, 8, 64, 16, BF16)
            t.k_cache, t.v_cache, t.table, t.q = s.k_cache, s.v_cache, s.table, s.q[:M]
            want, bound, _, _ = t.attended(0.125)
            inside(o, want, bound, counts)
        seen.append(af.attention_paged_workspace(part, M, s.Hq))
    assert max(seen) <= n
