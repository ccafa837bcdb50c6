"""The operators over a paged key-value cache as a program uses them: one behind the other, captured and replayed, on
several streams, beside the ring, and on caches whose offsets pass 32 bits."""
import math

import pytest
import torch

from tests.paged_plain import HALF_STEP, Step, inside

pytestmark = pytest.mark.gpu

af = pytest.importorskip("paper_2512_20276_amd")

F32, BF16 = torch.float32, torch.bfloat16
THETA = 10000.0


class Layer:
    """One attention layer of a program: requests come, run for some tokens and grow in a pool of pages."""

    def __init__(self, n_seq, Hkv, group, hd, page, max_pages, dtype, seed=0):
        self.n_seq, self.Hkv, self.Hq, self.hd, self.page, self.dtype = n_seq, Hkv, Hkv * group, hd, page, dtype
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        n_pages = n_seq * max_pages + 2
        self.k, self.v = (torch.full((n_pages, Hkv, page, hd), math.nan, dtype=dtype, device="cuda") for _ in range(2))
        self.table = torch.randperm(n_pages, generator=self.gen, device="cuda")[:n_seq * max_pages].view(n_seq, max_pages).to(torch.int32)
        self.lens = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
        self.seen = [[] for _ in range(n_seq)]  # (rotated k, v) of every row so far, as the cache holds them

    def step(self, counts, window=0, sinks=0, positions=None, sections=None):
        """Rows of every request; returns the attention's output, and the plain one in 64 bits."""
        M, Hq, Hkv, hd = sum(counts), self.Hq, self.Hkv, self.hd
        single = all(c == 1 for c in counts)
        starts = [0]
        for c in counts:
            starts.append(starts[-1] + c)
        st = None if single else torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.lens += torch.tensor(counts, dtype=torch.int32, device="cuda")
        kv = af.PagedKV(self.k, self.v, self.table, self.lens, st)
        qkv = torch.randn(M, Hq + 2 * Hkv, hd, generator=self.gen, device="cuda").to(self.dtype)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        plain = qkv.clone()
        af.op_rope_append_paged(kv, q, k, v, q, THETA, positions, sections)
        ws = torch.empty(af.attention_paged_workspace(kv, M, Hq), dtype=torch.uint8, device="cuda")
        o = torch.empty(M, Hq, hd, dtype=self.dtype, device="cuda")
        scale = 1.0 / math.sqrt(hd)
        af.op_attention_paged(kv, q, o, scale, ws, window, sinks)
        lens = self.lens.tolist()
        want = torch.empty(M, Hq, hd, dtype=torch.float64, device="cuda")
        half = hd // 2
        turn = THETA ** (torch.arange(half, dtype=torch.float64, device="cuda") * (-2.0 / hd))
        for b, c in enumerate(counts):
            rows = slice(starts[b], starts[b + 1])
            at = torch.arange(lens[b] - c, lens[b], device="cuda")
            pos = at[:, None].double() if positions is None else positions[rows].double().view(c, -1)
            axis = [a for a, n in enumerate(sections or [half]) for _ in range(n)]
            z = torch.polar(torch.ones(c, half, dtype=torch.float64, device="cuda"), pos[:, axis] * turn)[:, None]
            turned = lambda x: (lambda y: torch.cat([y.real, y.imag], -1))(torch.complex(x[..., :half].double(), x[..., half:].double()) * z).to(self.dtype).double()  # noqa: E731
            self.seen[b].append((turned(plain[rows, Hq:Hq + Hkv]), plain[rows, Hq + Hkv:].double()))
            K, V = (torch.cat([x[i] for x in self.seen[b]]) for i in (0, 1))
            Q = turned(plain[rows, :Hq])
            see = torch.arange(K.shape[0], device="cuda")[None] <= at[:, None]
            if window:
                see &= (torch.arange(K.shape[0], device="cuda")[None] > at[:, None] - window) | (torch.arange(K.shape[0], device="cuda")[None] < sinks)
            for h in range(Hq):
                s = (Q[:, h] @ K[:, h * Hkv // Hq].t().contiguous() * scale).masked_fill(~see, -math.inf)
                want[rows, h] = torch.softmax(s, 1) @ V[:, h * Hkv // Hq]
        return o, want


def close(o, want, dtype):
    """Of the plain form's, a rotated value is off by 2^-20 of its row's size in fp32 and by a step of bf16 where the
    two lie on different sides of a border (few do: counted as one a score, of a product below 9).  So a score, scale times hd terms
    of unit normal rows, is off by ds <= sqrt(hd) 1.2 2^-18 (fp32) or 9 2^-7 / sqrt(hd) (bf16), and the output by 2 ds and
    half a step of values below 5."""
    hd = o.shape[2]
    ds = math.sqrt(hd) * 1.2 * 2.0 ** -18 if dtype is F32 else 9 * 2.0 ** -7 / math.sqrt(hd)
    err = (o.double() - want).abs().max().item()
    assert err <= 5 * (2 * ds + HALF_STEP[dtype]), err


@pytest.mark.parametrize("dtype,hd,Hkv,group,page", [(BF16, 128, 2, 4, 16), (F32, 64, 4, 1, 8), (BF16, 64, 1, 16, 32)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 3)])
def test_a_prompt_chunks_and_tokens(dtype, hd, Hkv, group, page, window, sinks):
    """Prompts of several lengths, a second chunk beside single rows, and tokens, all in one cache that held NaN."""
    L = Layer(4, Hkv, group, hd, page, 512 // page, dtype)
    for counts in ([37, 1, 120, 5], [1, 40, 1, 1], [1, 1, 1, 1], [1, 1, 1, 1], [0, 1, 33, 2], [1, 1, 1, 1]):
        o, want = L.step(counts, window, sinks)
        close(o, want, dtype)


def test_image_positions():
    """Patches of two frames (time, height, width), then text on all axes alike."""
    t = torch.arange(2).repeat_interleave(20)
    h, w = torch.arange(40) // 5 % 4, torch.arange(40) % 5
    text = torch.arange(7) + 6
    pos = torch.stack([torch.cat([a, text]) for a in (t, h, w)], dim=1).to(torch.int32).cuda()
    L = Layer(1, 2, 2, 64, 16, 16, BF16)
    close(*L.step([47], positions=pos, sections=[8, 12, 12]), BF16)
    close(*L.step([1], positions=torch.full((1, 3), 13, dtype=torch.int32, device="cuda"), sections=[8, 12, 12]), BF16)


def test_captured_and_replayed_with_other_lengths():
    """A captured decode step replays with the lengths, table and rows that are there then; every replay is compared with
    the eager call's, with the program's own eager work between."""
    for n_seq, max_pages in ((5, 8), (5, 80)):
        s = Step([(1, 100)] * n_seq, 2, 4, 128, 16, BF16, single=True, spare_pages=n_seq * max_pages, extra_table=max_pages - 7)
        kv = s.to_gpu(af)
        n = s.k_cache.shape[0]
        o, q_out = torch.zeros_like(s.g["q"]), torch.zeros_like(s.g["q"])
        lse = torch.zeros(s.M, s.Hq, device="cuda")
        ws = torch.empty(af.attention_paged_workspace(kv, s.M, s.Hq), dtype=torch.uint8, device="cuda")

        def step(o, lse):
            af.op_rope_append_paged(kv, s.g["q"], s.g["k"], s.g["v"], q_out, THETA)
            af.op_attention_paged(kv, q_out, o, 0.09, ws, 0, 0, lse)

        step(o, lse)
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            step(o, lse)
        g = torch.Generator(device="cuda").manual_seed(3)
        for turn in range(5):
            s.g["lens"].copy_(torch.randint(0, 16 * max_pages, (n_seq,), generator=g, device="cuda"))
            s.g["table"].copy_(torch.randperm(n, generator=g, device="cuda")[:n_seq * max_pages].view(n_seq, max_pages))
            s.g["q"].normal_(generator=g)
            s.g["k"].normal_(generator=g)
            graph.replay()
            torch.cuda.synchronize()
            want_o, want_lse = torch.ones_like(o), torch.ones_like(lse)
            step(want_o, want_lse)
            torch.cuda.synchronize()
            assert torch.equal(o, want_o) and torch.equal(lse, want_lse), turn


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_captured_packed_rows_replayed_with_other_requests(dtype):
    """A captured step of packed rows replays with other starts, so that prompts, chunks, single rows and requests without rows
    change places, and with other lengths: keys that were split are not, and the other way round."""
    for hkv, group, past in ((1, 4, 2500), (4, 8, 300)):
        s = Step([(90, 100 + past)] * 4, hkv, group, 64, 16, dtype)
        kv = s.to_gpu(af)
        o = torch.zeros_like(s.g["q"])
        ws = torch.empty(af.attention_paged_workspace(kv, s.M, s.Hq), dtype=torch.uint8, device="cuda")
        step = lambda o: af.op_attention_paged(kv, s.g["q"], o, 0.1, ws)  # noqa: E731
        step(o)
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            step(o)
        for counts in ([360, 0, 0, 0], [1, 1, 300, 1], [2, 355, 1, 2], [90, 90, 90, 90], [0, 0, 1, 4]):
            lens = [max(n, (37 * i + 11 * n + past) % (100 + past)) for i, n in enumerate(counts)]
            starts = [sum(counts[:i]) for i in range(5)]
            kv.q_starts.copy_(torch.tensor(starts, dtype=torch.int32))
            s.g["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
            o.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            want = torch.full_like(o, 7.0)
            step(want)
            torch.cuda.synchronize()
            assert torch.equal(o, want), counts
            assert (o[starts[4]:] == 7).all()
            scores = torch.full((s.M, s.Hq), -1.0, dtype=torch.float32, device="cuda")
            af.op_attention_paged(kv, s.g["q"], want, 0.1, ws, 0, 0, scores)
            rows = [starts[b] + i for b in range(4) for i in range(counts[b])]
            assert torch.isfinite(scores[rows]).all()


def test_several_streams():
    """Calls on streams of their own, with a workspace each, give what one behind the other gives."""
    steps = [Step([(9, 700), (1, 2000), (64, 64)], 2, 4, 128, 32, BF16, seed=i) for i in range(3)]
    alone, outs = [], []
    for s in steps:
        s.to_gpu(af)
        s.ws = torch.empty(af.attention_paged_workspace(s.kv, s.M, s.Hq), dtype=torch.uint8, device="cuda")
        o = torch.zeros_like(s.g["q"])
        af.op_attention_paged(s.kv, s.g["q"], o, 0.1, s.ws)
        alone.append(o)
        outs.append(torch.zeros_like(o))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for s, o, st in zip(steps, outs, streams):
            af.op_attention_paged(s.kv, s.g["q"], o, 0.1, s.ws, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, o) for a, o in zip(alone, outs))


def test_requests_that_share_pages():
    """A common prompt in pages that several requests read, alone and behind each other."""
    s = Step([(1, 90), (1, 70), (3, 100)], 2, 2, 64, 16)
    s.table[1, :4] = s.table[0, :4]
    s.table[2, :4] = s.table[0, :4]
    kv = s.to_gpu(af)
    o = torch.zeros_like(s.g["q"])
    ws = torch.empty(af.attention_paged_workspace(kv, s.M, s.Hq), dtype=torch.uint8, device="cuda")
    af.op_attention_paged(kv, s.g["q"], o, 0.125, ws)
    want, bound, _, _ = s.attended(0.125)
    inside(o, want, bound)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_same_as_the_ring(dtype):
    """A prompt in a ring slot and in pages: both within the bound of the same 64-bit result."""
    H, hd, n, page = 4, 64, 70, 16
    s = Step([(n, n)], H, 1, hd, page, dtype)
    s.to_gpu(af)
    k, v = (torch.stack([c[s.cell(0, j)[0], :, s.cell(0, j)[1]] for j in range(n)]) for c in (s.g["k_cache"], s.g["v_cache"]))
    ring = af.Ring(1, 2, 96, H, hd, dtype=dtype)
    seg = ring.append(0, n)
    ring.write_kv(0, seg.slot, 0, k, v)
    of_ring, of_pages = torch.empty_like(s.g["q"]), torch.empty_like(s.g["q"])
    af.op_attention(ring, 0, s.g["q"], [seg], of_ring)
    ws = torch.empty(af.attention_paged_workspace(s.kv, n, H), dtype=torch.uint8, device="cuda")
    af.op_attention_paged(s.kv, s.g["q"], of_pages, 1.0 / math.sqrt(hd), ws)
    want, bound, _, _ = s.attended(1.0 / math.sqrt(hd))
    inside(of_ring, want, bound, "ring")
    inside(of_pages, want, bound, "pages")


def test_a_cache_past_32_bits():
    """Pages past 2^31 elements and 2^32 bytes of a cache, written and read."""
    Hkv, hd, page = 8, 128, 64
    n_pages = (1 << 31) // (Hkv * page * hd) + 2048
    k = torch.empty(n_pages, Hkv, page, hd, dtype=BF16, device="cuda")
    v = torch.empty_like(k)
    small = Step([(1, 150), (40, 70)], Hkv, 2, hd, page, BF16)
    small.to_gpu(af)
    there = (n_pages - 1 - 7 * torch.arange(small.k_cache.shape[0])).cuda()
    k[there], v[there] = small.g["k_cache"], small.g["v_cache"]
    table = torch.where(small.g["table"] >= 0, n_pages - 1 - 7 * small.g["table"], -1).to(torch.int32)
    kv = af.PagedKV(k, v, table, small.g["lens"], small.kv.q_starts)
    results = []
    for c, ck, cv in ((small.kv, small.g["k_cache"], small.g["v_cache"]), (kv, k, v)):
        q_out, o = torch.zeros_like(small.g["q"]), torch.zeros_like(small.g["q"])
        af.op_rope_append_paged(c, small.g["q"], small.g["k"], small.g["v"], q_out, THETA)
        ws = torch.empty(af.attention_paged_workspace(c, small.M, small.Hq), dtype=torch.uint8, device="cuda")
        af.op_attention_paged(c, q_out, o, 0.1, ws)
        results.append((q_out, o))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert torch.equal(k[there], small.g["k_cache"]) and torch.equal(v[there], small.g["v_cache"])


def test_rows_of_any_stride():
    """Queries and outputs that are parts of wider rows; the rest of the rows stays."""
    s = Step([(9, 40), (1, 30), (1, 600)], 2, 2, 128, 16)
    s.to_gpu(af)
    wide = torch.randn(s.M, 9, 128, device="cuda").to(BF16)
    wide[:, 3:7] = s.g["q"]
    out = torch.full((s.M, 6, 128), 7.0, dtype=BF16, device="cuda")
    ws = torch.empty(af.attention_paged_workspace(s.kv, s.M, s.Hq), dtype=torch.uint8, device="cuda")
    af.op_attention_paged(s.kv, wide[:, 3:7], out[:, 1:5], 0.1, ws)
    want, bound, _, _ = s.attended(0.1)
    inside(out[:, 1:5], want, bound)
    assert bool((out[:, 0] == 7.0).all()) and bool((out[:, 5] == 7.0).all())
