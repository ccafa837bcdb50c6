"""The 8-bit operators and the sampler as a program uses them: one behind the other, captured and replayed,
on several streams, in the pipeline, and on tensors whose offsets pass 32 bits."""
import types

import numpy as np
import pytest
import torch

import workload as wl
from tests.helpers import to_np
from tests.plain_ops import FP8, U32, blocks, check_fp8, linear_fp8, norm_rel, rmsnorm, sample_row

pytestmark = pytest.mark.gpu

af = pytest.importorskip("paper_2512_20276_amd")
from paper_2512_20276_amd.pipeline import Pipeline  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16


def q8(*shape):
    return torch.zeros(shape, dtype=torch.uint8, device="cuda").view(FP8)


def f32(*shape):
    return torch.zeros(shape, dtype=F32, device="cuda")


class Tail:
    """The end of a decoder layer and the head: norm, MLP projection up and down, norm, head, draw."""

    def __init__(self, M, D=512, F=1040, V=1000, tag=0):
        d = lambda name, *s, **kw: wl.draw((name, tag, *s), s, dtype=BF16, device="cuda", **kw)  # noqa: E731
        self.M, self.D, self.F, self.V = M, D, F, V
        self.g1, self.g2 = d("tog_g1", D, std=0.2, mean=1.0), d("tog_g2", D, std=0.2, mean=1.0)
        self.up, self.down, self.head = (self.weight(d(n, *s, std=0.05)) for n, s in
                                         (("tog_up", (F, D)), ("tog_down", (D, F)), ("tog_head", (V, D))))
        self.x, self.r = d("tog_x", M, D), d("tog_r", M, D)
        self.uniforms = torch.rand(M, generator=torch.Generator().manual_seed(5 + tag)).cuda()
        self.settings = dict(temperature=torch.full((M,), 0.9, device="cuda"), top_p=torch.full((M,), 0.95, device="cuda"),
                             top_k=torch.full((M,), 50, dtype=torch.int32, device="cuda"))
        self.out = self.buffers()

    @staticmethod
    def weight(w):
        q, s = q8(*w.shape), f32(blocks(w.shape[0]), blocks(w.shape[1]))
        af.op_quantize_fp8(w, q, s, 128)
        return q, s

    def buffers(self):
        M, D, F, V = self.M, self.D, self.F, self.V
        return dict(h1=torch.zeros(M, D, dtype=BF16, device="cuda"), n1=q8(M, D), s1=f32(M, blocks(D)),
                    a=torch.zeros(M, F, dtype=BF16, device="cuda"), aq=q8(M, F), as_=f32(M, blocks(F)),
                    y=torch.zeros(M, D, dtype=BF16, device="cuda"), h2=torch.zeros(M, D, dtype=BF16, device="cuda"),
                    n2=q8(M, D), s2=f32(M, blocks(D)), z=f32(M, V), tokens=torch.zeros(M, dtype=torch.int32, device="cuda"))

    def run(self, b=None, stream=None):
        b = self.out if b is None else b
        af.op_add_rmsnorm_fp8(self.x, self.r, self.g1, b["h1"], b["n1"], b["s1"], 1e-6, stream)
        af.op_linear_fp8(b["n1"], b["s1"], *self.up, b["a"], stream)
        af.op_quantize_fp8(b["a"], b["aq"], b["as_"], 1, stream)
        af.op_linear_fp8(b["aq"], b["as_"], *self.down, b["y"], stream)
        af.op_add_rmsnorm_fp8(b["y"], b["h1"], self.g2, b["h2"], b["n2"], b["s2"], 1e-6, stream)
        af.op_linear_fp8(b["n2"], b["s2"], *self.head, b["z"], stream)
        af.op_sample(b["z"], self.uniforms, b["tokens"], **self.settings, stream=stream)
        return b


def same(a, b):
    bits = lambda t: t.view(torch.uint8) if t.dtype is FP8 else t  # noqa: E731
    return all(torch.equal(bits(a[k]), bits(b[k])) for k in a)


def check_linear(y, xq, xs, w):
    """A result is a sum of K products, each exact before it is added.  An 8-bit product instruction adds
    eight neighbouring ones on a grid that ends 2^-13 below the largest of them: each is off by less than a
    step, so the eight by 2^-10 of the largest and all by 2^-10 of the sum of absolute terms.  The fp32 sums,
    K + blocks of them, and a block's two products add U32 each; a bf16 result is rounded once (2^-8 of it)."""
    want, absolute = linear_fp8(xq, xs, *w)
    K = xq.shape[1]
    bound = (K + 3 * blocks(K)) * U32 * absolute
    if y.dtype is BF16:
        bound = bound + 2.0 ** -10 * absolute + 2.0 ** -8 * np.abs(want)
    err = np.abs(to_np(y) - want)
    assert np.all(err <= bound), (float((err / np.maximum(absolute, 1e-30)).max()), y.dtype)


@pytest.mark.parametrize("M", [1, 7, 34, 282])
def test_one_behind_the_other(M):
    t = Tail(M)
    b = t.run()
    torch.cuda.synchronize()
    assert torch.equal(b["h1"], (t.x.float() + t.r.float()).to(BF16))
    check_fp8(b["n1"], b["s1"], rmsnorm(to_np(b["h1"]), to_np(t.g1), 1e-6), 1, norm_rel(t.D))
    check_linear(b["a"], b["n1"], b["s1"], t.up)
    check_fp8(b["aq"], b["as_"], to_np(b["a"]), 1, 0.0)
    check_linear(b["y"], b["aq"], b["as_"], t.down)
    assert torch.equal(b["h2"], (b["y"].float() + b["h1"].float()).to(BF16))
    check_fp8(b["n2"], b["s2"], rmsnorm(to_np(b["h2"]), to_np(t.g2), 1e-6), 1, norm_rel(t.D))
    check_linear(b["z"], b["n2"], b["s2"], t.head)
    z, u = to_np(b["z"]), t.uniforms.cpu().numpy()
    want = [sample_row(z[r], u[r], t=np.float32(0.9), k=50, p=np.float32(0.95)) for r in range(M)]
    assert b["tokens"].cpu().tolist() == want


@pytest.mark.parametrize("M", [1, 7, 282])
def test_captured_and_replayed(M):
    t = Tail(M, tag=1)
    t.run()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        t.run()
    for turn in range(4):  # inputs change in place; eager work of the program in between
        t.x.copy_(wl.draw(("tog_new", turn, M), (M, t.D), dtype=BF16, device="cuda"))
        t.uniforms.uniform_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(t.out, t.run(t.buffers())), turn
        torch.cuda.synchronize()


def test_two_graphs_and_two_streams_at_once():
    a, b = Tail(34, tag=2), Tail(7, tag=3)
    want = [{k: v.clone() for k, v in t.run().items()} for t in (a, b)]
    torch.cuda.synchronize()
    streams, graphs = [torch.cuda.Stream() for _ in range(2)], []
    for t, s in zip((a, b), streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            t.run()
        graphs.append(g)
    for turn in range(3):
        for t in (a, b):
            for v in t.out.values():
                v.view(torch.uint8).zero_()
        torch.cuda.synchronize()
        for t, s, g in zip((a, b), streams, graphs):
            if turn == 0:
                t.run(stream=s)  # the stream as an argument
            else:
                with torch.cuda.stream(s):
                    g.replay() if turn == 1 else t.run()
        torch.cuda.synchronize()
        assert same(a.out, want[0]) and same(b.out, want[1]), turn


def test_a_stream_of_another_device_is_refused():
    t = Tail(2)
    other = types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0)
    for call in (lambda: af.op_quantize_fp8(t.x, t.out["n1"], t.out["s1"], 1, other),
                 lambda: af.op_sample(t.out["z"], t.uniforms, t.out["tokens"], stream=other),
                 lambda: af.op_linear_fp8(t.out["n1"], t.out["s1"], *t.up, t.out["a"], other),
                 lambda: af.op_add_rmsnorm_fp8(t.x, None, t.g1, None, t.out["n1"], t.out["s1"], 1e-6, other)):
        with pytest.raises(ValueError, match="the stream is of cuda:1"):
            call()


# ----------------------------------------------------------------------------- the pipeline
def run_pipeline(P, sampling, seed=0, n_steps=6):
    shape, K, L_P = wl.TINY, 3, 16
    g, layers = wl.model_weights(shape, seed=0, device="cuda", random_gains=True)
    w = af.Weights(shape, g, layers)
    ring = af.Ring(shape.n_layers, P * K + P, L_P + K, shape.n_heads, shape.head_dim, dtype=F32)
    embeds = wl.draw(("tog_pipe", P), (P * (L_P + K - 1), shape.d_model), device="cuda", dtype=F32)
    pids = torch.full((L_P,), -1, dtype=torch.int32, device="cuda")
    pids[-4:] = torch.arange(4, dtype=torch.int32)
    pipe = Pipeline(w, ring, K, pids, lambda t: embeds, keep_logits=True, n_pipes=P, sampling=sampling,
                    sampling_seed=seed)
    steps = []
    for t in range(n_steps):
        n_in = pipe.ids[t % 2][P * L_P:].clone()
        res = pipe.step()
        torch.cuda.synchronize()
        u = pipe.uniforms[:len(res.segments)].clone().cpu() if sampling is not None else None
        steps.append((res.tokens.cpu().tolist(), to_np(res.logits), u, n_in.cpu().tolist()))
    w.close()
    ring.close()
    return steps


@pytest.mark.parametrize("P", [1, 2])
def test_pipeline_draws_its_tokens(P):
    settings = dict(temperature=1.5, top_k=40, top_p=0.9, min_p=0.01)
    steps = run_pipeline(P, settings)
    name = {"temperature": "t", "top_k": "k", "top_p": "p", "min_p": "m"}
    plain = {name[k]: v if k == "top_k" else np.float32(v) for k, v in settings.items()}
    seen = set()
    for t, (tokens, z, u, fed) in enumerate(steps):
        assert len(set(u.tolist())) == len(u) and u.tolist() != (steps[t - 1][2].tolist() if t else None)
        assert tokens == [sample_row(z[r], u[r], **plain) for r in range(len(tokens))]
        if t:  # what a step drew is what the next one is fed
            n = min(len(steps[t - 1][0]), 2 * P)
            assert fed[:n] == steps[t - 1][0][:n]
        seen.update(tokens)
    assert [s[0] for s in run_pipeline(P, settings)] == [s[0] for s in steps]      # by its seed
    assert [s[0] for s in run_pipeline(P, settings, seed=1)] != [s[0] for s in steps]
    assert [s[0] for s in run_pipeline(P, dict(temperature=0.0))] == [s[0] for s in run_pipeline(P, None)]


# ----------------------------------------------------------------------------- offsets past 32 bits
ROWS, COLS = (1 << 20) + 3, 4096  # 2^32 elements and three rows


def ends(t, rows):
    """t with its first and its last rows set to `rows` (of twice as many), the rest as it came."""
    n = rows.shape[0] // 2
    t[:n], t[-n:] = rows[:n], rows[n:]
    return t


def test_long_norm_and_quantisation():
    x = ends(torch.empty(ROWS, COLS, dtype=BF16, device="cuda"), wl.draw(("long_x",), (10, COLS), device="cuda"))
    g = wl.draw(("long_g",), (COLS,), std=0.2, mean=1.0, device="cuda")
    q, s = torch.empty(ROWS, COLS, dtype=FP8, device="cuda"), torch.empty(ROWS, COLS // 128, device="cuda")
    both = lambda t: torch.cat([t[:5].cpu().view(torch.uint8), t[-5:].cpu().view(torch.uint8)]).view(t.dtype)  # noqa: E731
    v = to_np(torch.cat([x[:5], x[-5:]]))
    af.op_quantize_fp8(x, q, s, 1)
    check_fp8(both(q), both(s), v, 1, 0.0)
    af.op_add_rmsnorm_fp8(x, None, g, None, q, s, 1e-6)
    check_fp8(both(q), both(s), rmsnorm(v, to_np(g), 1e-6), 1, norm_rel(COLS))
    af.op_add_rmsnorm_fp8(x, x, g, x, q, s, 1e-6)
    assert torch.equal(x[-5:].cpu(), torch.from_numpy(2 * v[5:]).to(BF16))
    check_fp8(both(q), both(s), rmsnorm(2 * v, to_np(g), 1e-6), 1, norm_rel(COLS))
    sb = torch.empty(blocks(ROWS), COLS // 128, device="cuda")
    af.op_quantize_fp8(x, q, sb, 128)
    check_fp8(q[-3:], sb[-1:], to_np(x[-3:]), 128, 0.0)  # the last block has three rows


@pytest.mark.parametrize("long", ["rows", "columns"])
def test_long_projection(long):
    ends_q = torch.empty(10, COLS, dtype=FP8, device="cuda")
    ends_s = torch.empty(10, COLS // 128, device="cuda")
    af.op_quantize_fp8(wl.draw(("long_l",), (10, COLS), device="cuda"), ends_q, ends_s, 1)
    q = torch.empty(ROWS, COLS, dtype=FP8, device="cuda")
    ends(q.view(torch.uint8), ends_q.view(torch.uint8))
    few = torch.empty(24, COLS, dtype=FP8, device="cuda")
    if long == "rows":
        s = ends(torch.zeros(ROWS, COLS // 128, device="cuda"), ends_s)
        few_s = f32(1, COLS // 128)
        af.op_quantize_fp8(wl.draw(("long_w",), (24, COLS), device="cuda"), few, few_s, 128)
        y = torch.empty(ROWS, 24, dtype=BF16, device="cuda")
        af.op_linear_fp8(q, s, few, few_s, y)
        check_linear(torch.cat([y[:5], y[-5:]]), ends_q, ends_s, (few, few_s))
    else:
        s = f32(blocks(ROWS), COLS // 128)
        s[0], s[-1] = 0.01, 0.02
        few_s = f32(24, COLS // 128)
        af.op_quantize_fp8(wl.draw(("long_w",), (24, COLS), device="cuda"), few, few_s, 1)
        y = torch.empty(24, ROWS, dtype=F32, device="cuda")
        af.op_linear_fp8(few, few_s, q, s, y)
        check_linear(y[:, :5], few, few_s, (ends_q[:5], s[:1]))
        check_linear(y[:, -3:], few, few_s, (ends_q[-3:], s[-1:]))  # the last three are a block of their own


def test_long_batch_of_logits():
    n, V = (1 << 15) + 3, 1 << 17
    rows = wl.draw(("long_z",), (6, V), std=2.0, device="cuda")
    z = ends(torch.empty(n, V, dtype=BF16, device="cuda"), rows)
    u = torch.rand(n, generator=torch.Generator().manual_seed(3)).cuda()
    tokens = torch.zeros(n, dtype=torch.int32, device="cuda")
    top_p = torch.full((n,), 0.9, device="cuda")
    af.op_sample(z, u, tokens, top_p=top_p)
    at = [0, 1, 2, n - 3, n - 2, n - 1]
    rows, u, tokens = to_np(rows), u.cpu().numpy(), tokens.cpu().numpy()
    assert [int(tokens[i]) for i in at] == [sample_row(rows[j], u[i], p=np.float32(0.9)) for j, i in enumerate(at)]
