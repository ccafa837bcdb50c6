"""A pipeline on a stream of its own: which stream its device work is issued to (no GPU), and what it answers while the
current stream is behind (GPU)."""
import contextlib
import types

import pytest
import torch

import workload as wl

af = pytest.importorskip("paper_2512_20276_amd")
from paper_2512_20276_amd import naive_pipe as npipe  # noqa: E402
from paper_2512_20276_amd import pipeline as pl  # noqa: E402


class Streams:
    """Stands for torch.cuda's streams: which is current, and who waits for whom."""

    def __init__(self, monkeypatch):
        self.current, self.log = "caller's", []
        monkeypatch.setattr(torch.cuda, "stream", self.entered)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.current)
        for name in ("zeros", "empty", "full"):
            monkeypatch.setattr(torch, name, self.noted(name, getattr(torch, name)))

    @contextlib.contextmanager
    def entered(self, stream):
        before, self.current = self.current, self.current if stream is None else stream
        yield
        self.current = before

    def noted(self, what, fn):
        def call(*args, **kw):
            self.log.append((what, self.current))
            return fn(*args, **kw)
        return call


class OnGpu(torch.Tensor):
    """A CPU tensor that says that it is on a GPU."""
    is_cuda = True
    record_stream = lambda self, stream: self.recorded.append(stream)  # noqa: E731


@pytest.mark.parametrize("sampling", [None, dict(temperature=0.7, top_k=5)])
@pytest.mark.parametrize("own", [True, False])
def test_device_work_goes_to_the_stream_of_the_pipeline(monkeypatch, sampling, own):
    w = types.SimpleNamespace(shape=wl.TINY, dtype=torch.float32)
    waits, ring = [], af.Ring(0, 6, 16)
    pids = torch.full((4,), -1, dtype=torch.int32).as_subclass(OnGpu)
    pids.recorded = []
    streams = Streams(monkeypatch)
    mine = types.SimpleNamespace(wait_stream=waits.append, synchronize=lambda: streams.log.append(("sync", "mine")))
    stream, at = (mine, mine) if own else (None, "caller's")
    pipe = pl.Pipeline(w, ring, 2, pids, lambda t: streams.log.append(("embeds", streams.current)) or torch.zeros(5, 4),
                       stream=stream, sampling=sampling)
    assert all(s == at for _, s in streams.log) and len(streams.log) >= (3 if sampling is None else 7)
    assert waits == (["caller's"] if own else []) and pids.recorded == ([mine] if own else [])

    ran = []
    monkeypatch.setattr(pl, "packed_forward", lambda *a: ran.append(a[-1]))
    monkeypatch.setattr(pl, "op_sample", lambda *a, stream=None, **kw: ran.append(stream))
    monkeypatch.setattr(torch.Tensor, "uniform_", streams.noted("uniform_", torch.Tensor.uniform_))
    monkeypatch.setattr(torch.Tensor, "clone", streams.noted("clone", torch.Tensor.clone))
    del streams.log[:]
    pipe.step()
    assert ran == [stream] * (1 if sampling is None else 2)
    log = [e for e in streams.log if e[0] in ("embeds", "uniform_", "clone")]
    assert log == [("embeds", "caller's")] + ([("uniform_", at)] if sampling else []) + [("clone", at)]
    pipe.request_tokens(0)
    assert (("sync", "mine") in streams.log) == own


@pytest.mark.parametrize("own", [True, False])
def test_naive_pipeline_reads_its_tokens_on_its_stream(monkeypatch, own):
    w = types.SimpleNamespace(shape=wl.TINY, dtype=torch.float32)
    staging = af.Ring(0, 2, 16)
    staging.copy_kv_to = lambda *a: None
    monkeypatch.setattr(npipe, "Ring", lambda *a: staging)
    for name in ("op_embed", "packed_layer_forward", "op_lm_head_argmax"):
        monkeypatch.setattr(npipe, name, lambda *a, **kw: None)
    stream = types.SimpleNamespace(synchronize=lambda: None) if own else None
    pipe = npipe.NaivePipeline(w, 2, torch.full((4,), -1, dtype=torch.int32), lambda t: torch.zeros(5, 4), False, stream=stream)
    pipe.tokens.zero_()
    streams = Streams(monkeypatch)
    monkeypatch.setattr(torch.Tensor, "cpu", streams.noted("cpu", torch.Tensor.cpu))
    pipe.step()
    assert [e for e in streams.log if e[0] == "cpu"] == [("cpu", stream if own else "caller's")]


@pytest.mark.gpu
@pytest.mark.parametrize("sampling", [None, dict(temperature=1.5, top_k=40)])
def test_answers_do_not_depend_on_the_stream(sampling):
    shape, K, L_P = wl.TINY, 3, 16
    g, layers = wl.model_weights(shape, seed=0, device="cuda", random_gains=True)
    w = af.Weights(shape, g, layers)
    embeds = wl.draw(("own_stream",), (L_P + K - 1, shape.d_model), device="cuda", dtype=torch.float32)

    def run(stream, late):
        ring = af.Ring(shape.n_layers, K + 1, L_P + K, shape.n_heads, shape.head_dim, dtype=torch.float32)
        torch.cuda.synchronize()
        if late:  # the current stream is some milliseconds behind, with the ids among what it has yet to write
            torch.cuda._sleep(20_000_000)
        pids = torch.full((L_P,), -1, dtype=torch.int32, device="cuda")
        pids[-4:] = torch.arange(4, dtype=torch.int32, device="cuda")
        pipe = pl.Pipeline(w, ring, K, pids, lambda t: embeds, stream=stream, sampling=sampling, sampling_seed=3)
        del pids
        if late:
            torch.cuda._sleep(20_000_000)
        for _ in range(5):
            pipe.step()
        got = [pipe.request_tokens(r) for r in range(3)]
        torch.cuda.synchronize()
        ring.close()
        return got

    want = run(None, False)
    assert run(torch.cuda.Stream(), False) == want
    assert run(torch.cuda.Stream(), True) == want
    w.close()
