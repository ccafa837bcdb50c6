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
