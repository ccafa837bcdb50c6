"""CPU tests of what the operators over a paged key-value cache refuse on the host, before any launch, and of the
workspace they ask for."""
import ctypes as C
import math

import pytest
import torch

import paper_2512_20276_amd as af

lib = af.lib
P = 1 << 20  # an aligned address that no refused call ever follows
INV, UNS = af.AF_ERR_INVALID_ARG, af.AF_ERR_UNSUPPORTED


def desc(**at):
    d = dict(k=P, v=P, page_table=P, kv_lens=P, q_starts=None, n_pages=9, page_size=16, n_kv_heads=2, head_dim=64, n_seq=3,
             max_pages=4, dtype=af.AF_BF16, reserved=0)
    return af.PagedKVDesc(**{**d, **at})


def append_args(d, **at):
    a = dict(kv=C.byref(d), q=P, q_stride=256, k=P, k_stride=128, v=P, v_stride=128, positions=None, sections=None, n_axes=1,
             theta=1e4, q_out=P, q_out_stride=256, M=3, n_heads=4, stream=None)
    return list({**a, **at}.values())


def attend_args(d, **at):
    a = dict(kv=C.byref(d), q=P, q_stride=256, o=P, o_stride=256, lse=None, M=3, n_heads=4, scale=0.1, window=0, n_sink=0,
             workspace=None, workspace_bytes=0, stream=None)
    return list({**a, **at}.values())


def refused(code, says, fn, args):
    assert fn(*args) == code, af.last_error()
    assert says in af.last_error() and af.last_error().startswith("af_"), af.last_error()


@pytest.mark.parametrize("code,says,at", [
    (INV, "dtype", dict(dtype=2)), (INV, "reserved", dict(reserved=1)),
    (INV, "non-NULL", dict(k=None)), (INV, "non-NULL", dict(v=None)), (INV, "non-NULL", dict(page_table=None)),
    (INV, "non-NULL", dict(kv_lens=None)), (INV, "positive", dict(n_pages=0)), (INV, "positive", dict(page_size=0)),
    (INV, "positive", dict(page_size=-16)), (INV, "positive", dict(n_kv_heads=0)), (INV, "positive", dict(n_seq=-1)),
    (INV, "positive", dict(max_pages=0)), (INV, "multiple", dict(n_kv_heads=3)), (INV, "n_seq", dict(n_seq=2)),
    (INV, "aligned", dict(page_table=P + 2)), (INV, "aligned", dict(kv_lens=P + 1)), (INV, "aligned", dict(q_starts=P + 3)),
    (UNS, "head_dim", dict(head_dim=96)), (UNS, "head_dim", dict(head_dim=256)), (UNS, "page_size", dict(page_size=4)),
    (UNS, "page_size", dict(page_size=24)), (UNS, "2^30", dict(max_pages=(1 << 26) + 1)),
    (UNS, "16-byte", dict(k=P + 8)), (UNS, "16-byte", dict(v=P + 2)),
])
def test_a_cache_is_refused(code, says, at):
    d = desc(**at)
    n = C.c_size_t()
    refused(code, says, lib.af_op_rope_append_paged, append_args(d))
    refused(code, says, lib.af_op_attention_paged, attend_args(d))
    refused(code, says, lib.af_attention_paged_workspace, [C.byref(d), 3, 4, C.byref(n)])


def test_sizes_that_no_launch_takes():
    d = desc(q_starts=P, n_seq=1 << 20, max_pages=1 << 20)
    refused(UNS, "2^31", lib.af_op_attention_paged, attend_args(d))
    refused(UNS, "2^30", lib.af_op_attention_paged, attend_args(desc(q_starts=P), M=1 << 29))
    refused(UNS, "2^24", lib.af_op_rope_append_paged, append_args(desc(q_starts=P), M=1 << 24))
    refused(UNS, "launch", lib.af_op_attention_paged,
            attend_args(desc(n_seq=1 << 23, n_kv_heads=8), M=1 << 23, n_heads=8, q_stride=512, o_stride=512))


def test_append_refuses():
    fn, d = lib.af_op_rope_append_paged, desc()
    three = (C.c_int32 * 3)(16, 8, 8)
    refused(INV, "kv must", fn, append_args(d, kv=None))
    for n in ("q", "k", "v", "q_out"):
        refused(INV, f"{n} must be non-NULL", fn, append_args(d, **{n: None}))
        refused(UNS, f"rows of {n}", fn, append_args(d, **{n: P + 8}))
        refused(INV, f"rows of {n}", fn, append_args(d, **{n + "_stride": 120}))
        refused(INV, f"rows of {n}", fn, append_args(d, **{n + "_stride": 0}))
        refused(UNS, f"rows of {n}", fn, append_args(d, **{n + "_stride": 260}))
        refused(INV, f"rows of {n}", fn, append_args(d, **{n + "_stride": 1 << 32}))
    for n_axes in (0, 4, -1):
        refused(INV, "n_axes", fn, append_args(d, n_axes=n_axes, positions=P, sections=three))
    refused(INV, "several axes", fn, append_args(d, n_axes=3, sections=three))
    refused(INV, "several axes", fn, append_args(d, n_axes=3, positions=P))
    refused(INV, "aligned", fn, append_args(d, positions=P + 2))
    for bad in ((16, 8, 9), (16, 8, 7), (33, -1, 0), (0, 0, 0), (2 ** 31 - 1, 2 ** 31 - 1, 34)):
        refused(INV, "sections", fn, append_args(d, n_axes=3, positions=P, sections=(C.c_int32 * 3)(*bad)))
    for theta in (0.0, -1.0, math.inf, math.nan):
        refused(INV, "theta", fn, append_args(d, theta=theta))
    refused(INV, "positive", fn, append_args(d, M=0))
    refused(INV, "positive", fn, append_args(d, n_heads=0))


def test_attention_refuses():
    fn, d = lib.af_op_attention_paged, desc()
    for n in ("q", "o"):
        refused(INV, f"{n} must be non-NULL", fn, attend_args(d, **{n: None}))
        refused(UNS, f"rows of {n}", fn, attend_args(d, **{n: P + 4}))
        refused(INV, f"rows of {n}", fn, attend_args(d, **{n + "_stride": 255}))
    refused(INV, "window", fn, attend_args(d, window=-1))
    refused(INV, "n_sink", fn, attend_args(d, n_sink=-1))
    for scale in (math.inf, math.nan, 3e38):
        refused(INV, "scale", fn, attend_args(d, scale=scale))
    refused(INV, "aligned", fn, attend_args(d, lse=P + 2))
    long = desc(max_pages=100)
    n = C.c_size_t()
    assert lib.af_attention_paged_workspace(C.addressof(long), 3, 4, C.byref(n)) == af.AF_OK and n.value > 0
    refused(INV, "workspace", fn, attend_args(long))
    refused(INV, "workspace", fn, attend_args(long, workspace=P, workspace_bytes=n.value - 1))
    refused(INV, "16-byte", fn, attend_args(long, workspace=P + 8, workspace_bytes=n.value))
    refused(INV, "bytes", lib.af_attention_paged_workspace, [C.addressof(long), 3, 4, None])


def test_workspace():
    """Short tables of single rows need none, long ones some, and it is bounded whatever the sizes are."""
    n = C.c_size_t()
    for max_pages, page, M, n_seq, starts, Hkv, group in ((4, 16, 3, 3, None, 2, 2), (4000, 64, 300, 300, None, 8, 4), (1 << 20, 256, 1, 1, None, 1, 64),
                                                         (500, 64, 900, 32, P, 8, 4), (500, 64, 1 << 16, 2, P, 32, 1)):
        d = desc(max_pages=max_pages, page_size=page, n_seq=n_seq, q_starts=starts, n_kv_heads=Hkv, head_dim=128)
        assert lib.af_attention_paged_workspace(C.addressof(d), M, Hkv * group, C.byref(n)) == af.AF_OK, af.last_error()
        assert n.value % 16 == 0 and n.value <= 256 << 20
        assert (n.value == 0) == (max_pages * page <= 512 and starts is None)


def test_binding_refuses_before_the_library_is_called():
    f = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    good = dict(k=f(9, 2, 16, 64), v=f(9, 2, 16, 64), page_table=i(3, 4), kv_lens=i(3), q_starts=i(4))
    for n, bad in (("v", f(9, 2, 16, 32)), ("v", f(9, 2, 16, 64, dt=torch.float32)), ("k", f(9, 2, 16)), ("k", f(9, 2, 64, 16).transpose(2, 3)),
                   ("page_table", f(3, 4)), ("page_table", i(4, 3).t()), ("page_table", i(12)), ("kv_lens", i(4)), ("kv_lens", i(3).long()),
                   ("q_starts", i(3))):
        with pytest.raises(ValueError, match="must be"):
            af.PagedKV(**{**good, n: bad})
    with pytest.raises(ValueError, match="dtype"):
        af.PagedKV(f(9, 2, 16, 64, dt=torch.float16), f(9, 2, 16, 64, dt=torch.float16), i(3, 4), i(3))
    kv = af.PagedKV(**good)
    rows = dict(q=f(5, 4, 64), k=f(5, 2, 64), v=f(5, 2, 64), q_out=f(5, 4, 64), theta=1e4)
    with pytest.raises(ValueError, match="on a GPU"):
        af.op_rope_append_paged(kv, **rows)
    for n, bad in (("q", f(5, 4, 32)), ("q", f(5, 4, 128)[..., ::2]), ("k", f(5, 4, 64)), ("v", f(4, 2, 64)), ("q_out", f(5, 2, 64)),
                   ("k", f(5, 2, 64, dt=torch.float32)), ("v", f(5, 64, 2).transpose(1, 2)), ("q", f(4, 5, 64).transpose(0, 1)),
                   ("positions", i(4)), ("positions", i(5, 3).long()), ("sections", [16, 16])):
        with pytest.raises(ValueError, match="must be|axes"):
            af.op_rope_append_paged(kv, **{**rows, n: bad})
    rows = dict(q=f(5, 4, 64), o=f(5, 4, 64), scale=0.1, workspace=None)
    with pytest.raises(ValueError, match="on a GPU"):
        af.op_attention_paged(kv, **rows)
    for n, bad in (("o", f(5, 4, 64, dt=torch.float32)), ("o", f(6, 4, 64)), ("lse", f(5, 4)), ("lse", f(5, 3, dt=torch.float32)),
                   ("workspace", f(1000)), ("workspace", torch.zeros(1000, dtype=torch.uint8)[::2])):
        with pytest.raises(ValueError, match="must be"):
            af.op_attention_paged(kv, **{**rows, n: bad})
