"""CPU tests of what the 8-bit operators and the sampler refuse on the host, before any launch."""
import ctypes as C

import pytest
import torch

import paper_2512_20276_amd as af

lib = af.lib
P = 1 << 20  # an aligned address that no refused call ever follows


def refused(code, fn, *args, says=None):
    assert fn(*args) == code, af.last_error()
    if says:
        assert says in af.last_error()


def test_norm_refuses():
    ok = [af.AF_BF16, P, P, P, P, P, P, 4, 256, 1e-6, None]
    fn = lib.af_op_add_rmsnorm_fp8

    def bad(code, says=None, **at):
        names = ["dtype", "x", "resid", "g", "out", "q", "scales", "M", "D", "eps", "stream"]
        args = list(ok)
        for n, v in at.items():
            args[names.index(n)] = v
        refused(code, fn, *args, says=says)

    inv, uns = af.AF_ERR_INVALID_ARG, af.AF_ERR_UNSUPPORTED
    bad(inv, "dtype", dtype=2)
    for n in ("x", "g", "q", "scales"):
        bad(inv, "non-NULL", **{n: None})
    bad(inv, "both or neither", resid=None)
    bad(inv, "both or neither", out=None)
    for M, D in ((0, 256), (-1, 256), (4, 0), (4, -8)):
        bad(inv, "positive", M=M, D=D)
    bad(inv, "aligned", x=P + 1)
    bad(inv, "aligned", scales=P + 2)
    bad(uns, "rows", M=1 << 23)


def test_quantize_refuses():
    fn, inv, uns = lib.af_op_quantize_fp8, af.AF_ERR_INVALID_ARG, af.AF_ERR_UNSUPPORTED
    refused(inv, fn, 7, P, P, P, 4, 256, 1, None, says="dtype")
    refused(inv, fn, af.AF_F32, None, P, P, 4, 256, 1, None)
    refused(inv, fn, af.AF_F32, P, P, None, 4, 256, 1, None)
    refused(inv, fn, af.AF_F32, P, P, P, 0, 256, 1, None)
    refused(inv, fn, af.AF_F32, P, P, P, 4, 0, 1, None)
    refused(inv, fn, af.AF_F32, P, P, P, 4, 256, 64, None, says="block_rows")
    refused(inv, fn, af.AF_F32, P + 2, P, P, 4, 256, 1, None, says="aligned")
    refused(uns, fn, af.AF_F32, P, P, P, 1 << 28, 128, 1, None, says="blocks")
    refused(uns, fn, af.AF_F32, P, P, P, 0x7fffffff, 0x7fffffff, 128, None, says="blocks")


def test_linear_refuses():
    fn, inv, uns = lib.af_op_linear_fp8, af.AF_ERR_INVALID_ARG, af.AF_ERR_UNSUPPORTED
    refused(inv, fn, P, P, P, P, P, 2, 4, 16, 256, None, says="out_dtype")
    for i in range(5):
        args = [P] * 5
        args[i] = None
        refused(inv, fn, *args, af.AF_BF16, 4, 16, 256, None, says="non-NULL")
    for M, N, K in ((0, 16, 256), (4, 0, 256), (4, 16, 0), (-4, 16, 256)):
        refused(inv, fn, P, P, P, P, P, af.AF_BF16, M, N, K, None, says="positive")
    refused(inv, fn, P, P + 1, P, P, P, af.AF_BF16, 4, 16, 256, None, says="aligned")
    refused(inv, fn, P, P, P, P, P + 2, af.AF_F32, 4, 16, 256, None, says="aligned")
    refused(uns, fn, P, P, P, P, P, af.AF_BF16, 4, 16, 8, None, says="K % 16")
    refused(uns, fn, P + 8, P, P, P, P, af.AF_BF16, 4, 16, 256, None, says="16-byte")
    refused(uns, fn, P, P, P + 4, P, P, af.AF_BF16, 4, 16, 256, None, says="16-byte")
    refused(uns, fn, P, P, P, P, P, af.AF_BF16, 4, 16, (1 << 22) + 16, None, says="columns")
    refused(uns, fn, P, P, P, P, P, af.AF_BF16, 0x7fffffff, 0x7fffffff, 256, None, says="tiles")


def test_sample_refuses():
    fn, inv, uns = lib.af_op_sample, af.AF_ERR_INVALID_ARG, af.AF_ERR_UNSUPPORTED
    tail = (None, None, None, None, P, P, None)
    refused(inv, fn, 5, P, 4, 100, *tail, says="dtype")
    refused(inv, fn, af.AF_F32, None, 4, 100, *tail, says="non-NULL")
    refused(inv, fn, af.AF_F32, P, 4, 100, None, None, None, None, None, P, None, says="non-NULL")
    refused(inv, fn, af.AF_F32, P, 4, 100, None, None, None, None, P, None, None, says="non-NULL")
    refused(inv, fn, af.AF_F32, P, 0, 100, *tail, says="positive")
    refused(inv, fn, af.AF_F32, P, 4, 0, *tail, says="positive")
    refused(inv, fn, af.AF_F32, P + 2, 4, 100, *tail, says="aligned")
    refused(inv, fn, af.AF_F32, P, 4, 100, P + 1, None, None, None, P, P, None, says="aligned")
    refused(uns, fn, af.AF_F32, P, 4, (1 << 22) + 1, *tail, says="tokens")
    refused(uns, fn, af.AF_F32, P, 1 << 22, 100, *tail, says="rows")


def test_binding_refuses_before_the_library_is_called():
    """Shapes, types, layouts and devices that would have the library read or write outside a tensor."""
    f = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    q8 = lambda *s: torch.zeros(s, dtype=torch.uint8).view(af.FP8)  # noqa: E731
    good = dict(x=f(4, 256), resid=f(4, 256), g=f(256), resid_out=f(4, 256), q=q8(4, 256), scales=f(4, 2), eps=1e-6)
    with pytest.raises(ValueError, match="on a GPU"):
        af.op_add_rmsnorm_fp8(**good)
    for n, v in (("g", f(255)), ("q", q8(4, 255)), ("q", f(4, 256)), ("scales", f(4, 1)), ("resid", f(3, 256)),
                 ("resid_out", f(4, 256, dt=torch.bfloat16)), ("x", f(256, 4).t()), ("resid_out", None)):
        with pytest.raises(ValueError, match="must be|go together"):
            af.op_add_rmsnorm_fp8(**{**good, n: v})
    with pytest.raises(ValueError, match="block_rows"):
        af.op_quantize_fp8(f(4, 256), q8(4, 256), f(4, 2), 64)
    with pytest.raises(ValueError, match="scales"):
        af.op_quantize_fp8(f(130, 256), q8(130, 256), f(1, 2), 128)
    with pytest.raises(ValueError, match="ws"):
        af.op_linear_fp8(q8(4, 256), f(4, 2), q8(130, 256), f(1, 2), f(4, 130))
    with pytest.raises(ValueError, match="wq"):
        af.op_linear_fp8(q8(4, 256), f(4, 2), q8(130, 240), f(2, 2), f(4, 130))
    with pytest.raises(ValueError, match="unsupported dtype|on a GPU"):
        af.op_linear_fp8(q8(4, 256), f(4, 2), q8(130, 256), f(2, 2), f(4, 130, dt=torch.float16))
    for kw in (dict(uniforms=f(3)), dict(tokens=f(4)), dict(top_k=f(4)), dict(temperature=f(5)), dict(logits=f(4, 9)[:, :8])):
        args = dict(logits=f(4, 9), uniforms=f(4), tokens=f(4, dt=torch.int32))
        with pytest.raises(ValueError, match="must be"):
            af.op_sample(**{**args, **kw})


def test_every_refusal_leaves_its_message():
    assert lib.af_op_sample(9, None, 0, 0, *([None] * 7)) == af.AF_ERR_INVALID_ARG
    assert af.last_error().startswith("af_op_sample:")
    assert C.c_int32(lib.af_op_linear_fp8(*([None] * 5), 1, 1, 1, 16, None)).value == af.AF_ERR_INVALID_ARG
    assert af.last_error().startswith("af_op_linear_fp8:")
