"""Argument checks of the pipeline's sampling and of the operators' largest launches (no GPU)."""
import types

import pytest
import torch

import workload as wl

af = pytest.importorskip("paper_2512_20276_amd")
from paper_2512_20276_amd.pipeline import Pipeline  # noqa: E402

P = 0x10000  # stands for a device pointer; never read


def test_pipeline_refuses_unknown_settings():
    w = types.SimpleNamespace(shape=wl.TINY, dtype=torch.float32)
    with pytest.raises(ValueError, match="sampling takes temperature"):
        Pipeline(w, None, 3, torch.zeros(4, dtype=torch.int32), lambda t: None, sampling=dict(top_n=3))


def test_pipeline_keeps_its_settings_per_row():
    w = types.SimpleNamespace(shape=wl.TINY, dtype=torch.float32)
    pids = torch.zeros(4, dtype=torch.int32)
    pipe = Pipeline(w, None, 3, pids, lambda t: None, n_pipes=2, sampling=dict(temperature=0.5, top_k=7))
    assert pipe.sampling["temperature"].tolist() == [0.5] * 6 and pipe.sampling["top_k"].tolist() == [7] * 6
    assert pipe.sampling["top_k"].dtype is torch.int32 and pipe.logits.shape == (6, wl.TINY.vocab)
    assert Pipeline(w, None, 3, pids, lambda t: None).logits is None


@pytest.mark.parametrize("fn,args,says", [
    ("af_op_quantize_fp8", (1, P, P, P, (1 << 28) - 15, 128, 1), "blocks"),
    ("af_op_quantize_fp8", (1, P, P, P, 1 << 21, 128 * 128, 1), "blocks"),
    ("af_op_quantize_fp8", (1, P, P, P, 1 << 24, 128 * 128, 128), "blocks"),
    ("af_op_linear_fp8", (P, P, P, P, P, 1, 1, 1 << 27, 16), "tiles"),
    ("af_op_linear_fp8", (P, P, P, P, P, 1, 1 << 27, 1, 16), "tiles"),
    ("af_op_linear_fp8", (P, P, P, P, P, 1, 1 << 16, 1 << 15, 16), "tiles"),
])
def test_launches_of_2_32_work_items_are_refused(fn, args, says):
    assert getattr(af.lib, fn)(*args, None) == af.AF_ERR_UNSUPPORTED
    assert says in af.last_error()
