"""The sampler on rows that are not kept in LDS (more than 32768 logits), and around that border: masked rows, infinite,
equal and signed-zero logits, in both types."""
import pytest
import torch

from tests.test_gpu_sample import DT, INF, NAN, SETTINGS, check, draw, normal, uniforms

pytestmark = pytest.mark.gpu

LONG = [32767, 32768, 32769, 40000, 70001]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", LONG)
def test_masked_rows(V, dtype):
    lowest = torch.finfo(DT[dtype]).min
    z = normal((8, V), 51, dtype=DT[dtype])
    z[0] = -INF
    z[1] = NAN
    z[2, :V - 1] = -INF
    z[3, 1:] = -INF
    z[4, ::2] = -INF
    z[5, ::3] = NAN
    z[6, 5:] = lowest
    z[7] = lowest
    for s in SETTINGS + [dict(temperature=0.0), dict(temperature=INF), dict(top_k=V - 1), dict(top_p=0.5, min_p=0.5)]:
        check(z, [0.0, 0.37, 0.999, 0.0, 0.99, 0.5, 0.2, 0.7], **s)
    got, _, _ = draw(z, 0.5)
    assert got[:4] == [0, 0, V - 1, 0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", LONG)
def test_infinite_logits_share_the_row(V, dtype):
    z = normal((5, V), 52, dtype=DT[dtype])
    z[0, V - 2] = z[1, 3] = z[1, V // 2] = z[1, V - 1] = INF
    z[2, 10] = 3e38
    z[3, 10], z[3, 11] = 3e38, -3e38
    z[4, ::7], z[4, 1::7] = INF, NAN
    for s in SETTINGS + [dict(temperature=INF), dict(temperature=1e-30), dict(temperature=0.0), dict(top_k=2), dict(top_p=0.5)]:
        for u in (0.0, 0.4, 0.6, 0.99):
            check(z, u, **s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [32768, 40000])
def test_zeros_of_either_sign_and_a_value_below_them(V, dtype):
    z = torch.full((4, V), -1.0, dtype=DT[dtype], device="cuda")
    z[0, V // 3::5], z[0, V // 2::5] = 0.0, -0.0
    z[1, 10], z[1, V - 1] = -0.0, 0.0
    z[2, ::2] = -0.0
    z[3] = -0.0
    for s in (dict(), dict(top_k=1), dict(top_k=2), dict(top_k=5000), dict(top_p=0.4), dict(top_p=0.8, top_k=20000), dict(min_p=0.5),
              dict(temperature=0.0)):
        check(z, uniforms(4, 53), **s)
        check(z, 0.97, **s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("off", [1, 2, 3, 5])
def test_rows_at_any_alignment(dtype, off):
    V = 32771
    flat = normal((3 * V + off,), off, dtype=DT[dtype])
    z = flat[off:].view(3, V)
    for s in SETTINGS:
        check(z, uniforms(3, off), **s)
