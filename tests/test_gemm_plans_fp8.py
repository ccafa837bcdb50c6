"""Which kernel an 8-bit projection takes, on the CPU."""
import ctypes as C
import random

import pytest

import paper_2512_20276_amd as af
from tests.test_gpu_fp8 import KERNEL_SHAPES, LINEAR_SHAPES

_plan = af.lib["_ZN2af13gemm_fp8_planEiiii"]
_plan.restype, _plan.argtypes = C.c_int, [C.c_int] * 4


def plan(out, M, N, K):
    return _plan(out, M, N, K)


@pytest.mark.parametrize("out,n", [(af.AF_BF16, 14), (af.AF_F32, 12)])
def test_shapes_reach_every_kernel(out, n):
    """The shapes of the exactness test run every kernel that any call reaches."""
    rng = random.Random(7)
    reached = set()
    for _ in range(20000):
        M, N = int(2 ** rng.uniform(0, 11.2)), int(2 ** rng.uniform(0, 15))
        reached.add(plan(out, M, N, 16 * int(2 ** rng.uniform(0, 10))))
    assert reached == set(range(n))
    assert {plan(out, *s) for s in LINEAR_SHAPES + KERNEL_SHAPES} == reached


@pytest.mark.parametrize("M,N,K,kernel", [
    (7, 32000, 4096, 1),     # 16 x 32 streamed 26.3 us; 16 x 16 32
    (1, 4096, 4096, 0),      # 16 x 16 streamed 4.7; 16 x 32 6.3
    (64, 4096, 4096, 3),     # 32 x 32, four groups 10.3; 64 x 64 12.4
    (282, 4096, 11008, 7),   # 96 x 64 33.1; 64 x 64 39.6
    (282, 22016, 4096, 11),  # 160 x 256 55.3; 256 x 256 59.7
    (1000, 4096, 4096, 8),   # 128 x 128 25.7; 160 x 128 26.9
    (2264, 22016, 4096, 13),  # 288 x 256 212; 256 x 256 237
])
def test_kernels_of_timed_shapes(M, N, K, kernel):
    assert plan(af.AF_BF16, M, N, K) == kernel


def test_many_rows_never_stream():
    rng = random.Random(3)
    for _ in range(3000):
        M, N, K = rng.randint(33, 4096), rng.randint(1, 40000), 16 * rng.randint(1, 1000)
        assert plan(af.AF_BF16, M, N, K) >= 3 and plan(af.AF_F32, M, N, K) >= 3
