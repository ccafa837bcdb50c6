"""GPU parity of the sampler with its definition in 64 bits: tokens have to be equal."""
import numpy as np
import pytest
import torch

from tests.plain_ops import sample_row

pytestmark = pytest.mark.gpu

af = pytest.importorskip("paper_2512_20276_amd")

INF, NAN = float("inf"), float("nan")
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def draw(logits, u, **settings):
    """Tokens of the rows; settings are scalars, lists or None."""
    n = logits.shape[0]
    per_row = {}
    for name, v in settings.items():
        dt = torch.int32 if name == "top_k" else torch.float32
        per_row[name] = None if v is None else torch.as_tensor(v, dtype=dt).expand(n).contiguous().cuda()
    tokens = torch.full((n + 1,), -5, dtype=torch.int32, device="cuda")
    uniforms = torch.as_tensor(u, dtype=torch.float32).expand(n).contiguous().cuda()
    af.op_sample(logits, uniforms, tokens[:n], **per_row)
    got = tokens.cpu()
    assert got[n] == -5
    return got[:n].tolist(), uniforms.cpu(), {k: None if v is None else v.cpu() for k, v in per_row.items()}


def check(logits, u, **settings):
    got, uniforms, per_row = draw(logits, u, **settings)
    z = logits.detach().float().cpu().numpy()
    names = {"temperature": "t", "top_k": "k", "top_p": "p", "min_p": "m"}
    for r in range(z.shape[0]):
        want = sample_row(z[r], uniforms[r], **{names[k]: v[r].item() for k, v in per_row.items() if v is not None})
        assert got[r] == want, (r, got[r], want, float(uniforms[r]), {k: v[r].item() for k, v in per_row.items() if v is not None})


def normal(shape, seed, std=2.0, dtype=torch.float32):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def uniforms(n, seed):
    gen = torch.Generator()
    gen.manual_seed(seed)
    return torch.rand(n, generator=gen)


SETTINGS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=50, temperature=0.8), dict(top_p=0.9),
            dict(min_p=0.05), dict(top_k=300, top_p=0.95, temperature=1.2), dict(top_p=0.8, min_p=0.1),
            dict(top_k=40, min_p=0.02), dict(temperature=1.5, top_k=2000, top_p=0.99, min_p=0.001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 63, 64, 65, 512, 1000, 1023, 1024, 1025, 4097, 32000])
@pytest.mark.parametrize("settings", SETTINGS, ids=str)
def test_sample(dtype, V, settings):
    """bf16 logits have many equal ones, so that cuts fall between tokens of one value."""
    check(normal((9, V), V, dtype=DT[dtype]), uniforms(9, V + 1), **settings)


@pytest.mark.parametrize("V", [32001, 50000, 65536, 100003, 131072, 262147])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=64, top_p=0.9), dict(top_p=0.95), dict(min_p=0.01), dict(top_k=20000)], ids=str)
def test_sample_long_vocabulary(V, settings):
    check(normal((3, V), V), uniforms(3, V), **settings)


@pytest.mark.parametrize("rows", [1, 5, 64, 300])
def test_every_row_has_settings_of_its_own(rows):
    gen = torch.Generator()
    gen.manual_seed(rows)
    r = lambda lo, hi: torch.rand(rows, generator=gen) * (hi - lo) + lo  # noqa: E731
    t, k, p, m = r(0.3, 2.0), r(-5, 400).int(), r(0.3, 1.2), r(-0.1, 0.3)
    t[::7] = 0.0
    check(normal((rows, 5000), rows), uniforms(rows, 3), temperature=t, top_k=k, top_p=p, min_p=m)


@pytest.mark.parametrize("V", [5, 1024, 3001, 40000])
@pytest.mark.parametrize("value", [0.0, -3.5, 1e30])
def test_equal_logits_are_kept_by_index(V, value):
    """Every weight is exactly 1, so the cuts of top-k and top-p and the draw are whole numbers."""
    z = torch.full((6, V), value, device="cuda")
    u = torch.tensor([0.0, 0.1, 0.5, 0.75, 0.999, 1.0 - 2.0 ** -24])
    check(z, u)
    check(z, u, top_k=3)
    check(z, u, top_p=0.5)
    check(z, u, top_k=V - 1, top_p=0.25)
    check(z, u, min_p=1.0)


def test_two_values_only():
    """Two large groups of ties: a cut falls inside either of them."""
    z = torch.zeros((8, 3000), device="cuda")
    z[:, 1::3] = 1.0
    u = uniforms(8, 1)
    for s in (dict(top_k=500), dict(top_k=1000), dict(top_k=1001), dict(top_k=2500), dict(top_p=0.2), dict(top_p=0.7),
              dict(top_k=1700, top_p=0.9), dict(min_p=0.3), dict(min_p=0.4), dict(top_k=1700, min_p=0.3)):
        check(z, u, **s)


def test_masked_rows():
    """-inf and NaN are never drawn; a row that has nothing else gives token 0."""
    z = normal((8, 2000), 1)
    z[0] = -INF
    z[1] = NAN
    z[2, :1999] = -INF
    z[3, 1:] = -INF
    z[4, ::2] = -INF
    z[5, ::3] = NAN
    z[6, 5:] = torch.finfo(torch.float32).min
    z[7] = torch.finfo(torch.float32).min
    for s in SETTINGS + [dict(temperature=0.0), dict(temperature=INF), dict(top_k=1999)]:
        for u in (0.0, 0.37, 0.999):
            check(z, u, **s)
    got, _, _ = draw(z, 0.5)
    assert got[:4] == [0, 0, 1999, 0]


def test_infinite_logits_share_the_row():
    z = normal((4, 700), 2)
    z[0, 5] = z[1, 3] = z[1, 600] = INF
    z[2, 10] = 3e38
    z[3, 10], z[3, 11] = 3e38, -3e38
    for s in SETTINGS + [dict(temperature=INF), dict(temperature=1e-30), dict(temperature=0.0)]:
        for u in (0.0, 0.4, 0.6, 0.99):
            check(z, u, **s)


def test_extreme_settings():
    z = normal((5, 1500), 3)
    u = uniforms(5, 4)
    for s in (dict(temperature=1e-45), dict(temperature=1e-6), dict(temperature=1e6), dict(temperature=INF),
              dict(temperature=-1.0), dict(temperature=NAN), dict(top_k=0), dict(top_k=-1), dict(top_k=2 ** 31 - 1),
              dict(top_k=1500), dict(top_k=1499), dict(top_p=0.0), dict(top_p=-1.0), dict(top_p=1e-30), dict(top_p=2.0),
              dict(top_p=NAN), dict(top_p=1.0 - 2.0 ** -24), dict(min_p=1.0), dict(min_p=7.0), dict(min_p=NAN),
              dict(min_p=1e-30), dict(temperature=INF, top_p=0.5, top_k=100), dict(top_p=INF), dict(min_p=INF)):
        check(z, u, **s)


def test_numbers_outside_the_unit_interval():
    z = normal((6, 900), 5)
    check(z, torch.tensor([-1.0, NAN, 1.0, 5.0, INF, -INF]), top_k=20)
    check(z, torch.tensor([-1.0, NAN, 1.0, 5.0, INF, -INF]))


def test_negative_zero_equals_zero():
    z = torch.full((2, 64), -1.0, device="cuda")
    z[0, 10], z[0, 20] = 0.0, -0.0
    z[1, 10], z[1, 20] = -0.0, 0.0
    check(z, 0.9, top_k=1)
    check(z, 0.9, top_k=2)
    check(z, 0.0, temperature=0.0)


@pytest.mark.parametrize("scale", [1e-3, 0.1, 30.0, 1e4])
def test_flat_and_steep_rows(scale):
    z = normal((6, 7001), 6, std=scale)
    u = uniforms(6, 7)
    for s in SETTINGS:
        check(z, u, **s)


def test_one_outlier_far_below_or_above():
    """A range of logits that leaves nearly all of them next to one end of it."""
    z = normal((4, 9000), 8)
    z[0, 17], z[1, 17], z[2, 17], z[3, 17] = -1e30, 1e30, -3e38, 1e4
    for s in SETTINGS:
        check(z, uniforms(4, 9), **s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("off", [1, 2, 3, 5])
def test_rows_at_any_alignment(dtype, off):
    V = 2047
    flat = normal((4 * V + off,), off, dtype=DT[dtype])
    z = flat[off:].view(4, V)
    for s in SETTINGS:
        check(z, uniforms(4, off), **s)


def test_draws_follow_the_weights():
    """4096 evenly spaced numbers draw every token within one number of its share."""
    z = torch.log(torch.tensor([0.1, 0.2, 0.05, 0.4, 0.25])).cuda().expand(4096, 5).contiguous()
    got, _, _ = draw(z, (torch.arange(4096) + 0.5) / 4096)
    assert got == sorted(got)
    n = np.bincount(got, minlength=5)
    assert np.all(np.abs(n - 4096 * np.array([0.1, 0.2, 0.05, 0.4, 0.25])) <= 1.0)


# bf16 weights are read from a table of 15 octaves below the larger of the top logit and 16 temperatures
@pytest.mark.parametrize("V", [777, 5000, 40000])
@pytest.mark.parametrize("temperature", [0.001, 0.3, 1.0, 50.0, INF])
@pytest.mark.parametrize("scale,shift", [(1e-38, 0), (1e-4, 0), (1e-2, 0.02), (1.0, 0), (1.0, -100.0), (30.0, 0), (1e4, 0), (1e37, 0)])
def test_bf16_values_of_any_magnitude(V, temperature, scale, shift):
    z = (normal((6, V), 31 + V, std=scale) + shift).to(torch.bfloat16)
    z[1, ::3] = -INF
    z[2, 1::2] *= 2.0 ** -14
    z[3, ::2] = z[3, 1]
    z[4, ::5] = NAN
    u = uniforms(6, 32 + V)
    check(z, u, temperature=temperature)
    check(z, u, temperature=temperature, top_p=[0.99, 0.9, 0.7, 0.5, 0.3, 0.05], min_p=[0, 0, 0, 0.01, 0.5, 0])
    check(z, u, temperature=temperature, top_k=[1100, 2000, 0, 1300, 1, 1025], top_p=0.8)


@pytest.mark.parametrize("V", [3000, 40000])
def test_bf16_cut_outside_the_table(V):
    """Most of the weight lies among logits so near to 0, or so far below, that the table has no place for them."""
    near = normal((8, V), 41, std=2.0 ** -14).to(torch.bfloat16)  # under a top of 1 and 16 temperatures of 16
    near[:, 17] = 1.0
    far = (normal((8, V), 42, std=1.5) - 132.0).to(torch.bfloat16)  # |z| >= 128 under a top of -127: past its octave
    far[:, 23] = -127.0
    p = [0.01, 0.1, 0.3, 0.5, 0.7, 0.9, 0.99, 0.9999]
    for z, t in ((near, 1.0), (near, 0.1), (far, 1.0), (far, 0.6)):
        check(z, uniforms(8, 43), temperature=t, top_p=p)
        check(z, uniforms(8, 44), temperature=t, top_p=p, min_p=0.0001, top_k=2000)
    both = torch.where(torch.arange(V, device="cuda") % 2 == 0, near, far)
    check(both, uniforms(8, 45), temperature=0.3, top_p=p)
    both[:, 5] = INF
    both[:, 900::31] = INF
    check(both, uniforms(8, 46), temperature=0.3, top_p=p)


@pytest.mark.parametrize("V", [130, 5000, 40000, 140000])
@pytest.mark.parametrize("min_p", [0.0, 0.2])
def test_bf16_few_values_cut_anywhere(V, min_p):
    """The cut splits tokens of one value, wherever that is in the row, and the draw falls before, in and behind it."""
    n = 32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(V)
    z = torch.randint(1, 5, (n, V), generator=gen, device="cuda").to(torch.bfloat16)
    z[: n // 2, V // 3:] = 1.0  # nearly all the equal ones at the end
    z[n // 2: n // 2 + 4, : V // 2] = 2.0
    p = torch.linspace(0.02, 0.98, n)
    check(z, uniforms(n, V + 1), top_p=p.tolist(), min_p=min_p)
    check(z, 0.97, top_p=p.tolist(), min_p=min_p, temperature=2.0)
