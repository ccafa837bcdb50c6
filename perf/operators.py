"""The 8-bit path and the sampler next to the packed forward's norm, projections and greedy head,
as calls that can be timed and compared.

Four operators of the tail of every step (residual + norm -> 8-bit projection -> token):

  norm    ``op_add_rmsnorm_fp8``: residual addition, RMSNorm and e4m3 output with one fp32 scale for
          128 columns of a row.
  quant   ``op_quantize_fp8``: the same 8-bit form of rows that no norm produced (blocks of 1 x 128)
          and of weights (128 x 128).
  linear  ``op_linear_fp8``: product of e4m3 activations and weights with those scales.
  sample  ``op_sample``: temperature, top-k, top-p and min-p from given uniform numbers.

Ranges: 1..2264 packed rows (a single decode row up to eight pipelines of depth 8), widths of
64..22016 (odd ones for the norm and the quantisation, outputs of any width and K in multiples of 16
for the product), vocabularies of 100..131072 and 1..256 sampled rows.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
SMALLEST_SCALE = 2.0 ** -126
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LARGEST = {"norm": 2264 * 4096, "quant": 22016 * 4096, "linear": 2264 * 22016 * 4096, "sample": 256 * 131072}


# ----------------------------------------------------------------------------- cases
def _case(name, op, **kw):
    c = {"op": op}
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the fp32 decoder's step (d 256, 32 prompt rows and 2 decode rows): latency only
        _case("norm_tiny_f32", "norm", M=34, D=256, dtype="f32", resid=True),
        # the K = 7 step of the 7B shape: 276 prefill rows and 6 decode rows
        _case("norm_step_282", "norm", M=282, D=4096, dtype="bf16", resid=True),
        # eight pipelines of depth 8 in one forward
        _case("norm_stress_2264", "norm", M=2264, D=4096, dtype="bf16", resid=True),
        # the MLP activation of the K = 7 step before its down projection
        _case("quant_act_282", "quant", M=282, K=11008, dtype="bf16", block_rows=1),
        # gate/up weights of a 7B-shape layer, as a checkpoint is loaded
        _case("quant_weight_gateup", "quant", M=22016, K=4096, dtype="bf16", block_rows=128),
        # one request's decode row through the output projection: launch and latency
        _case("linear_decode_1", "linear", M=1, N=4096, K=4096, out="bf16"),
        # LM head of the K = 7 step, fp32 logits
        _case("linear_head_7", "linear", M=7, N=32000, K=4096, out="f32"),
        # the down projection of the K = 7 step
        _case("linear_down_282", "linear", M=282, N=4096, K=11008, out="bf16"),
        # gate/up of eight pipelines of depth 8
        _case("linear_gateup_2264", "linear", M=2264, N=22016, K=4096, out="bf16"),
        # the K = 7 step's tokens with the usual chat settings: temperature, top-k and top-p
        _case("sample_step_7", "sample", rows=7, V=32000, dtype="f32", settings="chat"),
        # the tokens of eight pipelines, every request with settings of its own
        _case("sample_mixed_64", "sample", rows=64, V=32000, dtype="f32", settings="mixed"),
        # a full serving batch over a long vocabulary, top-p alone
        _case("sample_nucleus_256", "sample", rows=256, V=131072, dtype="bf16", settings="nucleus"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "quant", "linear", "linear", "sample", "sample"])
    if op == "norm":
        D = rng.choice([256, 4096, 11008, _log_int(rng, 64, 11008), 8 * _log_int(rng, 8, 1376)])
        M = min(_log_int(rng, 1, 2264), LARGEST["norm"] // D)
        return _case(None, op, M=M, D=D, dtype=rng.choice(["bf16", "bf16", "f32"]), resid=rng.random() < 0.75)
    if op == "quant":
        block = rng.choice([1, 1, 128])
        K = rng.choice([4096, 11008, _log_int(rng, 64, 22016), 16 * _log_int(rng, 4, 1376)])
        M = min(_log_int(rng, 1, 2264 if block == 1 else 22016), LARGEST["quant"] // K)
        return _case(None, op, M=M, K=K, dtype=rng.choice(["bf16", "bf16", "f32"]), block_rows=block)
    if op == "linear":
        N = rng.choice([4096, 12288, 22016, _log_int(rng, 64, 22016), 16 * _log_int(rng, 4, 1376)])
        K = rng.choice([4096, 11008, 16 * _log_int(rng, 4, 688)])
        M = min(_log_int(rng, 1, 2264), LARGEST["linear"] // (N * K))
        return _case(None, op, M=max(1, M), N=N, K=K, out=rng.choice(["bf16", "bf16", "f32"]))
    return _case(None, op, rows=_log_int(rng, 1, 256), V=rng.choice([32000, _log_int(rng, 100, 131072)]),
                 dtype=rng.choice(["f32", "f32", "bf16"]),
                 settings=rng.choice(["chat", "mixed", "mixed", "nucleus", "min_p", "plain"]))


# ----------------------------------------------------------------------------- inputs
def _blocks(n):
    return (n + 127) // 128


def _normal(gen, shape, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std)


def _activations(gen, M, K):
    """Rows as a residual stream has them: unit normal with a few columns many times as large."""
    x = _normal(gen, (M, K))
    wide = torch.randint(0, K, (max(1, K // 512),), generator=gen, device="cuda")
    x[:, wide] *= 12.0
    return x


def _settings(gen, kind, rows):
    """Per-row temperature, top-k, top-p and min-p (None: not used by the program)."""
    u = lambda lo, hi: torch.rand(rows, generator=gen, device="cuda").mul_(hi - lo).add_(lo)  # noqa: E731
    if kind == "chat":
        return u(0.7, 1.0), torch.full((rows,), 50, dtype=torch.int32, device="cuda"), u(0.9, 0.97), None
    if kind == "nucleus":
        return u(0.7, 1.0), None, u(0.85, 0.97), None
    if kind == "min_p":
        return u(0.8, 1.5), None, None, u(0.02, 0.1)
    if kind == "plain":
        return u(0.6, 1.2), None, None, None
    which = torch.randint(0, 6, (rows,), generator=gen, device="cuda")
    t, k, p, m = u(0.6, 1.3), u(1, 200).to(torch.int32), u(0.8, 0.99), u(0.01, 0.2)
    t = torch.where(which == 5, torch.zeros_like(t), t)                                  # greedy
    k = torch.where((which == 0) | (which == 3), k, torch.zeros_like(k))                 # 0: off
    p = torch.where((which == 1) | (which == 3), p, torch.ones_like(p))                  # 1: off
    m = torch.where((which == 2) | (which == 3), m, torch.zeros_like(m))                 # 0: off
    return t, k, p, m


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"op": case["op"]}
    fp8 = torch.float8_e4m3fn
    if case["op"] == "norm":
        M, D, dt = case["M"], case["D"], DTYPES[case["dtype"]]
        s["x"] = _normal(gen, (M, D), 0.5).to(dt)
        s["resid"] = _activations(gen, M, D).to(dt) if case["resid"] else None
        s["g"] = _normal(gen, (D,), 0.1).add_(1.0).to(dt)
        s["resid_out"] = torch.empty((M, D), dtype=dt, device="cuda") if case["resid"] else None
        s["q"] = torch.empty((M, D), dtype=fp8, device="cuda")
        s["scales"] = torch.empty((M, _blocks(D)), dtype=torch.float32, device="cuda")
    elif case["op"] == "quant":
        M, K, dt = case["M"], case["K"], DTYPES[case["dtype"]]
        s["x"] = (_activations(gen, M, K) if case["block_rows"] == 1 else _normal(gen, (M, K), 0.02)).to(dt)
        s["block_rows"] = case["block_rows"]
        s["q"] = torch.empty((M, K), dtype=fp8, device="cuda")
        s["scales"] = torch.empty((M if case["block_rows"] == 1 else _blocks(M), _blocks(K)), dtype=torch.float32,
                                  device="cuda")
    elif case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        s["xq"], s["xs"] = _quantize(_activations(gen, M, K), 1)
        s["wq"], s["ws"] = _quantize(_normal(gen, (N, K), 0.02), 128)
        s["y"] = torch.empty((M, N), dtype=DTYPES[case["out"]], device="cuda")
    else:
        rows, V = case["rows"], case["V"]
        z = _normal(gen, (rows, V), 2.0)
        likely = torch.randint(0, V, (rows, 6), generator=gen, device="cuda")  # what the model favours
        z.scatter_add_(1, likely, torch.rand((rows, 6), generator=gen, device="cuda").mul_(8.0))
        z[:, :3] = float("-inf")  # tokens that the program never lets through
        s["logits"] = z.to(DTYPES[case["dtype"]])
        s["temperature"], s["top_k"], s["top_p"], s["min_p"] = _settings(gen, case["settings"], rows)
        s["uniforms"] = torch.rand(rows, generator=gen, device="cuda")
        s["tokens"] = torch.empty(rows, dtype=torch.int32, device="cuda")
    return s


# ----------------------------------------------------------------------------- plain forms
def _quantize(x, block_rows):
    """e4m3 values and fp32 scales of an fp32 matrix, blocks of block_rows x 128."""
    M, K = x.shape
    kb, mb = _blocks(K), (M + block_rows - 1) // block_rows
    full = torch.zeros((mb * block_rows, kb * 128), dtype=torch.float32, device=x.device)
    full[:M, :K] = x
    tiles = full.view(mb, block_rows, kb, 128)
    scales = (tiles.abs().amax(dim=(1, 3)) / E4M3_MAX).clamp_min(SMALLEST_SCALE)
    q = (tiles / scales[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    q = q.view(mb * block_rows, kb * 128)[:M, :K].contiguous().view(torch.float8_e4m3fn)
    return q, scales


def _plain_norm(s):
    h, out = s["x"], []
    if s["resid"] is not None:
        h = (h.float() + s["resid"].float()).to(h.dtype)
        out.append(h)
    hf = h.float()
    y = hf * torch.rsqrt(hf.square().mean(dim=1, keepdim=True) + EPS) * s["g"].float()
    return (*out, *_quantize(y, 1))


def _wide(scales, n, dim):
    return scales.repeat_interleave(128, dim=dim).narrow(dim, 0, n)


def _plain_linear(s):
    M, K = s["xq"].shape
    N = s["wq"].shape[0]
    x = s["xq"].float() * _wide(s["xs"], K, 1)
    w = s["wq"].float() * _wide(_wide(s["ws"], K, 1), N, 0)
    return (x @ w.t()).to(s["y"].dtype)


def _plain_sample(s):
    z = s["logits"].double()
    rows, V = z.shape
    t = torch.ones(rows, dtype=torch.float64, device=z.device) if s["temperature"] is None else s["temperature"].double()
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp((z - top) / t.clamp_min(1e-30)[:, None])
    zs, order = z.sort(dim=1, descending=True, stable=True)
    es = e.gather(1, order)
    rank = torch.arange(V, device=z.device)[None, :]
    keep = zs > float("-inf")
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        keep &= (rank < k) | (k <= 0)
    if s["top_p"] is not None:
        kept = es * keep
        before = kept.cumsum(dim=1) - kept
        p = s["top_p"].double()[:, None]
        keep &= (before < p * kept.sum(dim=1, keepdim=True)) | (p >= 1)
    if s["min_p"] is not None:
        keep &= es >= s["min_p"].double()[:, None]
    keep[:, 0] = True
    if s["temperature"] is not None:
        keep &= (rank == 0) | (t > 0)[:, None]
    weight = e * torch.zeros_like(keep).scatter_(1, order, keep)
    c = weight.cumsum(dim=1)
    return (c <= s["uniforms"].double()[:, None] * c[:, -1:]).sum(dim=1).to(torch.int32)


def _run_own(s):
    import paper_2512_20276_amd as af
    if s["op"] == "norm":
        af.op_add_rmsnorm_fp8(s["x"], s["resid"], s["g"], s["resid_out"], s["q"], s["scales"], EPS)
        return (s["q"], s["scales"]) if s["resid"] is None else (s["resid_out"], s["q"], s["scales"])
    if s["op"] == "quant":
        af.op_quantize_fp8(s["x"], s["q"], s["scales"], s["block_rows"])
        return s["q"], s["scales"]
    if s["op"] == "linear":
        af.op_linear_fp8(s["xq"], s["xs"], s["wq"], s["ws"], s["y"])
        return s["y"]
    af.op_sample(s["logits"], s["uniforms"], s["tokens"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    return s["tokens"]


def run(state):
    if own:
        return _run_own(state)
    if state["op"] == "norm":
        return _plain_norm(state)
    if state["op"] == "quant":
        return _quantize(state["x"].float(), state["block_rows"])
    if state["op"] == "linear":
        return _plain_linear(state)
    return _plain_sample(state)


# ----------------------------------------------------------------------------- work
def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["op"] == "norm":
        n, t = case["M"] * case["D"], size[case["dtype"]]
        moved = n * t * (3 if case["resid"] else 1) + case["D"] * t + n + 4 * case["M"] * _blocks(case["D"])
        return {"bytes": moved, "flops": 8 * n}
    if case["op"] == "quant":
        n = case["M"] * case["K"]
        return {"bytes": n * (size[case["dtype"]] + 1) + 4 * _blocks(case["K"]) * -(-case["M"] // case["block_rows"]),
                "flops": 3 * n}
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": (M + N) * K + M * N * size[case["out"]] + 4 * _blocks(K) * (M + _blocks(N)),
                "flops": 2 * M * N * K}
    n = case["rows"] * case["V"]
    return {"bytes": n * size[case["dtype"]] + 24 * case["rows"], "flops": 4 * n}


# ----------------------------------------------------------------------------- 64-bit results
def _exact_blocks(v, block_rows):
    """(value / scale, scale) in 64 bits: what the 8-bit elements would be without their rounding."""
    M, K = v.shape
    scales = torch.empty((-(-M // block_rows), _blocks(K)), dtype=torch.float64, device=v.device)
    out = torch.empty_like(v)
    for b in range(_blocks(K)):
        part = v[:, 128 * b:128 * b + 128]
        largest = part.abs().max(dim=1).values
        if block_rows > 1:
            largest = torch.stack([g.max() for g in largest.split(block_rows)])
        scales[:, b] = torch.maximum(largest / E4M3_MAX, torch.full_like(largest, SMALLEST_SCALE))
        out[:, 128 * b:128 * b + 128] = part / scales[:, b].repeat_interleave(block_rows)[:M, None]
    return out, scales


def _exact_sample(s):
    import numpy as np
    host = {n: v.double().cpu().numpy() for n, v in s.items() if isinstance(v, torch.Tensor) and n != "tokens"}
    tokens = []
    for r, z in enumerate(host["logits"]):
        value = lambda n, off: float(host[n][r]) if n in host else off  # noqa: E731
        t, k, p, m = value("temperature", 1.0), value("top_k", 0), value("top_p", 1.0), value("min_p", 0.0)
        if t <= 0:
            tokens.append(int(np.argmax(z)))
            continue
        order = np.lexsort((np.arange(z.size), -z))
        order = order[np.isfinite(z[order])]
        if k >= 1:
            order = order[:int(k)]
        mass = np.exp((z[order] - z[order[0]]) / t)
        if p < 1:
            order = order[:max(1, int(np.searchsorted(np.cumsum(mass), p * mass.sum(), side="left")) + 1)]
        mass = mass[:order.size]
        order = np.sort(order[(mass >= m) | (np.arange(order.size) == 0)])
        total = np.cumsum(np.exp((z[order] - z[order].max()) / t))
        tokens.append(int(order[min(order.size - 1, int(np.searchsorted(total, host["uniforms"][r] * total[-1], side="right")))]))
    return torch.tensor(tokens, dtype=torch.int32)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h, out = s["x"].double(), []
        if s["resid"] is not None:
            total = h + s["resid"].double()
            out.append(total)
            h = total.to(s["x"].dtype).double()  # the norm is of the sum as it is stored
        length = torch.linalg.vector_norm(h, dim=1, keepdim=True)
        y = s["g"].double() * h / torch.sqrt(length * length / case["D"] + EPS)
        return (*out, *_exact_blocks(y, 1))
    if case["op"] == "quant":
        return _exact_blocks(s["x"].double(), case["block_rows"])
    if case["op"] == "linear":
        y = torch.zeros((case["M"], case["N"]), dtype=torch.float64, device="cuda")
        for b in range(_blocks(case["K"])):
            k = slice(128 * b, 128 * b + 128)
            part = s["xq"][:, k].double() @ s["wq"][:, k].double().t().contiguous()
            y += part * s["xs"][:, b:b + 1].double() * s["ws"][:, b].double().repeat_interleave(128)[:case["N"]]
        return y
    return _exact_sample(s)
