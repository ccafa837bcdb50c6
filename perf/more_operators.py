"""A paged key-value cache and the attention that reads it, as calls that can be timed and compared.

Two operators of a step whose requests keep their keys and values in pages instead of ring slots:

  append  ``op_rope_append_paged``: rotates queries and keys (positions of one axis, or of time, height
          and width) and writes keys and values to their pages.
  attend  ``op_attention_paged``: attention of packed rows over the pages, one row a request (split over
          the cache's length) or prompts, chunks of prompts and single rows together; grouped heads,
          a sliding window and first keys that stay visible.

Ranges: 1..64 requests, 1..8192 packed rows, caches of 1..131072 keys, pages of 8..256, 1..32 heads in
groups of 1..8 with head sizes 64 and 128, bf16 and fp32.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
THETA = 10000.0
NO_REQUESTS = {"n_pre": 0, "q_rows": 0, "past": 0, "n_dec": 0, "kv": 0}
# what the largest listed cases have
MOST_SCORES = 32 * 8192 * 8192  # all rows against the longest cache
MOST_KEY_BYTES = 131072 * 8 * 128 * 2
MOST_FLOPS = {"bf16": 137e9, "f32": 137e9 / 16}  # a matrix instruction's rates are 1 : 16


# ----------------------------------------------------------------------------- cases
def _case(name, op, **kw):
    c = {"op": op, **NO_REQUESTS, "Hq": 32, "Hkv": 32, "hd": 128, "page": 16, "dtype": "bf16", "ragged": False, "salt": 0}
    c.update({"axes": 0} if op == "append" else {"window": 0, "sinks": 0, "lse": False})
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # decode rows of the fp32 decoder: latency only
        _case("append_tiny_f32", "append", n_dec=2, kv=36, Hq=4, Hkv=4, hd=64, dtype="f32"),
        # the K = 7 step: a 276-row prefill of image patches and instruction, and 6 decode rows
        _case("append_step_282", "append", n_pre=1, q_rows=276, n_dec=6, kv=282, axes=3),
        # eight pipelines of depth 8 in one step
        _case("append_stress_2264", "append", n_pre=8, q_rows=276, n_dec=56, kv=283, page=64),
        # two requests of the fp32 decoder: latency only
        _case("decode_tiny_f32", "attend", n_dec=2, kv=36, Hq=4, Hkv=4, hd=64, dtype="f32"),
        # the decode rows of sixty-four requests behind a 276-row prompt
        _case("decode_short_64", "attend", n_dec=64, kv=283),
        # a serving batch of requests of very different age, four heads to a key head
        _case("decode_ragged_48", "attend", n_dec=48, kv=16384, Hkv=8, page=64, ragged=True, salt=1),
        # one request with a very long history
        _case("decode_long_1", "attend", n_dec=1, kv=131072, Hkv=8, page=64, lse=True),
        # robots that run for hours: a window over the last frames, the instruction stays visible
        _case("decode_window_32", "attend", n_dec=32, kv=32768, Hkv=8, window=4096, sinks=20),
        # the K = 7 step's attention
        _case("step_282", "attend", n_pre=1, q_rows=276, n_dec=6, kv=282),
        # one long prompt
        _case("prompt_4096", "attend", n_pre=1, q_rows=4096, Hkv=8, page=64, lse=True),
        # chunks of prompts on what is there of them, with other requests' decode rows
        _case("chunks_mixed_32", "attend", n_pre=4, q_rows=256, past=8192, n_dec=28, kv=8192, Hkv=8, page=32, ragged=True, salt=2),
        # a prompt of many frames under a window
        _case("prompt_window_8192", "attend", n_pre=1, q_rows=8192, Hkv=8, page=64, window=1000, sinks=20),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    group = rng.choice([1, 1, 2, 4, 4, 8])
    heads = {"hd": rng.choice([64, 128, 128]), "Hkv": max(1, rng.choice([4, 8, 16, 32]) // group), "page": 2 ** rng.randint(3, 8),
             "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"]), "ragged": rng.random() < 0.6, "salt": rng.randrange(1 << 20)}
    heads["Hq"] = heads["Hkv"] * group
    kind = rng.choice(["append", "decode", "decode", "rows", "rows"])
    if kind == "append":
        c = _case(None, "append", **heads, axes=rng.choice([0, 0, 1, 2, 3]), n_dec=rng.randint(1, 64), kv=_log_int(rng, 1, 4096))
        if rng.random() < 0.6:
            c["n_pre"], c["q_rows"], c["past"] = rng.randint(1, 8), _log_int(rng, 2, 276), rng.choice([0, _log_int(rng, 1, 1024)])
        return c
    limits = {}
    if rng.random() < 0.4:
        limits = {"window": _log_int(rng, 1, 4096), "sinks": rng.choice([0, 4, _log_int(rng, 1, 64)])}
    limits["lse"] = rng.random() < 0.4
    if kind == "decode":
        keys = MOST_KEY_BYTES // (SIZE[heads["dtype"]] * heads["Hkv"] * heads["hd"])
        kv = min(_log_int(rng, 1, 131072), keys)
        return _case(None, "attend", **heads, **limits, n_dec=rng.randint(1, min(64, keys // kv)), kv=kv)
    c = _case(None, "attend", **heads, **limits, n_pre=rng.choice([1, 1, 2, 4, 8]), q_rows=_log_int(rng, 2, 4096),
              past=rng.choice([0, 0, _log_int(rng, 1, 8192)]))
    if rng.random() < 0.5:
        c["n_dec"], c["kv"] = rng.randint(1, 32), _log_int(rng, 1, 8192)
    while ((c["n_pre"] + c["n_dec"]) * c["q_rows"] * c["Hq"] * max(c["q_rows"] + c["past"], c["kv"]) > MOST_SCORES // 2
           or work(c)["flops"] > MOST_FLOPS[c["dtype"]]):
        if c["n_dec"] > 1:
            c["n_dec"] //= 2
        else:
            c["q_rows"] = max(2, c["q_rows"] * 3 // 4)
            c["past"] = c["past"] * 3 // 4
    return c


def _requests(case):
    """(rows, cache length with them) of every request, the prompts first: the same for every seed."""
    rng = random.Random("%s %s" % (case["salt"], case["kv"]))
    some = lambda most: _log_int(rng, 1, most) if case["ragged"] and most > 1 else most  # noqa: E731
    got = []
    for _ in range(case["n_pre"]):
        rows = max(2, case["q_rows"] - rng.randrange(1 + case["q_rows"] // 4)) if case["ragged"] else case["q_rows"]
        got.append((rows, rows + (some(case["past"]) if case["past"] else 0)))
    for i in range(case["n_dec"]):
        got.append((1, some(case["kv"]) if case["ragged"] else max(1, case["kv"] - i % 7)))
    return got


# ----------------------------------------------------------------------------- inputs
def _normal(gen, shape, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std)


def _sections(n_axes, hd):
    """Pairs of a head that turn with each axis: time takes an eighth and what is left over."""
    each = 3 * (hd // 2) // (8 if n_axes == 3 else 4)
    return [hd // 2 - (n_axes - 1) * each] + [each] * (n_axes - 1)


def _positions(gen, case, requests):
    """Positions of packed rows: patches of frames of 16 x 16 and then text, on from where each request is."""
    parts = []
    for n, length in requests:
        start = length - n + int(torch.randint(0, 100000, (1,), generator=gen, device="cuda"))
        r = torch.arange(n, device="cuda")
        patch = r < n // 256 * 256
        axes = [r // 256, r // 16 % 16, r % 16]
        text = r - n // 256 * 255
        parts.append(start + torch.stack([torch.where(patch, a, text) for a in axes[:case["axes"]]], dim=1))
    return torch.cat(parts).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, hd, P, Hq, Hkv = DTYPES[case["dtype"]], case["hd"], case["page"], case["Hq"], case["Hkv"]
    requests = _requests(case)
    M = sum(n for n, _ in requests)
    pages = [-(-length // P) for _, length in requests]
    order = torch.randperm(sum(pages) + 3, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(requests), max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n, _ in requests:
        starts.append(starts[-1] + n)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"op": case["op"], "table": table, "lens": i32([length for _, length in requests]),
         "starts": i32(starts) if case["n_pre"] else None, "most_rows": max(n for n, _ in requests),
         "most_keys": max(length for _, length in requests), "Hq": Hq}
    for name in ("k_cache", "v_cache"):
        s[name] = torch.randn((sum(pages) + 3, Hkv, P, hd), generator=gen, device="cuda", dtype=dt)
    if case["op"] == "append":
        # rows as the fused projection leaves them: queries, keys and values of a row side by side
        qkv = _normal(gen, (M, Hq + 2 * Hkv, hd)).to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["positions"] = _positions(gen, case, requests) if case["axes"] else None
        s["sections"] = _sections(case["axes"], hd) if case["axes"] > 1 else None
    else:
        s["q"] = _normal(gen, (M, Hq, hd), 1.5).to(dt)
        s["scale"], s["window"], s["sinks"] = 1.0 / math.sqrt(hd), case["window"], case["sinks"]
        s["lse"] = torch.empty((M, Hq), dtype=torch.float32, device="cuda") if case["lse"] else None
    s["out"] = torch.empty((M, Hq, hd), dtype=dt, device="cuda")
    return s


# ----------------------------------------------------------------------------- plain forms
def _row_places(s):
    """(request, cache position) of every packed row."""
    M, n = s["q"].shape[0], s["lens"].shape[0]
    row = torch.arange(M, device="cuda", dtype=torch.int32)
    if s["starts"] is None:
        return row.long(), (s["lens"] - 1).long()
    b = torch.searchsorted(s["starts"][1:].contiguous(), row, right=True).clamp_max(n - 1)
    return b, (s["lens"][b] - s["starts"][b + 1] + row).long()


def _plain_append(s):
    b, at = _row_places(s)
    hd, P = s["q"].shape[2], s["k_cache"].shape[2]
    pos = at[:, None] if s["positions"] is None else s["positions"]
    j = torch.arange(hd // 2, device="cuda", dtype=torch.float64)
    turn = torch.exp(j * (-2.0 * math.log(THETA) / hd))
    axis = torch.zeros(hd // 2, dtype=torch.int64, device="cuda")
    for start in ([] if s["sections"] is None else [sum(s["sections"][:a]) for a in range(1, len(s["sections"]))]):
        axis[start:] += 1
    angle = pos.double()[:, axis] * turn
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def rotated(x):
        lo, hi = x[..., :hd // 2].float(), x[..., hd // 2:].float()
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1).to(x.dtype)

    page = s["table"][b, at // P].long()
    s["k_cache"][page, :, at % P] = rotated(s["k"])
    s["v_cache"][page, :, at % P] = s["v"]
    return rotated(s["q"]), s["k_cache"], s["v_cache"]


def _plain_attend(s):
    M, Hq, hd = s["q"].shape
    n, Hkv, kmax, qmax = s["lens"].shape[0], s["k_cache"].shape[1], s["most_keys"], s["most_rows"]
    G = Hq // Hkv
    b, at = _row_places(s)

    def whole(cache):  # [n, Hkv, kmax, hd] in 32 bits
        x = cache[s["table"].clamp_min(0).long()].transpose(1, 2)
        return x.reshape(n, Hkv, -1, hd)[:, :, :kmax].float().contiguous()

    first = torch.arange(n, device="cuda") if s["starts"] is None else s["starts"][:-1].long()
    rows = first[:, None] + torch.arange(qmax, device="cuda")
    if s["starts"] is not None:
        rows = torch.minimum(rows, s["starts"][1:, None].long() - 1)
    q = s["q"][rows].float().view(n, qmax, Hkv, G, hd).permute(0, 2, 1, 3, 4).reshape(n, Hkv, qmax * G, hd)
    score = torch.matmul(q, whole(s["k_cache"]).transpose(2, 3)).mul_(s["scale"])
    key, last = torch.arange(kmax, device="cuda"), at[rows][:, :, None]
    hidden = key > last
    if s["window"]:
        hidden |= (key <= last - s["window"]) & (key >= s["sinks"])
    score.view(n, Hkv, qmax, G, kmax).masked_fill_(hidden[:, None, :, None], float("-inf"))
    top = score.amax(dim=3, keepdim=True)
    weight = score.sub_(top).exp_()
    total = weight.sum(dim=3, keepdim=True)
    o = torch.matmul(weight, whole(s["v_cache"])).div_(total).view(n, Hkv, qmax, G, hd)
    within = torch.arange(M, device="cuda") - first[b]
    out = o[b, :, within].reshape(M, Hq, hd).to(s["q"].dtype)
    if s["lse"] is None:
        return out
    lse = (top + total.log()).view(n, Hkv, qmax, G)
    return out, lse[b, :, within].reshape(M, Hq)


def _run_own(s):
    import paper_2512_20276_amd as af
    kv = s.get("kv")
    if kv is None:  # what a program keeps beside its cache
        kv = s["kv"] = af.PagedKV(s["k_cache"], s["v_cache"], s["table"], s["lens"], s["starts"])
        if s["op"] == "attend":
            need = af.attention_paged_workspace(kv, s["q"].shape[0], s["Hq"])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    if s["op"] == "append":
        af.op_rope_append_paged(kv, s["q"], s["k"], s["v"], s["out"], THETA, s["positions"], s["sections"])
        return s["out"], s["k_cache"], s["v_cache"]
    af.op_attention_paged(kv, s["q"], s["out"], s["scale"], s["workspace"], s["window"], s["sinks"], s["lse"])
    return s["out"] if s["lse"] is None else (s["out"], s["lse"])


def run(state):
    if own:
        return _run_own(state)
    return _plain_append(state) if state["op"] == "append" else _plain_attend(state)


# ----------------------------------------------------------------------------- work
def _seen(case, p):
    """Keys that a row at cache position p sees."""
    if not case["window"] or p < case["window"]:
        return p + 1
    return case["window"] + min(case["sinks"], p + 1 - case["window"])


def work(case):
    size, requests = SIZE[case["dtype"]], _requests(case)
    M = sum(n for n, _ in requests)
    if case["op"] == "append":
        values = M * (case["Hq"] + 2 * case["Hkv"]) * case["hd"]
        return {"bytes": 2 * values * size + 4 * M * max(1, case["axes"]), "flops": 3 * M * (case["Hq"] + case["Hkv"]) * case["hd"]}
    keys = rows = 0
    for n, length in requests:
        # the last row's window and first keys, and what the rows before it see besides
        keys += min(length, _seen(case, length - 1) + (n - 1 if case["window"] else 0))
        rows += sum(_seen(case, p) for p in range(length - n, length))
    moved = 2 * keys * case["Hkv"] * case["hd"] * size + 2 * M * case["Hq"] * case["hd"] * size
    return {"bytes": moved + (4 * M * case["Hq"] if case["lse"] else 0), "flops": 4 * rows * case["Hq"] * case["hd"]}


# ----------------------------------------------------------------------------- 64-bit results
def _exact_append(case, s):
    requests, hd, P = _requests(case), case["hd"], case["page"]
    half, table = hd // 2, s["table"].tolist()
    sections = s["sections"] or [half]
    turn = torch.tensor([THETA ** (-2.0 * j / hd) for j in range(half)], dtype=torch.float64, device="cuda")
    places = [(b, length - n + i) for b, (n, length) in enumerate(requests) for i in range(n)]
    if s["positions"] is None:
        pos = torch.tensor([[float(p)] for _, p in places], dtype=torch.float64, device="cuda")
    else:
        pos = s["positions"].double()
    angle = torch.cat([pos[:, a:a + 1].expand(-1, w) for a, w in enumerate(sections)], dim=1) * turn
    phase = torch.polar(torch.ones_like(angle), angle)[:, None]

    def rotated(x):
        z = torch.complex(x[..., :half].double(), x[..., half:].double()) * phase
        return torch.cat([z.real, z.imag], dim=-1)

    cell = torch.tensor([table[b][p // P] * P + p % P for b, p in places], device="cuda")

    def written(cache, rows):
        flat = cache.double().transpose(1, 2).reshape(-1, case["Hkv"], hd).clone()
        flat[cell] = rows
        return flat.view(-1, P, case["Hkv"], hd).transpose(1, 2)

    return rotated(s["q"]), written(s["k_cache"], rotated(s["k"])), written(s["v_cache"], s["v"].double())


def _exact_attend(case, s):
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    Hkv, hd, G = case["Hkv"], case["hd"], case["Hq"] // case["Hkv"]
    row = 0
    for b, (n, length) in enumerate(_requests(case)):
        ids = s["table"][b, :-(-length // case["page"])].long()
        K, V = (torch.cat(list(c[ids].unbind(0)), dim=1)[:, :length].double() for c in (s["k_cache"], s["v_cache"]))
        step = max(1, (1 << 28) // (length * case["Hq"]))
        for i in range(0, n, step):
            m = min(step, n - i)
            q = s["q"][row + i:row + i + m].double().view(m, Hkv, G, hd)
            p = torch.arange(length - n + i, length - n + i + m, device="cuda")[:, None]
            j = torch.arange(length, device="cuda")[None, :]
            see = j <= p
            if case["window"]:
                see &= (p - j < case["window"]) | (j < case["sinks"])
            for h in range(Hkv):
                z = q[:, h].reshape(m * G, hd) @ K[h].t().contiguous() * s["scale"]
                z = z.view(m, G, length).masked_fill(~see[:, None], float("-inf"))
                norm = torch.logsumexp(z, dim=2)
                out[row + i:row + i + m, h * G:h * G + G] = (torch.exp(z - norm[..., None]).view(m * G, length) @ V[h]).view(m, G, hd)
                lse[row + i:row + i + m, h * G:h * G + G] = norm
        row += n
    return out if s["lse"] is None else (out, lse)


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(case, s) if case["op"] == "append" else _exact_attend(case, s)
