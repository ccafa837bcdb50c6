"""Plain 64-bit forms of the operators over a paged key-value cache, and the bounds that their tests hold the
kernels to."""
from __future__ import annotations

import math

import torch

U32 = 2.0 ** -24                                            # half a step of fp32, relative
HALF_STEP = {torch.float32: U32, torch.bfloat16: 2.0 ** -8}  # torch.finfo(t).eps / 2


class Step:
    """Requests of one step and a pool with their keys: ``requests`` is a list of (rows, length with them).
    ``before`` and ``behind`` packed rows belong to no request; ``single``: no q_starts."""

    def __init__(self, requests, Hkv=2, group=2, hd=64, page=16, dtype=torch.bfloat16, single=False, before=0, behind=0,
                 spare_pages=3, extra_table=0, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.requests, self.Hkv, self.group, self.hd, self.page, self.dtype = requests, Hkv, group, hd, page, dtype
        self.Hq, self.device = Hkv * group, device
        pages = [max(0, -(-length // page)) for _, length in requests]
        n_pages = sum(pages) + spare_pages
        order = torch.randperm(n_pages, generator=g).tolist()
        self.table = torch.full((len(requests), max(max(pages), 1) + extra_table), -1, dtype=torch.int32)
        for b, n in enumerate(pages):
            self.table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
        self.starts = [before]
        for n, _ in requests:
            self.starts.append(self.starts[-1] + n)
        self.M = self.starts[-1] + behind
        self.single = single
        draw = lambda *s: torch.randn(s, generator=g).to(dtype)  # noqa: E731
        self.k_cache, self.v_cache = draw(n_pages, Hkv, page, hd), draw(n_pages, Hkv, page, hd)
        self.q = draw(self.M, self.Hq, hd)
        self.k, self.v = draw(self.M, Hkv, hd), draw(self.M, Hkv, hd)
        self.lens = torch.tensor([length for _, length in requests], dtype=torch.int32)

    def rows(self):
        """(row, request, cache position) of every row that a request has."""
        for b, (n, length) in enumerate(self.requests):
            for i in range(n):
                yield self.starts[b] + i, b, length - n + i

    def cell(self, b, j):
        """(page, offset) of key j of request b, None: it does not exist."""
        if j < 0 or j >= self.table.shape[1] * self.page:
            return None
        page = int(self.table[b, j // self.page])
        return (page, j % self.page) if 0 <= page < self.k_cache.shape[0] else None

    def to_gpu(self, af):
        dev = self.device
        self.g = {n: getattr(self, n).to(dev) for n in ("k_cache", "v_cache", "table", "lens", "q", "k", "v")}
        starts = None if self.single else torch.tensor(self.starts, dtype=torch.int32, device=dev)
        self.kv = af.PagedKV(self.g["k_cache"], self.g["v_cache"], self.g["table"], self.g["lens"], starts)
        return self.kv

    # ------------------------------------------------------------------ append
    def rotated(self, theta, positions=None, sections=None):
        """Rotated q and k in 64 bits and the bound of each result's error.

        The angle, in half turns, is rounded to fp32 once (2^-25 of a half turn: pi 2^-25), after a product in 64 bits
        (its own rounding, 2^-53 of the whole angle, and the frequency's: two powers within an ulp's half and a little, their
        product and a division by 2 pi, which is rounded itself: 6 2^-53 in all).  A sine or cosine is within 4 ulp
        (2^-22).  So each is off by less than 2^-22 + pi 2^-25 + 6 2^-53 angle < 2^-21 - 2^-23 + ..; two products and their sum add
        2 U32 of |x| + |y| at most: (|x| + |y|) (2^-21 + 6 2^-53 angle), and the result's rounding."""
        half = self.hd // 2
        pos = torch.zeros(self.M, 1, dtype=torch.float64)
        if positions is None:
            for row, _, p in self.rows():
                pos[row, 0] = p
        else:
            pos = positions.double().view(self.M, -1)
        axis = [a for a, n in enumerate(sections or [half]) for _ in range(n)]
        turn = torch.tensor([float(theta) ** (-2.0 * j / self.hd) for j in range(half)], dtype=torch.float64)
        angle = pos[:, axis] * turn
        out = []
        for x in (self.q, self.k):
            a, b = x[..., :half].double(), x[..., half:].double()
            co, si = angle.cos()[:, None], angle.sin()[:, None]
            y = torch.cat([a * co - b * si, b * co + a * si], dim=-1)
            each = (a.abs() + b.abs()) * (2.0 ** -21 + 6 * 2.0 ** -53 * angle.abs()[:, None])
            each = torch.cat([each, each], dim=-1)
            out.append((y, each + HALF_STEP[self.dtype] * (y.abs() + each)))
        return out

    # ------------------------------------------------------------------ attention
    def attended(self, scale, window=0, sinks=0):
        """(o, its bound, lse, its bound) in 64 bits for every row; rows of no request are NaN.

        A score is a product of hd exact terms summed in fp32, and scaled: off by (hd + 3) U32 of the sum of their
        magnitudes; its distance to the maximum is rounded once more.  exp2 is within an ulp (2^-23).  A weight is
        multiplied with values as it is (fp32), as a bf16 number and a bf16 remainder (bf16, requests with a single row:
        2^-8 of 2^-8 is lost) or as a bf16 number (bf16, several rows: half a step, 2^-8).  n weights, and their products
        with values, are summed in fp32, in any order: n U32.  A weight's error counts in the numerator and in the
        denominator, but for its rounding to bf16, which the sum of weights does not have."""
        o = torch.full((self.M, self.Hq, self.hd), math.nan, dtype=torch.float64)
        o_bound, lse = torch.full_like(o, math.nan), torch.full((self.M, self.Hq), math.nan, dtype=torch.float64)
        lse_bound = torch.full_like(lse, math.nan)
        kc, vc = self.k_cache.double(), self.v_cache.double()
        for b, (n, length) in enumerate(self.requests):
            if n == 0:
                continue
            held = 0.0 if self.dtype is torch.float32 else 2.0 ** -16 if n == 1 else 2.0 ** -8
            keys = [j for j in range(max(length, 0)) if self.cell(b, j) is not None]
            cells = [self.cell(b, j) for j in keys]
            pg, off = torch.tensor([c[0] for c in cells], dtype=torch.long), torch.tensor([c[1] for c in cells], dtype=torch.long)
            j = torch.tensor(keys, dtype=torch.long)
            K, V = kc[pg, :, off], vc[pg, :, off]  # [keys, Hkv, hd]
            for i in range(n):
                row, p = self.starts[b] + i, length - n + i
                see = j <= p
                if window:
                    see &= (j > p - window) | (j < sinks)
                k, v = K[see], V[see]
                if k.shape[0] == 0:
                    o[row], o_bound[row], lse[row], lse_bound[row] = 0, 0, -math.inf, 0
                    continue
                q = self.q[row].double().view(self.Hkv, self.group, self.hd)
                s = torch.einsum("hgd,khd->hgk", q, k) * scale
                size = torch.einsum("hgd,khd->hgk", q.abs(), k.abs()) * abs(scale)
                w = torch.softmax(s, dim=2)
                far = (s.amax(dim=2, keepdim=True) - s) * U32
                each = (self.hd + 3) * U32 * size + far + 2.0 ** -23
                worst = each.amax(dim=2, keepdim=True) + see.sum() * U32
                r = torch.einsum("hgk,khd->hgd", w, v)
                total = torch.einsum("hgk,khd->hgd", w, v.abs())
                err = (2 * worst + held) * total
                o[row] = r.reshape(self.Hq, self.hd)
                o_bound[row] = (err + HALF_STEP[self.dtype] * (r.abs() + err)).reshape(self.Hq, self.hd)
                top = torch.logsumexp(s, dim=2)
                lse[row] = top.reshape(-1)
                # the maximum's own error, the sum's, a logarithm's (2 ulp), and three roundings of results of this size
                lse_bound[row] = (each.amax(dim=2) + see.sum() * U32 + (s.abs().amax(dim=2) + top.abs() + 1 + math.log(see.sum())) * 6 * U32).reshape(-1)
        return o, o_bound, lse, lse_bound


def inside(got: torch.Tensor, want: torch.Tensor, bound: torch.Tensor, what=""):
    """got is within bound of want wherever want is not NaN."""
    got = got.cpu().double()
    told = ~torch.isnan(want)
    same = got == want  # infinities
    bad = told & ~same & ~((got - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist(),
                           float(((got - want).abs() / bound.clamp_min(1e-300))[bad].nan_to_num(1e30).max()))
