"""CPU tests of the sizes that the operators over a paged cache take, and of the workspace they ask for."""
import ctypes as C
import math
import random

import paper_2512_20276_amd as af

lib = af.lib
P = 1 << 20  # an aligned address that no query ever follows


def desc(**at):
    d = dict(k=P, v=P, page_table=P, kv_lens=P, q_starts=None, n_pages=9, page_size=16, n_kv_heads=1, head_dim=128, n_seq=1,
             max_pages=4, dtype=af.AF_BF16, reserved=0)
    return af.PagedKVDesc(**{**d, **at})


def workspace(d, M, n_heads):
    n = C.c_size_t()
    code = lib.af_attention_paged_workspace(C.addressof(d), M, n_heads, C.byref(n))
    return n.value if code == af.AF_OK else code


def test_shares_of_the_longest_caches_fit_32_bits():
    """Single rows' keys are counted in tiles of 32, with up to three a request beside what the table holds, and cut into at
    most 512 shares of the same whole number of tiles: the last share's end, up to 511 past the tiles of all, is an int."""
    for n_seq in (64, 65, 71, 96, 102):
        most = (2 ** 31 - 1) // n_seq  # tiles of a request's table, and a few
        taken = [tiles for tiles in range(most - 40, min(most, 1 << 25) + 1)
                 if workspace(desc(n_seq=n_seq, page_size=32, max_pages=tiles), n_seq, 1) >= 0]
        assert taken and all(n_seq * (tiles + 3) + 511 <= 2 ** 31 - 1 for tiles in taken), (n_seq, taken[-1:])
        assert len(taken) >= 20  # no more is refused than that needs


def test_a_workspace_is_enough_for_smaller_steps():
    """A program asks once, for its largest step: fewer rows, requests or pages, with q_starts or without, need no more."""
    rng = random.Random(0)
    spread = lambda most: int(math.exp(rng.uniform(0, math.log(most))) + 0.5)  # noqa: E731
    for _ in range(3000):
        Hkv, group, hd = rng.choice([1, 2, 3, 8, 32]), rng.choice([1, 2, 4, 5, 8, 17]), rng.choice([64, 128])
        fixed = dict(n_kv_heads=Hkv, head_dim=hd, page_size=2 ** rng.randint(3, 8), dtype=rng.choice([af.AF_BF16, af.AF_F32]))
        n_seq, max_pages, M = spread(200), spread(4096), spread(20000)
        most = workspace(desc(**fixed, q_starts=P, n_seq=n_seq, max_pages=max_pages), M, Hkv * group)
        assert most >= 0, af.last_error()
        for _ in range(6):
            m, b, pages = (rng.choice([x, spread(x), max(x - 1, 1)]) for x in (M, n_seq, max_pages))
            starts = P if rng.random() < 0.7 or b > M else None
            d, m = desc(**fixed, q_starts=starts, n_seq=b, max_pages=pages), m if starts else b
            row = Hkv * group * hd
            # an address that is not aligned, which is looked at behind the size: nothing is launched
            code = lib.af_op_attention_paged(C.addressof(d), P, row, P, row, None, m, Hkv * group, 0.1, 0, 0, P + 8, most, None)
            assert code == af.AF_ERR_INVALID_ARG and "16-byte aligned" in af.last_error(), (fixed, group, (n_seq, max_pages, M), (b, pages, m, starts), af.last_error())
