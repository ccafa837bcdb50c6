"""CPU tests of the sizes that the operators over a paged cache take, and of the workspace they ask for."""
import ctypes as C

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
