"""Where hydra_attn_decode draws the line at large tables: fewer than 2^30 tiles of 64 rows, counted for rows of the table's full length.
What passes the check is refused for its missing workspace, before anything is read."""
import pytest

import paper_2609_34318_b200 as P

A = 1 << 20                                                 # an aligned address; never read
PASSED = P.HYDRA_ERR_INVALID_ARG                            # (no workspace)


def call(h, hk, n_seqs, max_pages, page):
    c = P.hydra_paged_cache_t()
    for name, value in dict(k=A, v=A, page_table=A, seq_lens=A, n_pages=10, page_size=page, n_kv_heads=hk, d_qk=128, d_v=128, n_seqs=n_seqs,
                            max_pages=max_pages).items():
        setattr(c, name, value)
    return P.hydra_attn_decode(A, c, h, 0.1, A, A, None, workspace_bytes=1 << 40, q_stride=h * 128, stream=0, check=False)


# m: K / V heads of a tile, 64 / m keys each; u: units of a sequence
@pytest.mark.parametrize("h,hk,m,u", [(1, 1, 1, 1), (4, 4, 4, 1), (16, 2, 2, 1), (16, 1, 1, 1), (32, 1, 1, 1), (33, 1, 1, 2), (80, 2, 1, 4), (8, 8, 4, 2),
                                      (15, 3, 1, 3), (12, 6, 2, 3)])
def test_tiles_of_a_full_table(h, hk, m, u):
    page, max_pages = 64, 16                                # 1024 keys a row
    tiles = 1024 * m // 64 + 1
    most = min(((1 << 30) - 1) // u // tiles, (2 ** 31 - 1) // h)
    assert call(h, hk, most, max_pages, page) == PASSED
    assert call(h, hk, most + 1, max_pages, page) == P.HYDRA_ERR_UNSUPPORTED
    assert call(h, hk, 1, (1 << 30) // page, page) == (PASSED if (2 ** 30 // 64 * m + 1) * u < 1 << 30 else P.HYDRA_ERR_UNSUPPORTED)
    assert call(h, hk, 1, (1 << 30) // page + 1, page) == P.HYDRA_ERR_UNSUPPORTED
