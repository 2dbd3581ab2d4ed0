"""How attention over 8-bit pages of many rows is laid out, as far as its workspace tells it: nothing here needs a GPU."""
import ctypes

import pytest

pytest.importorskip("torch")

from paper_2511_21759_amd import binding as B                        # noqa: E402
from test_quant_cpu import A, BIG, lib                               # noqa: E402, F401


def workspace(lib, rows, max_rows, n, heads=32, kv=8, dim=128, length=8192):        # noqa: F811
    pages = B.odb_quant_pages(k=A[0], v=A[1], k_scale=A[2], v_scale=A[3], n_pages=1000, page_size=64, n_kv_heads=kv, head_dim=dim, codes=4, group=64, dtype=1,
                              page_stride=64 * kv * dim, head_stride=64 * dim, pos_stride=dim, scale_page_stride=kv, scale_head_stride=1)
    a = B.odb_attention(q=BIG, out=2 * BIG, q_row=heads * dim, out_row=heads * dim, cu_rows=A[6], kv_len=A[7], tables=A[8], columns=length // 64, n=n, rows=rows,
                        n_heads=heads, scale=0.1, causal=1, max_rows=max_rows)
    return lib.odb_paged_attention_quant_workspace(ctypes.byref(a), ctypes.byref(pages))


@pytest.mark.parametrize("rows,max_rows,n", [(2048, 2048, 1), (4096, 4096, 1), (6144, 6144, 1), (8192, 8192, 1), (2048, 1024, 2), (4096, 1024, 4)])
def test_rounds_that_are_full_have_nothing_to_cut(lib, rows, max_rows, n):          # noqa: F811
    """64 tiles of 128 rows and heads run at once (512 workgroups, 8 K/V heads): whole rounds of them need no sums of parts, no join and no room for either."""
    assert workspace(lib, rows, max_rows, n, length=4032) == 0        # (two requests of longer keys go in pieces)


@pytest.mark.parametrize("rows,max_rows,n", [(2080, 2080, 1), (3000, 3000, 1), (4100, 4100, 1), (4200, 2400, 3)])
def test_tiles_of_a_last_round_that_holds_a_few_are_cut(lib, rows, max_rows, n):    # noqa: F811
    # parts of 64 places, heads of K/V, rows of a tile: sums and (reference, sum), twice; then where each row's parts are
    assert workspace(lib, rows, max_rows, n) >= 2 * 64 * 8 * 128 * (128 * 4 + 8) + rows * 32 * 8


@pytest.mark.parametrize("rows,max_rows,n,heads,kv,dim", [(768, 24, 32, 32, 8, 128), (2400, 24, 100, 32, 8, 128), (384, 12, 32, 64, 8, 64),
                                                          (1040, 8, 130, 16, 2, 256)])
def test_ragged_requests_of_long_keys_go_in_pieces(lib, rows, max_rows, n, heads, kv, dim):       # noqa: F811
    """Requests with a tile or two each, whose lengths may differ: whole tiles would all wait for the longest.  In pieces as over 16-bit pages."""
    assert workspace(lib, rows, max_rows, n, heads, kv, dim, 9024) > 0


@pytest.mark.parametrize("heads,kv,dim,rows,n,longest,whole", [(32, 32, 128, 320, 10, 1536, True), (32, 32, 128, 320, 10, 1600, False), (64, 8, 64, 80, 20, 1536, True),
                                                               (64, 8, 64, 80, 20, 3008, False), (16, 16, 256, 320, 10, 768, True), (16, 16, 256, 320, 10, 832, False)])
def test_few_rows_are_whole_up_to_1536_keys(lib, heads, kv, dim, rows, n, longest, whole):      # noqa: F811
    assert (workspace(lib, rows, rows // n, n, heads, kv, dim, longest) == 0) == whole
