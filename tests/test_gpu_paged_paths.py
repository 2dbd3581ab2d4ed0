"""Ways of computing of the paged operators that sizes lead to and test_gpu_paged.py does not: numbering of many requests without row
offsets, whole tiles of many rows over many requests, missing pages under windows, tables at the sizes where their LDS grows.  Plain
forms and bounds are those of test_gpu_paged.py."""
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paged_plain as plain                                          # noqa: E402
from test_gpu_paged import F, Requests, half_step, run_tables, tables_case       # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [2339, 2340, 2341])
def test_page_tables_where_their_lds_passes_64_kib(n):
    held, wanted, tables, free, n_free, first, count = tables_case(n, n, 16, 3, 900, 9000)
    blank = np.full(9000, -77, np.int32)
    want = plain.page_tables(held, wanted, tables, free, n_free, 16, first, count, 9000, blank, blank)
    for got in run_tables(held, wanted, tables, free, n_free, 16, first, count, 9000):
        for g, w in zip(got, want):
            assert np.array_equal(g.reshape(-1), np.asarray(w, np.int64).reshape(-1))


def test_page_tables_of_lengths_that_no_table_holds_and_default_rows():
    """Without row counts a request that wants what its table cannot hold has no rows, like one that wants less than it holds."""
    held, wanted, tables, free, n_free, _, _ = tables_case(3, 40, 16, 5, 300, 500, bad=True)
    blank = np.full(3000, -77, np.int32)
    want = plain.page_tables(held, wanted, tables, free, n_free, 16, None, None, 3000, blank, blank)
    cu = np.asarray(want[4])
    assert any(w > 80 and cu[r + 1] == cu[r] for r, w in enumerate(wanted)) and any(w < 0 for w in wanted)
    for got in run_tables(held, wanted, tables, free, n_free, 16, None, None, 3000):
        for g, w in zip(got, want):
            assert np.array_equal(g.reshape(-1), np.asarray(w, np.int64).reshape(-1))


# with max_rows 1: tiles of 16, 32 and 64 rows whose waves split the keys, then of 128 and 64 whose waves split the rows, one and two a
# request; without it the second kind throughout
@pytest.mark.parametrize("n,heads,kv,dim", [(513, 1, 1, 64), (700, 4, 2, 128), (600, 20, 1, 256), (600, 33, 1, 128), (513, 70, 1, 64), (600, 130, 1, 64), (600, 90, 1, 256),
                                            (4096, 3, 1, 64)])
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 20, 3)])
def test_single_tokens_of_many_requests_without_row_offsets(n, heads, kv, dim, causal, window, sinks):
    rng = random.Random(n + heads)
    lens = [rng.choice([0, 1, 16, 17, 33, rng.randint(1, 90)]) for _ in range(n)]
    rq = Requests(n + dim, [1] * n, lens, heads, kv, dim, "bf16" if dim == 128 else "f16", 16)
    for max_rows, max_len in ((1, 0), (1, 90), (0, 0)):
        rq.check(rq.run(cu=False, causal=causal, window=window, sinks=sinks, max_rows=max_rows, max_len=max_len), causal=causal, window=window, sinks=sinks)


@pytest.mark.parametrize("cache,dim,heads,kv", [("f16", 64, 2, 1), ("bf16", 128, 4, 2), ("f16", 256, 1, 1)])
@pytest.mark.parametrize("max_rows", [0, 150])
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 30, 5)])
def test_whole_tiles_of_many_rows_over_many_requests(cache, dim, heads, kv, max_rows, causal, window, sinks):
    rng = random.Random(dim)
    n = 700
    lens = [rng.choice([1, 5, 33, 70]) for _ in range(n)]
    rows = [min(length, rng.choice([0, 1, 1, 2, 3])) for length in lens]
    for r in (0, 255, 511, 699):
        lens[r], rows[r] = 190 + r % 7, 150 - r % 5
    rq = Requests(dim + 3, rows, lens, heads, kv, dim, cache, 16)
    rq.check(rq.run(causal=causal, window=window, sinks=sinks, max_rows=max_rows), causal=causal, window=window, sinks=sinks, oracle=plain.attention_many)


@pytest.mark.parametrize("cache,dim,heads,rows,length,pages", [("bf16", 64, 128, 200, 4500, (0, 7, 70, 150, 260, 281)), ("f16", 256, 64, 200, 2500, (3, 80, 120, 156))])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 4200, 70), (False, 2400, 3), (True, 300, 130)])
def test_missing_pages_of_whole_tiles_over_more_than_64_stages(cache, dim, heads, rows, length, pages, causal, window, sinks):
    """Pages that are not there, in the first positions, in front of windows and inside them, against a form that leaves their positions out."""
    rq = Requests(dim, [rows], [length], heads, heads, dim, cache, 16)
    here = torch.ones(length, dtype=torch.bool)
    ids = torch.from_numpy(rq.tables[0, :-1].astype(np.int64))
    for i, j in enumerate(pages):
        rq.tables[0, j] = (-1, rq.k.shape[0], 2 ** 31 - 1)[i % 3]
        here[16 * j:16 * j + 16] = False
    got = rq.run(causal=causal, window=window, sinks=sinks).cpu().double()
    p, key = (length - rows + torch.arange(rows))[:, None], torch.arange(length)[None, :]
    seen = here.expand(rows, length).clone()
    if causal:
        seen &= key <= p
    if window:
        seen &= ((p - key).abs() < window) | (key < sinks)
    u = half_step(rq.q.dtype)
    for h in range(heads):
        k, v = (x[ids, h].reshape(-1, dim)[:length].double() for x in (rq.k, rq.v))
        x = rq.q[:, h].double()
        w = torch.softmax((x @ k.t() * dim ** -0.5).masked_fill(~seen, float("-inf")), -1)
        want, size, big = w @ v, w @ v.abs(), (x.abs() @ k.abs().t()).masked_fill(~seen, 0.0).amax(-1, keepdim=True) * dim ** -0.5
        off = u + (dim + 4) * F * big + 8 * F + length * F / 4                                        # (as in Requests.check)
        bound = 2 * off * size * (1 + 4 * off) + u * want.abs() * (1 + u) + torch.finfo(rq.q.dtype).tiny * torch.finfo(rq.q.dtype).eps
        assert ((got[:, h] - want).abs() <= bound).all(), h
