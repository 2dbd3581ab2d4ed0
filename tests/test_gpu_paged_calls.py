"""Calls of the paged K/V operators that a serving program makes beside the ordinary ones: buffers larger than a step's rows, captured
steps that get shorter, scores far outside the usual range.  Plain forms and bounds are those of test_gpu_paged.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paged_plain as plain                                          # noqa: E402
from paper_2511_21759_amd import binding as B                        # noqa: E402

pytestmark = pytest.mark.gpu
F = 2.0 ** -24


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


# ---- rows behind a step's last one ---------------------------------------------------------------------------------------

def test_entries_behind_the_last_row_of_own_buffers_are_padding():
    """Without given buffers the binding allocates slots and positions; torch hands out memory that was used before."""
    cap = 4096
    for _ in range(3):
        old = [torch.full((k * cap,), 5, dtype=torch.int32, device="cuda") for k in (1, 1, 2)]
        del old
        length, cu, slots, positions, state = B.odb_page_tables(ints([0, 7]), ints([3, 8]), ints([[-1, -1], [2, -1]]), ints([0, 1, 3, 4]), ints([2]), 16, 4,
                                                                rows_cap=cap)
        assert cu.tolist() == [0, 3, 4]
        assert slots.tolist()[:4] == [16, 17, 18, 2 * 16 + 7] and positions.tolist()[:4] == [0, 1, 2, 7]
        assert (slots[4:] == -1).all() and (positions[4:] == -1).all()


class Step:
    """A step of at most `cap` rows over buffers that stay: tables, rotation and store, attention."""
    heads, kv, dim, page, n_pages, columns = 4, 2, 64, 16, 60, 9

    def __init__(self, n, cap, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.n = n
        self.pools = [torch.randn(self.n_pages, self.kv, self.page, self.dim, generator=g, device="cuda").half() for _ in range(2)]
        self.qkv = torch.randn(cap, self.heads + 2 * self.kv, self.dim, generator=g, device="cuda").half()
        ids = torch.randperm(self.n_pages, generator=g, device="cuda").int()
        self.tables = ids[:n * self.columns].view(n, self.columns).contiguous()
        self.free, self.n_free = torch.zeros(self.n_pages, dtype=torch.int32, device="cuda"), ints([0])
        self.held, self.first, self.count = ints([0] * n), ints([0] * n), ints([0] * n)
        self.slots, self.positions = ints([-1] * cap), ints([-1] * cap)
        self.table = B.odb_rope_table(self.page * self.columns, self.dim, 10000.0)

    def run(self):
        length, cu, slots, positions, _ = B.odb_page_tables(self.held, self.held, self.tables, self.free, self.n_free, self.page, self.n_pages, slots=self.slots,
                                                            positions=self.positions, row_first=self.first, row_count=self.count)
        h, kv = self.heads, self.kv
        q = B.odb_qk_norm_rope(self.qkv[:, :h], self.qkv[:, h:h + kv], self.qkv[:, h + kv:], *self.pools, self.table, positions, slots, row_end=cu[self.n:])
        return q, B.odb_paged_attention(q, *self.pools, self.tables, length, causal=True, cu_rows=cu, first_pos=self.first)

    def set(self, held, first, count):
        for to, x in ((self.held, held), (self.first, first), (self.count, count)):
            to.copy_(ints(x))


@pytest.mark.parametrize("graphed", [False, True])
def test_a_long_step_followed_by_shorter_ones_stores_live_rows_only(graphed):
    """Slots and positions keep the entries of the longer step behind the last row; row_end says where the rows end."""
    n, cap = 3, 48
    s = Step(n, cap, 4)
    s.set([100, 90, 140], [80, 70, 140], [20, 20, 0])
    s.run()
    torch.cuda.synchronize()
    if graphed:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = s.run()
    for held, first, count in (([100, 90, 140], [80, 70, 120], [20, 8, 20]), ([101, 91, 141], [100, 90, 140], [1, 1, 1]), ([102, 90, 141], [101, 90, 0], [1, 0, 0]),
                               ([0, 0, 0], [0, 0, 0], [0, 0, 0]), ([110, 90, 144], [100, 60, 142], [10, 30, 2])):
        s.set(held, first, count)
        s.qkv.copy_(torch.randn(s.qkv.shape, generator=torch.Generator().manual_seed(sum(held))))
        before = [x.clone() for x in s.pools]
        if graphed:
            graph.replay()
        else:
            out = s.run()
        torch.cuda.synchronize()
        q = out[0].clone()
        live = sum(count)
        assert (q[live:] == 0).all() and (q[:live] != 0).any(-1).all()
        at = [(r, p) for r in range(n) for p in range(first[r], first[r] + count[r])]
        slots = [int(s.tables[r, p // 16]) * 16 + p % 16 for r, p in at]
        for pool, was, lane in ((s.pools[0], before[0], slice(4, 6)), (s.pools[1], before[1], slice(6, 8))):
            changed = (pool != was).any(-1).any(1).reshape(-1).nonzero().flatten().tolist()
            assert changed == sorted(slots)
        for i, slot in enumerate(slots):
            assert torch.equal(s.pools[1][slot // 16, :, slot % 16], s.qkv[i, 6:8])


@pytest.mark.parametrize("end,live", [(0, 0), (-5, 0), (-2 ** 31, 0), (3, 3), (20, 20), (21, 20), (2 ** 31 - 1, 20)])
def test_row_end_of_any_value(end, live):
    s = Step(1, 20, 9)
    s.positions.copy_(torch.arange(20)), s.slots.copy_(torch.arange(20) + 32)
    before = [x.clone() for x in s.pools]
    q = B.odb_qk_norm_rope(s.qkv[:, :4], s.qkv[:, 4:6], s.qkv[:, 6:], *s.pools, s.table, s.positions, s.slots, row_end=ints([end]))
    want_pools = [x.clone() for x in before]
    cut = s.slots.clone()
    cut[live:] = -1
    want = B.odb_qk_norm_rope(s.qkv[:, :4], s.qkv[:, 4:6], s.qkv[:, 6:], *want_pools, s.table, s.positions, cut)
    assert torch.equal(q[:live], want[:live]) and (q[live:] == 0).all()
    for x, y in zip(s.pools, want_pools):
        assert torch.equal(x, y)


# ---- scores far outside the usual range -----------------------------------------------------------------------------------

# (rows of each request, positions, query heads, K/V heads, head size, page, columns beside those that are needed): what reaches each
# way of computing - keys whole and split over workgroups with 1, 2 and 4 row tiles, many rows whole and in pieces
WAYS = [([1, 1], [100, 333], 4, 2, 64, 16, 1), ([1, 1], [1700, 900], 4, 2, 128, 32, 300), ([5, 3], [200, 150], 8, 2, 128, 16, 1),
        ([9, 9], [1500, 2000], 6, 2, 256, 16, 100), ([33, 40], [2000, 900], 4, 2, 64, 32, 300), ([40, 20], [300, 70], 4, 2, 128, 32, 1),
        ([260, 131], [301, 140], 64, 64, 64, 16, 1), ([150, 129], [3500, 2000], 16, 16, 64, 16, 500), ([150], [1500], 16, 16, 256, 16, 400)]


@pytest.mark.parametrize("cache", ["f16", "bf16"])
@pytest.mark.parametrize("rows,lens,heads,kv,dim,page,more", WAYS)
@pytest.mark.parametrize("power,step,scale", [(18, 0, 1.0), (23, 0, 1.0), (25, 2, 1.0), (27, 4, 2.0 ** -4), (27, 4, 1.0), (28, 5, 1.0), (30, 7, 2.0 ** -2)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_any_size(rows, lens, heads, kv, dim, page, more, cache, power, step, scale, sign):
    """Scores sign * 2^power + 2^step * f, f whole numbers: exact in 32 bits, whatever the order of their sums, so the softmax is known."""
    dt = torch.float16 if cache == "f16" else torch.bfloat16
    g = torch.Generator().manual_seed(power + dim)
    need = [-(-x // page) for x in lens]
    n_pages = sum(need) + 1
    k, v = torch.zeros(n_pages, kv, page, dim), torch.randn(n_pages, kv, page, dim, generator=g).to(dt)
    q = torch.zeros(sum(rows), heads, dim)
    q[..., 0], q[..., 1] = 2.0 ** step, sign * 2.0 ** (power // 2)
    # f of every 16 keys reaches 12 once; the first block of a request lies 2^(power - 4) lower, so that references are raised
    f = torch.randint(0, 12, (n_pages, 1, page), generator=g).float().expand(n_pages, kv, page).clone()
    f[:, :, ::16] = 12
    k[..., 0], k[..., 1] = f, 2.0 ** (power - power // 2)
    tables, at = np.full((len(lens), max(need) + more), -1, np.int32), 0
    ids = torch.randperm(n_pages, generator=g).tolist()
    for r, x in enumerate(need):
        tables[r, :x] = ids[at:at + x]
        at += x
        if lens[r] > 64:
            k[tables[r, 0], :, :16, 1] -= sign * 2.0 ** (power - power // 2 - 4)
    q, k = q.to(dt), k.to(dt)
    cu = ints(np.r_[0, np.cumsum(rows)])
    got = B.odb_paged_attention(q.cuda(), k.cuda(), v.cuda(), ints(tables), ints(lens), causal=True, cu_rows=cu, scale=scale).cpu().double()
    want, size, _ = plain.attention_many(q.double(), k, v, tables, lens, rows, None, scale, True, 0, 0)
    # A probability is off by its rounding u to the type; by exp2, 4 F; by the 32-bit forms of scale * log2(e), 2 F of the distance of a score
    # from the largest, which is at most 12 steps where the probability counts, and below 2^15, where references are not taken from
    # scores, of the score; numerator and denominator both.  The sums over the keys add their number times F / 4.
    u = torch.finfo(dt).eps / 2
    off = u + 4 * F + 2 * F * 1.45 * scale * 12 * 2.0 ** step + max(lens) * F / 4
    bound = 2 * off * size * (1 + 4 * off) + u * want.abs() * (1 + u) + torch.finfo(dt).tiny
    assert torch.isfinite(got).all()
    err = (got - want).abs()
    assert (err <= bound).all(), (err / bound).max().item()


@pytest.mark.parametrize("cache", ["f16", "bf16"])
@pytest.mark.parametrize("rows,lens,heads,kv,dim,page,more", WAYS)
@pytest.mark.parametrize("sign", [1, -1])
def test_rows_whose_scores_are_beyond_the_range_become_no_numbers(rows, lens, heads, kv, dim, page, more, cache, sign):
    """The first row of each request has scores of 2^29 and more in units of log2; the others stay what they are."""
    dt = torch.float16 if cache == "f16" else torch.bfloat16
    g = torch.Generator().manual_seed(dim)
    need = [-(-x // page) for x in lens]
    k, v = (torch.randn(sum(need), kv, page, dim, generator=g) for _ in range(2))
    k[..., 0] = 2.0 ** 15
    tables, at = np.full((len(lens), max(need) + more), -1, np.int32), 0
    for r, x in enumerate(need):
        tables[r, :x] = np.arange(at, at + x)
        at += x
    q = torch.randn(sum(rows), heads, dim, generator=g)
    q[..., 0] = 0
    cu = np.r_[0, np.cumsum(rows)]
    args = k.to(dt).cuda(), v.to(dt).cuda(), ints(tables), ints(lens)
    kw = dict(causal=False, cu_rows=ints(cu), scale=1.0)
    q[cu[:-1], :, 0] = sign * 2.0 ** 14
    q = q.to(dt)
    got = B.odb_paged_attention(q.cuda(), *args, **kw).cpu().double()
    beyond = torch.zeros(sum(rows), dtype=torch.bool)
    beyond[cu[:-1]] = True
    assert got[beyond].isnan().all() and torch.isfinite(got[~beyond]).all()
    want, size, big = plain.attention_many(q.double(), k.to(dt), v.to(dt), tables, lens, rows, None, 1.0, False, 0, 0)
    # the bound of test_gpu_paged.py; the other rows are not the same to the last bit as without these neighbours, since rows of a tile raise
    # their references together, which moves the roundings of their probabilities
    u = torch.finfo(dt).eps / 2
    off = u + (dim + 4) * F * big[..., None] + 8 * F + max(lens) * F / 4
    bound = 2 * off * size * (1 + 4 * off) + u * want.abs() * (1 + u) + torch.finfo(dt).tiny * torch.finfo(dt).eps
    assert ((got - want).abs()[~beyond] <= bound[~beyond]).all()


# ---- in place -------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows", [1, 2, 33])
@pytest.mark.parametrize("order", ["qkv", "kvq", "vqk"])
def test_rotation_in_place_with_keys_and_values_on_either_side(rows, order):
    g = torch.Generator().manual_seed(rows)
    width = dict(q=4, k=2, v=2)
    fused = torch.randn(rows, 8, 64, generator=g).half().cuda()
    at, parts = 0, {}
    for name in order:
        parts[name] = fused[:, at:at + width[name]]
        at += width[name]
    table, positions, slots = B.odb_rope_table(64, 64, 10000.0), ints(np.arange(rows)), ints(np.arange(rows)[::-1] + 5)
    pools = [[torch.zeros(6, 2, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2)] for _ in range(2)]
    want = B.odb_qk_norm_rope(parts["q"], parts["k"], parts["v"], *pools[0], table, positions, slots)
    before = {name: x.clone() for name, x in parts.items()}
    got = B.odb_qk_norm_rope(parts["q"], parts["k"], parts["v"], *pools[1], table, positions, slots, out=parts["q"])
    assert got.data_ptr() == parts["q"].data_ptr() and torch.equal(got, want)
    assert all(torch.equal(parts[x], before[x]) for x in "kv") and all(torch.equal(x, y) for x, y in zip(*pools))


def test_queries_that_are_also_the_keys():
    """One tensor as Q and K: right into another buffer, refused in place, where keys would be read after they were turned."""
    x = torch.randn(20, 2, 64, generator=torch.Generator().manual_seed(1)).half().cuda()
    table, positions, slots = B.odb_rope_table(64, 64, 10000.0), ints(np.arange(20)), ints(np.arange(20))
    k, v = (torch.zeros(2, 2, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    q = B.odb_qk_norm_rope(x, x, x, k, v, table, positions, slots)
    assert torch.equal(q, k.permute(0, 2, 1, 3).reshape(-1, 2, 64)[:20])
    with pytest.raises(B.OdbError, match="in place"):
        B.odb_qk_norm_rope(x, x, x, k, v, table, positions, slots, out=x)
