"""The paged K/V operators against plain implementations in 64 bits (tests/paged_plain.py), element by element.

Tolerances count roundings.  u is half a step of the result's type (2^-11 binary16, 2^-8 bfloat16), f = 2^-24 that of 32 bits.
"""
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paged_plain as plain                                          # noqa: E402
from paper_2511_21759_amd import binding as B                        # noqa: E402

pytestmark = pytest.mark.gpu
F = 2.0 ** -24
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def half_step(dt):
    return torch.finfo(dt).eps / 2


def ints(x, device="cuda"):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=device)


def eager_generator(seed):
    return torch.Generator().manual_seed(seed)


# ---- page tables ------------------------------------------------------------------------------------------------------

def tables_case(seed, n, page, columns, spare, cap, bad=False):
    rng = random.Random(seed)
    most = columns * page
    held = [rng.choice([0, 1, page, rng.randint(0, most), most]) for _ in range(n)]
    wanted = [rng.choice([h, 0, min(h + 1, most), rng.randint(0, most), most]) for h in held]
    if bad:
        for r in range(0, n, 7):
            wanted[r] = rng.choice([-1, -2 ** 31, most + 1, 2 ** 31 - 1])
        for r in range(3, n, 11):
            held[r] = rng.choice([-5, most + 100, 2 ** 31 - 1])
    clamped = [min(max(h, 0), most) for h in held]
    need = [-(-h // page) for h in clamped]
    n_pages = max(1, sum(need) + spare)                  # (a pool of no pages is refused)
    ids = rng.sample(range(n_pages), n_pages)
    tables, at = np.full((n, columns), -7, np.int32), 0
    for r in range(n):
        tables[r, :need[r]] = ids[at:at + need[r]]
        at += need[r]
    free = np.full(n_pages, -9, np.int32)
    free[:spare] = ids[at:]
    first = [rng.randint(-3, most + 3) for _ in range(n)]
    count = [rng.choice([0, 1, rng.randint(0, 40), -4]) for _ in range(n)]
    return held, wanted, tables, free, spare, first, count


def run_tables(held, wanted, tables, free, n_free, page, first, count, cap):
    d = [ints(held), ints(wanted), ints(tables), ints(free), ints([n_free])]
    slots, positions = ints(np.full(cap, -77)), ints(np.full(cap, -77))
    first_d, count_d = (None if x is None else ints(x) for x in (first, count))
    out = []
    for _ in range(2):                                   # the second call writes the same again
        got = B.odb_page_tables(*d, page, len(free), row_first=first_d, row_count=count_d, slots=slots, positions=positions)
        length, cu, s, p, state = got
        out.append([x.cpu().numpy().copy() for x in (length, d[2], d[3], state, cu, s, p)])
    return out


@pytest.mark.parametrize("n,page,columns,spare,cap", [(1, 16, 1, 0, 1), (1, 16, 5, 9, 64), (3, 32, 4, 2, 50), (64, 16, 9, 30, 700), (65, 64, 3, 400, 2000),
                                                       (257, 16, 6, 100, 5000), (1000, 128, 4, 5000, 70000), (4096, 16, 3, 2000, 30000)])
@pytest.mark.parametrize("how", ["rows", "default", "bad"])
def test_page_tables_equal_the_sequential_form(n, page, columns, spare, cap, how):
    held, wanted, tables, free, n_free, first, count = tables_case(n * 31 + page, n, page, columns, spare, cap, how == "bad")
    if how == "default":
        first = count = None
    blank = np.full(cap, -77, np.int32)
    want = plain.page_tables(held, wanted, tables, free, n_free, page, first, count, cap, blank, blank)
    for got in run_tables(held, wanted, tables, free, n_free, page, first, count, cap):
        for g, w, name in zip(got, want, ("len", "tables", "free", "state", "cu_rows", "slots", "positions")):
            w = np.asarray(w, np.int64)
            assert np.array_equal(g.reshape(w.shape), w), (name, np.flatnonzero((g.reshape(w.shape) != w).reshape(-1))[:5])


def test_page_tables_hand_back_every_page_once():
    """Grow, cut, grow again for many steps: no page is ever in two places, none is lost."""
    rng, n, page, columns, n_pages = random.Random(5), 37, 16, 12, 260
    tables, free, n_free = ints(np.full((n, columns), -1)), ints(np.random.default_rng(1).permutation(n_pages)), ints([n_pages])
    held = ints(np.zeros(n))
    for _ in range(12):
        wanted = ints([rng.randint(0, columns * page) for _ in range(n)])
        length, cu, slots, positions, state = B.odb_page_tables(held, wanted, tables, free, n_free, page, n_pages, rows_cap=8000)
        held, n_free = length, state[:1].clone()
        t, lens, k = tables.cpu().numpy(), length.tolist(), int(n_free)
        used = [t[r, j] for r in range(n) for j in range(-(-lens[r] // page))]
        assert sorted(used + free[:k].tolist()) == list(range(n_pages))


# ---- angles -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n_pos,rot,base,kw", [
    (1, 2, 10000.0, {}), (7, 16, 10000.0, {}), (1000, 30, 500000.0, {}), (4096, 128, 1e6, {}),
    (333, 64, 10000.0, dict(scaling="linear", factor=4.0)), (50, 2, 10000.0, dict(scaling="ntk", factor=8.0)),
    (777, 128, 10000.0, dict(scaling="ntk", factor=3.5)), (2000, 128, 10000.0, dict(scaling="yarn", factor=16.0, original_len=4096)),
    (100, 256, 10000.0, dict(scaling="yarn", factor=2.0, original_len=77, beta_fast=8.0, beta_slow=0.0, magnitude=0.5)),
    (1 << 22, 6, 10000.0, {}),
])
def test_rope_table(n_pos, rot, base, kw):
    got = B.odb_rope_table(n_pos, rot, base, **kw)
    assert got.shape == (n_pos, rot // 2, 2) and got.dtype == torch.float32
    at = np.arange(n_pos) if n_pos <= 4096 else np.r_[0:100, n_pos // 2:n_pos // 2 + 1000, n_pos - 2000:n_pos]
    want = plain.rope_table(n_pos, rot, base, kw.get("scaling", "plain"), kw.get("factor", 1.0), kw.get("original_len", 0),
                            kw.get("beta_fast", 32.0), kw.get("beta_slow", 1.0), kw.get("magnitude", 0.0), at)
    err = np.abs(got.cpu().numpy()[at].astype(np.longdouble) - want)
    # one rounding of the value, and what the angle is off by: its extended-precision frequency by a few 2^-64 of at most 2^22
    assert (err <= F * np.abs(want) + 1e-11).all(), float(err.max())


# ---- norms and rotation -----------------------------------------------------------------------------------------------

def rotate_case(seed, rows, heads, kv, dim, given, cache, page):
    g = eager_generator(seed)
    qkv = torch.randn(rows, heads + 2 * kv, dim, generator=g).to(DT[given])
    n_pages = -(-max(rows, 1) // page) + 3
    pools = [torch.randn(n_pages, kv, page, dim, generator=g).to(DT[cache]) for _ in range(2)]
    slots = torch.randperm(n_pages * page, generator=g)[:rows].int()
    return g, qkv, pools, slots, n_pages


def check_rows(got, want, size, dt, steps, what):
    # `steps` roundings of 32 bits relative to the magnitudes that an element is made of, then one of the result's type (whose
    # smallest step is that of its subnormal numbers)
    tiny = torch.finfo(dt).tiny * torch.finfo(dt).eps / 2
    bound = half_step(dt) * want.abs() + (1 + half_step(dt)) * steps * F * size + tiny
    err = (got.double() - want).abs()
    assert (err <= bound).all(), (what, (err / bound).max().item())


@pytest.mark.parametrize("rows,heads,kv,dim,rot,given,cache,inter,norms,page", [
    (1, 1, 1, 64, 64, "f16", "f16", False, True, 16),
    (1, 32, 8, 128, 128, "bf16", "bf16", False, True, 16),
    (3, 5, 5, 128, 16, "bf16", "bf16", True, False, 32),
    (17, 7, 1, 256, 256, "f32", "bf16", False, True, 16),
    (33, 4, 2, 64, 32, "f32", "f16", False, False, 64),
    (33, 4, 2, 64, 32, "f32", "f16", True, True, 4096),
    (300, 12, 3, 128, 64, "f16", "f16", False, True, 128),
    (300, 12, 3, 256, 48, "f16", "f16", True, True, 16),
    (5000, 3, 1, 64, 48, "bf16", "bf16", False, True, 16),
])
def test_norm_rotation_and_store(rows, heads, kv, dim, rot, given, cache, inter, norms, page):
    g, qkv, pools, slots, n_pages = rotate_case(rows + dim, rows, heads, kv, dim, given, cache, page)
    n_pos = 600
    table = torch.from_numpy(plain.rope_table(n_pos, rot, 10000.0).astype(np.float32))
    positions = torch.randint(0, n_pos, (rows,), generator=g).int()
    gains = [1 + 0.3 * torch.randn(dim, generator=g) for _ in range(2)] if norms else [None, None]
    if rows > 16:                                   # padding rows, rows that are stored nowhere, slots outside the pool
        positions[3], positions[7], positions[9] = -1, n_pos, -2 ** 31
        slots[5], slots[8], slots[11] = -1, n_pages * page, 2 ** 31 - 1
    dev = qkv.cuda()
    k_dev, v_dev = (p.cuda() for p in pools)
    out = B.odb_qk_norm_rope(dev[:, :heads], dev[:, heads:heads + kv], dev[:, heads + kv:], k_dev, v_dev, table.cuda(), positions.cuda(),
                             slots.cuda(), q_gain=None if gains[0] is None else gains[0].cuda(),
                             k_gain=None if gains[1] is None else gains[1].cuda(), eps=1e-5, interleaved=inter)
    live = (positions >= 0) & (positions < n_pos)
    angles = table.double()[positions.long().clamp(0, n_pos - 1)]
    # mean of squares: 16 additions in a lane, up to four across lanes, each at most one rounding, half of them after the
    # root; scaling, root, division, two products; then two products and a sum: fewer than 24
    steps = 24
    q, size = plain.rotate(qkv[:, :heads].double(), None if gains[0] is None else gains[0].double(), 1e-5, angles, rot, inter)
    q[~live], size[~live] = 0, 0
    check_rows(out.cpu(), q, size, DT[cache], steps, "q")
    assert (out.cpu()[~live] == 0).all()
    k, size = plain.rotate(qkv[:, heads:heads + kv].double(), None if gains[1] is None else gains[1].double(), 1e-5, angles, rot, inter)
    want_k, want_v, size_k = pools[0].double(), pools[1].to(DT[cache]), torch.zeros_like(pools[0]).double()
    stored = live & (slots >= 0) & (slots < n_pages * page)
    at = slots[stored].long()
    want_k[at // page, :, at % page], size_k[at // page, :, at % page] = k[stored], size[stored]
    want_v[at // page, :, at % page] = qkv[:, heads + kv:].to(DT[cache])[stored]
    check_rows(k_dev.cpu(), want_k, size_k, DT[cache], steps, "k")
    assert torch.equal(v_dev.cpu(), want_v)


def test_rotation_in_place_and_through_strided_pools():
    """out = q inside a fused buffer; pools stored [page, position, head, channel]."""
    g, qkv, _, slots, n_pages = rotate_case(4, 40, 8, 4, 128, "bf16", "bf16", 16)
    table = B.odb_rope_table(64, 128, 10000.0)
    positions = torch.arange(40).int().cuda()
    dev = qkv.cuda()
    flat = [torch.zeros(n_pages, 16, 4, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    want_k, want_v = (torch.zeros(n_pages, 4, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    want = B.odb_qk_norm_rope(dev[:, :8], dev[:, 8:12], dev[:, 12:], want_k, want_v, table, positions, slots.cuda())
    got = B.odb_qk_norm_rope(dev[:, :8], dev[:, 8:12], dev[:, 12:], flat[0].permute(0, 2, 1, 3), flat[1].permute(0, 2, 1, 3), table, positions,
                             slots.cuda(), out=dev[:, :8])
    assert got.data_ptr() == dev.data_ptr() and torch.equal(got, want)
    assert torch.equal(flat[0].permute(0, 2, 1, 3), want_k) and torch.equal(flat[1].permute(0, 2, 1, 3), want_v)
    assert torch.equal(dev[:, 8:].cpu(), qkv[:, 8:])                  # keys and values of the fused buffer stay


# ---- attention --------------------------------------------------------------------------------------------------------

class Requests:
    """Random requests over a pool whose unused places hold what must not count: no numbers and infinities."""

    def __init__(self, seed, rows, lens, heads, kv, dim, cache, page, extra_columns=1, poison=True, sharp=1.5):
        g = eager_generator(seed)
        self.rows, self.lens, self.page = rows, lens, page
        need = [-(-max(length, 0) // page) for length in lens]
        n_pages = sum(need) + 2
        self.k, self.v = (torch.randn(n_pages, kv, page, dim, generator=g).to(DT[cache]) for _ in range(2))
        self.q = (sharp * torch.randn(sum(rows), heads, dim, generator=g)).to(DT[cache])
        ids = torch.randperm(n_pages, generator=g).tolist()
        self.tables, at = np.full((len(lens), max(need + [1]) + extra_columns), -1, np.int32), 0
        used = torch.zeros(n_pages, page, dtype=torch.bool)
        for r, length in enumerate(lens):
            mine = ids[at:at + need[r]]
            self.tables[r, :need[r]] = mine
            for j, page_id in enumerate(mine):
                used[page_id, :min(page, length - j * page)] = True
            at += need[r]
        if poison:
            hide = ~used[:, None, :, None].expand_as(self.k)
            self.k[hide], self.v[hide] = float("nan"), float("inf")

    def run(self, first=None, cu=True, **kw):
        cu_rows = ints(np.r_[0, np.cumsum(self.rows)]) if cu else None
        return B.odb_paged_attention(self.q.cuda(), self.k.cuda(), self.v.cuda(), ints(self.tables), ints(self.lens), cu_rows=cu_rows,
                                     first_pos=None if first is None else ints(first), **kw)

    def check(self, got, first=None, causal=False, window=0, sinks=0, scale=None, oracle=plain.attention):
        dim, dt = self.q.shape[2], self.q.dtype
        scale = dim ** -0.5 if scale is None else scale
        want, size, big = oracle(self.q.double(), self.k, self.v, self.tables, self.lens, self.rows, first, scale, causal, window, sinks)
        u = half_step(dt)
        # a probability is off by its rounding to the type, u, by that of the score's sum, dim F of sum |q||k| and F more for its
        # product with the scale, and by exp2, 4 F; numerator and denominator both; the sums over the keys add their number times F
        # times the largest (they are made in 16s: a quarter of that), and merged parts a few F more; then the result is rounded
        off = u + (dim + 4) * F * big[..., None] + 8 * F + max(self.lens + [1]) * F / 4
        bound = 2 * off * size * (1 + 4 * off) + u * want.abs() * (1 + u) + torch.finfo(dt).tiny * torch.finfo(dt).eps
        got = got.cpu().double()
        assert got.shape == want.shape and torch.isfinite(got).all()
        err = (got - want).abs()
        assert (err <= bound).all(), ((err / bound).max().item(), torch.nonzero(err > bound)[:3].tolist())


@pytest.mark.parametrize("cache", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv,dim", [(1, 1, 64), (8, 2, 128), (6, 6, 64), (7, 1, 128), (40, 2, 64), (4, 2, 256), (33, 1, 128), (70, 1, 256)])
def test_single_tokens(heads, kv, dim, cache):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 47, 64, 100, 129, 0, 257]
    rq = Requests(heads * dim, [1] * len(lens), lens, heads, kv, dim, cache, 16)
    for causal in (False, True):
        got = rq.run(causal=causal, cu=not causal)
        rq.check(got, causal=causal)
        assert (got[12] == 0).all()                       # no keys at all


@pytest.mark.parametrize("page", [16, 32, 256, 4096])
@pytest.mark.parametrize("max_len", [0, 600, 5])
def test_long_keys_split_over_workgroups(page, max_len):
    """Parts of one long and several short requests; a bound on the lengths that does not hold costs no correctness."""
    lens = [5000, 3, 1700, 0, 513]
    rq = Requests(page, [1] * 5, lens, 8, 2, 64, "bf16", page, extra_columns=3)
    rq.check(rq.run(causal=True, cu=False, max_len=max_len), causal=True)


@pytest.mark.parametrize("n,kv", [(64, 1), (65, 1), (300, 1), (300, 2), (700, 4), (4096, 1)])
@pytest.mark.parametrize("max_len", [0, 64])
def test_many_requests(n, kv, max_len):
    """Lists of requests longer than a wave, with and without split keys; most of them short, some without rows or keys."""
    rng = random.Random(n)
    lens = [rng.choice([0, 1, 17, 40, rng.randint(1, 60), 700 if rng.random() < 0.05 else 33]) for _ in range(n)]
    rows = [rng.choice([0, 1, 1, 1, min(3, max(1, length))]) for length in lens]
    rq = Requests(n + kv, rows, lens, 2 * kv, kv, 64, "f16", 16)
    rq.check(rq.run(causal=True, max_len=max_len), causal=True)


@pytest.mark.parametrize("cache,dim", [("f16", 64), ("bf16", 128), ("f16", 256)])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 1, 0), (True, 20, 3), (False, 20, 3), (True, 70, 40), (False, 300, 17), (True, 64, 2000)])
def test_ragged_rows_masks_and_sinks(cache, dim, causal, window, sinks):
    rows, lens = [5, 1, 33, 0, 70, 16], [40, 17, 210, 30, 70, 601]
    rq = Requests(dim + window, rows, lens, 6, 2, dim, cache, 32)
    rq.check(rq.run(causal=causal, window=window, sinks=sinks), causal=causal, window=window, sinks=sinks)


@pytest.mark.parametrize("cache,dim", [("f16", 64), ("bf16", 128), ("f16", 256)])
@pytest.mark.parametrize("rows", [[2, 1, 5, 0, 3, 4], [9, 1, 10, 0, 4, 7], [5, 1, 21, 0, 20, 16], [5, 1, 33, 0, 70, 16]])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 1700, 3), (False, 1700, 40), (True, 2000, 700)])
def test_ragged_rows_whose_keys_are_split_over_workgroups(cache, dim, rows, causal, window, sinks):
    """The tables are wide and the windows long, which is what the way of computing goes by; one request has many keys."""
    lens = [40, 17, 210, 30, 2300, 601]
    rq = Requests(dim + window + sum(rows), rows, lens, 6, 2, dim, cache, 32, extra_columns=300)
    rq.check(rq.run(causal=causal, window=window, sinks=sinks), causal=causal, window=window, sinks=sinks, oracle=plain.attention_many)


MANY = [("f16", 64, 64, 64), ("bf16", 128, 64, 64), ("bf16", 128, 96, 32), ("f16", 256, 40, 40), ("f16", 64, 120, 24)]


@pytest.mark.parametrize("cache,dim,heads,kv", MANY)
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 33, 5), (False, 100, 70), (True, 1, 0)])
def test_many_rows(cache, dim, heads, kv, causal, window, sinks):
    """Calls whose waves split the rows of a tile: row tiles and stages that are not full, requests without rows, lengths of one."""
    rows, lens = [260, 1, 0, 131, 64], [301, 1, 70, 131, 530]
    rq = Requests(dim + window + heads, rows, lens, heads, kv, dim, cache, 16)
    rq.check(rq.run(causal=causal, window=window, sinks=sinks), causal=causal, window=window, sinks=sinks, oracle=plain.attention_many)


@pytest.mark.parametrize("cache,dim,heads,kv", [("f16", 64, 16, 16), ("bf16", 128, 32, 32), ("f16", 256, 16, 16)])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 900, 5), (False, 300, 70)])
def test_many_rows_whose_keys_are_split_over_workgroups(cache, dim, heads, kv, causal, window, sinks):
    """Few row tiles and long keys: pieces that begin and end inside tiles, tiles that see much less than others."""
    rows, lens = [150, 0, 1, 129], [3500, 20, 1, 9000]
    rq = Requests(dim + window + heads, rows, lens, heads, kv, dim, cache, 16)
    cu = ints([0, 150, 150, 151, 280])                                     # rows that belong to no request stay
    q = torch.cat([rq.q, rq.q[:20]]).cuda()
    out = torch.full_like(q, 3.0)
    B.odb_paged_attention(q, rq.k.cuda(), rq.v.cuda(), ints(rq.tables), ints(rq.lens), causal=causal, window=window, sinks=sinks, cu_rows=cu, out=out)
    rq.check(out[:280], causal=causal, window=window, sinks=sinks, oracle=plain.attention_many)
    assert (out[280:] == 3.0).all()


@pytest.mark.parametrize("cache,dim", [("f16", 64), ("bf16", 128), ("f16", 256)])
@pytest.mark.parametrize("window,sinks", [(1, 50), (3, 700), (40, 45), (64, 2000)])
def test_positions_that_stay_visible_beyond_the_window(cache, dim, window, sinks):
    """... which, where rows see what lies behind them, are not the first of what a row sees: single tokens, few rows, keys split over workgroups, many
    rows, pieces of them."""
    for heads, kv, rows, lens, first, columns in ((4, 2, [1, 1, 5], [300, 40, 1000], [2, 39, 100], 1), (6, 2, [5, 1, 33], [40, 17, 2300], [0, 3, 9], 300),
                                                  (40, 40, [220, 130, 3], [220, 1000, 60], [0, 200, 1], 1), (16, 16, [150, 129], [3500, 9000], [7, 400], 1)):
        rq = Requests(dim + window + sum(rows), rows, lens, heads, kv, dim, cache, 16, extra_columns=columns)
        rq.check(rq.run(first=first, causal=False, window=window, sinks=sinks), first=first, window=window, sinks=sinks, oracle=plain.attention_many)


@pytest.mark.parametrize("cache,dim,heads,kv,rows,lens", [
    ("f16", 64, 32, 32, [66, 100, 1, 0, 70, 99, 80, 65, 91], [900, 101, 1, 40, 70, 0, 333, 640, 257]),                     # whole tiles
    ("bf16", 128, 96, 32, [23, 33, 1, 42, 30, 24, 29, 1, 36], [900, 101, 1, 40, 70, 0, 333, 640, 257]),
    ("f16", 64, 32, 32, [70, 80, 66, 1, 96], [4100, 1300, 70, 0, 2500]),                                                   # pieces
    ("bf16", 256, 48, 16, [20, 11, 17, 0, 1, 20], [4100, 50, 700, 9, 1, 1200])])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 600, 9)])
@pytest.mark.parametrize("hint", [1.0, 0.7])
def test_requests_that_fill_more_than_half_of_a_tile(cache, dim, heads, kv, rows, lens, causal, window, sinks, hint):
    """... of many rows, with a bound on the rows that holds, and one that does not."""
    rq = Requests(dim + len(rows), rows, lens, heads, kv, dim, cache, 16)
    got = rq.run(causal=causal, window=window, sinks=sinks, max_rows=int(hint * max(rows)))
    rq.check(got, causal=causal, window=window, sinks=sinks, oracle=plain.attention_many)


@pytest.mark.parametrize("cache,dim,heads,rows,length", [("bf16", 64, 128, 200, 4500), ("f16", 256, 64, 200, 2500)])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 4200, 70), (False, 2400, 3)])
def test_whole_tiles_over_more_than_64_stages(cache, dim, heads, rows, length, causal, window, sinks):
    rq = Requests(dim, [rows], [length], heads, heads, dim, cache, 16)
    rq.tables[0, 7] = -1                                                   # a page that is not there, which the oracle sees as a hole
    got = rq.run(causal=causal, window=window, sinks=sinks)
    rq.tables[0, :-1] = np.r_[rq.tables[0, :7], rq.tables[0, 8:]]          # (positions behind it are 16 lower for the oracle, and so are the rows)
    if window == 0:
        rq.lens = [length - 16]
        rq.check(got, first=[length - rows - 16], causal=causal, oracle=plain.attention_many)
    rq = Requests(dim + 1, [rows], [length], heads, heads, dim, cache, 32)
    rq.check(rq.run(causal=causal, window=window, sinks=sinks), causal=causal, window=window, sinks=sinks, oracle=plain.attention_many)


@pytest.mark.parametrize("n", [250, 600])
def test_split_rows_over_many_requests(n):
    """Many requests, one or two of many rows, most of one or none; their tables are wide, which is what the way of computing goes by."""
    rng = random.Random(8)
    lens = [rng.choice([1, 5, 33, 70]) for _ in range(n)]
    rows = [int(rng.random() < 20 / n) for _ in lens]
    for r in (3, 177) if n == 250 else (599,):
        lens[r], rows[r] = 1800 + r, 150
    rq = Requests(77, rows, lens, 1, 1, 64, "f16", 16, extra_columns=900)
    rq.check(rq.run(causal=True, max_rows=150), causal=True, oracle=plain.attention_many)


def test_many_rows_at_given_positions_and_with_hidden_numbers():
    rows, lens, first = [200, 200, 130], [400, 250, 130], [150, -20, 100]
    rq = Requests(71, rows, lens, 64, 64, 64, "f16", 32)
    for causal in (False, True):
        rq.check(rq.run(first=first, causal=causal), first=first, causal=causal, oracle=plain.attention_many)
    # a key that half of a tile's rows see holds no number: the others stay as they were
    clean = rq.run(first=first, causal=True).cpu()
    page_id, at = int(rq.tables[0, 200 // 32]), 200 % 32
    for pool in (rq.v, rq.k):
        keep = pool[page_id, :, at].clone()
        pool[page_id, :, at] = float("nan")
        got = rq.run(first=first, causal=True).cpu()
        assert torch.equal(got[:50], clean[:50]) and torch.isnan(got[50:200]).all() and torch.equal(got[200:], clean[200:])
        pool[page_id, :, at] = keep
    # a page outside the pool, in the middle and at the end
    rq.tables[0, 3], rq.tables[2, 4] = -1, rq.k.shape[0]
    gone = torch.ones(400, dtype=torch.bool)
    gone[96:128] = False
    got = rq.run(first=first, causal=False).cpu()
    q64, ids = rq.q.double(), torch.tensor(rq.tables[0, :13].astype(np.int64)).clamp(min=0)
    for h in (0, 63):
        k, v = (x[ids, h].reshape(-1, 64)[:400][gone].double() for x in (rq.k, rq.v))
        w = torch.softmax(q64[:200, h] @ k.t() * 0.125, -1)
        # (bounds as in check(), with the largest sum |q||k| of all rows)
        off = 2.0 ** -11 + 80 * F * (q64[:200, h].abs() @ k.abs().t()).max() * 0.125 + 8 * F + 400 * F / 4
        assert ((got[:200, h].double() - w @ v).abs() <= 2.1 * off * (w @ v.abs()) + 2.0 ** -11 * (w @ v).abs() + 1e-7).all()


@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 9, 2), (False, 9, 2)])
def test_rows_at_given_positions(causal, window, sinks):
    """Blocks in the middle of a sequence, rows before its start (they see nothing, or what a window reaches) and behind its end."""
    rows, lens, first = [32, 32, 8, 8, 8], [300, 64, 50, 50, 50], [100, 0, -4, 46, 2 ** 31 - 40]
    rq = Requests(3, rows, lens, 4, 4, 128, "f16", 16)
    got = rq.run(first=first, causal=causal, window=window, sinks=sinks)
    rq.check(got, first=first, causal=causal, window=window, sinks=sinks)


def test_windows_that_reach_over_the_ends():
    """Rows before the first position and behind the last whose window reaches back to it, with sinks and without."""
    rows, lens, first = [4, 3, 5, 1], [50, 300, 40, 700], [-7, -300, 45, 705]
    for max_len in (0, 5000):
        for sinks in (0, 3):
            rq = Requests(5 + sinks, rows, lens, 2, 1, 64, "f16", 16, extra_columns=100 if max_len else 1)
            rq.check(rq.run(first=first, causal=False, window=9, sinks=sinks), first=first, window=9, sinks=sinks)
            rq.check(rq.run(first=first, causal=True, window=9, sinks=sinks), first=first, causal=True, window=9, sinks=sinks)


def test_no_number_at_hidden_places_of_a_visible_block():
    """Causal rows and a window: keys that some rows of a tile see and others do not hold infinities and no numbers; the rows
    that do not see them stay finite and right, the others show it."""
    rq = Requests(9, [40], [100], 4, 2, 64, "f16", 16)
    page_id, at = int(rq.tables[0, 90 // 16]), 90 % 16
    clean = rq.v[page_id, :, at].clone()
    rq.v[page_id, :, at, :32], rq.v[page_id, :, at, 32:] = float("nan"), float("inf")
    got = rq.run(causal=True).cpu()
    assert torch.isnan(got[30:, :, :32]).all() and (got[30:, :, 32:] == float("inf")).all()       # rows at 60 ..: 90 is row 30
    rq.v[page_id, :, at] = clean
    clean_got = rq.run(causal=True)
    rq.check(clean_got, causal=True)
    assert torch.equal(got[:30], clean_got.cpu()[:30])
    rq.k[page_id, :, at] = float("nan")
    got = rq.run(causal=True).cpu()
    assert torch.equal(got[:30], clean_got.cpu()[:30]) and torch.isnan(got[30:]).all()


def test_pages_outside_the_pool_are_seen_by_nobody():
    rq = Requests(11, [1, 3, 20], [200, 90, 333], 8, 2, 128, "bf16", 16)
    rq.tables[0, 2], rq.tables[1, 0], rq.tables[2, 5], rq.tables[2, 20] = -1, rq.k.shape[0], 2 ** 31 - 1, -2 ** 31
    for causal in (True, False):
        rq.check(rq.run(causal=causal), causal=causal)
    rq.tables[:] = -1
    assert (rq.run(causal=False) == 0).all()


def test_rows_of_no_request_stay():
    rq = Requests(12, [3, 0, 2], [50, 9, 70], 4, 2, 64, "f16", 16)
    q = torch.cat([rq.q, rq.q, rq.q]).cuda()
    for max_len in (0, 5000):                              # one launch, and two with split keys
        tables = np.pad(rq.tables, ((0, 0), (0, 300)), constant_values=-1)
        out = torch.full_like(q, 7.0)
        B.odb_paged_attention(q, rq.k.cuda(), rq.v.cuda(), ints(tables), ints(rq.lens), causal=True, cu_rows=ints([0, 3, 3, 5]), out=out,
                              max_len=max_len)
        rq.check(out[:5], causal=True)
        assert (out[5:] == 7.0).all()


def test_strided_rows_and_pools_and_a_given_workspace():
    rq = Requests(13, [2, 30, 1], [700, 65, 1200], 6, 3, 128, "bf16", 32, poison=False)
    want = rq.run(causal=True)
    rq.check(want, causal=True)
    wide = torch.zeros(33, 10, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:8] = rq.q.cuda()
    k, v = (x.cuda().permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for x in (rq.k, rq.v))
    out = torch.full((33, 9, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    work = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    got = B.odb_paged_attention(wide[:, 2:8], k, v, ints(rq.tables), ints(rq.lens), causal=True, cu_rows=ints([0, 2, 32, 33]), out=out[:, 3:],
                                workspace=work)
    assert torch.equal(got, want) and (out[:, :3] == 5.0).all()
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.OdbError, match="workspace"):
        B.odb_paged_attention(wide[:, 2:8], k, v, ints(rq.tables), ints(rq.lens), causal=True, cu_rows=ints([0, 2, 32, 33]), workspace=small)


@pytest.mark.parametrize("cache", ["f16", "bf16"])
def test_scores_far_apart_rising_and_equal(cache):
    """The reference of the running softmax is raised block after block; all keys equal; one key far above the rest."""
    rq = Requests(17, [1, 1, 1], [900, 900, 900], 2, 1, 64, cache, 16)
    ramp = torch.linspace(-40, 40, 900)
    for j, page_id in enumerate(rq.tables[0, :57]):
        n = min(16, 900 - 16 * j)
        rq.k[page_id, :, :n] = 0
        rq.k[page_id, :, :n, 0] = ramp[16 * j:16 * j + n].to(DT[cache])
    for j, page_id in enumerate(rq.tables[1, :57]):
        rq.k[page_id, :, :min(16, 900 - 16 * j)] = 0.25
    rq.q[0] = 0
    rq.q[0, :, 0] = torch.tensor([30.0, -30.0]).to(DT[cache])
    rq.k[rq.tables[2, 31], :, 3] = 40 * rq.q[2, 0]
    rq.check(rq.run(causal=False, scale=1.0), scale=1.0)


def test_offsets_beyond_32_bits():
    """Pages more than 2^32 elements from the pool's start (the pools overlap in one buffer of 9.7 GB)."""
    page, kv, dim = 16, 1, 64
    stride = 1 << 30
    buf = torch.empty(4 * stride + (1 << 20), dtype=torch.float16, device="cuda")
    k = buf.as_strided((5, kv, page, dim), (stride, page * dim, dim, 1))
    v = buf[1 << 19:].as_strided((5, kv, page, dim), (stride, page * dim, dim, 1))
    rq = Requests(19, [1, 4], [30, 45], 2, 1, 64, "f16", 16)
    ids = [4, 2, 0, 3, 1]
    k.zero_(), v.zero_()
    tables, at = np.full_like(rq.tables, -1), 0
    for r, need in enumerate((2, 3)):
        for j in range(need):
            k[ids[at]], v[ids[at]] = rq.k[rq.tables[r, j]].cuda(), rq.v[rq.tables[r, j]].cuda()
            tables[r, j] = ids[at]
            at += 1
    got = B.odb_paged_attention(rq.q.cuda(), k, v, ints(tables), ints(rq.lens), causal=True, cu_rows=ints([0, 1, 5]))
    rq.check(got, causal=True)
    # and rows stored there
    table = B.odb_rope_table(64, 64, 10000.0)
    qkv = torch.randn(3, 3, 64, device="cuda").half()
    B.odb_qk_norm_rope(qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], k, v, table, ints([0, 0, 0]), ints([4 * 16 + 5, 3, 16]))
    assert torch.equal(v[4, 0, 5], qkv[0, 2]) and torch.equal(v[0, 0, 3], qkv[1, 2]) and torch.equal(k[1, 0, 0], qkv[2, 1])


# ---- as they are used together ----------------------------------------------------------------------------------------

def serve(steps, device, stream=None, graphed=False):
    """Some steps of three requests that are prefilled, decode a token each and get cut: tables, rotation, attention."""
    g = eager_generator(23)
    heads, kv, dim, page, columns, n_pages = 8, 2, 128, 16, 12, 24
    dev = torch.device(device)
    table = B.odb_rope_table(256, dim, 10000.0, device=dev)
    k_pages, v_pages = (torch.zeros(n_pages, kv, page, dim, dtype=torch.bfloat16, device=dev) for _ in range(2))
    tables, free = ints(np.full((3, columns), -1), dev), ints(np.arange(n_pages)[::-1].copy(), dev)
    n_free, held = ints([n_pages], dev), ints([0, 0, 0], dev)
    history, outs = [[torch.zeros(0, kv, dim)] * 2 for _ in range(3)], []
    plan = [[40, 3, 100], [41, 4, 101], [42, 5, 80], [43, 60, 81], [20, 61, 82], [21, 62, 83]][:steps]
    lens = [0, 0, 0]
    for want in plan:
        rows = [max(0, w - h) for w, h in zip(want, lens)]
        qkv = torch.randn(max(1, sum(rows)), heads + 2 * kv, dim, generator=g).bfloat16()
        dev_qkv = qkv.to(dev)
        length, cu, slots, positions, state = B.odb_page_tables(held, ints(want, dev), tables, free, n_free, page, n_pages, rows_cap=qkv.shape[0])
        q = B.odb_qk_norm_rope(dev_qkv[:, :heads], dev_qkv[:, heads:heads + kv], dev_qkv[:, heads + kv:], k_pages, v_pages, table, positions, slots)
        out = B.odb_paged_attention(q, k_pages, v_pages, tables, length, causal=True, cu_rows=cu)
        held, n_free = length, state[:1].clone()
        # the same in 64 bits on dense caches, from the rounded K and Q that the pages hold
        angles = plain.rope_table(256, dim, 10000.0)
        at = 0
        for r in range(3):
            new = qkv[at:at + rows[r]]
            pos = np.arange(lens[r], lens[r] + rows[r])
            a = torch.from_numpy(angles[pos].astype(np.float64))
            k = plain.rotate(new[:, heads:heads + kv].double(), None, 0, a, dim, False)[0]
            history[r] = [torch.cat([history[r][0], k])[:want[r]], torch.cat([history[r][1], new[:, heads + kv:].double()])[:want[r]]]
            q64 = plain.rotate(new[:, :heads].double(), None, 0, a, dim, False)[0]
            for i in range(rows[r]):
                n = lens[r] + i + 1
                for h in range(heads):
                    w = torch.softmax(history[r][0][:n, h // 4] @ q64[i, h] * dim ** -0.5, 0)
                    outs.append((out[at + i, h].cpu().double(), w @ history[r][1][:n, h // 4], w @ history[r][1][:n, h // 4].abs(), q64[i, h], history[r][0][:n, h // 4]))
            at += rows[r]
        lens = list(want)
        assert length.tolist() == want
    return outs


def test_steps_of_growing_and_cut_requests():
    u = half_step(torch.bfloat16)
    for got, want, size, q, k in serve(6, "cuda"):
        # Q and K are rounded on the way: a score is off by 2 u of sum |q||k| (and a little for 32 bits)
        off = 2.1 * u * (q.abs() @ k.abs().t()).max() * 128 ** -0.5 + u
        assert ((got - want).abs() <= 2 * off * size * torch.exp(2 * off) + 1.01 * u * want.abs() + 1e-6).all()


def test_captured_steps_equal_eager_ones_and_two_graphs_do_not_meet():
    """A captured step is replayed with new lengths and inputs; another graph of the same pool of memory runs in between."""
    heads, kv, dim, page, n_pages, n = 8, 2, 128, 16, 400, 4
    g = torch.Generator(device="cuda").manual_seed(3)
    table = B.odb_rope_table(2048, dim, 10000.0)
    tables = torch.randperm(n_pages, generator=g, device="cuda").int()[:n * 90].view(n, 90).contiguous()

    def make():
        pools = [torch.randn(n_pages, kv, page, dim, generator=g, device="cuda").half() for _ in range(2)]
        return dict(pools=pools, qkv=torch.randn(n, heads + 2 * kv, dim, generator=g, device="cuda").half(), held=ints([7, 100, 900, 1300]), tables=tables.clone(),
                    free=ints(np.arange(n_pages)), n_free=ints([40]), slots=ints([-1] * n), positions=ints([0] * n))

    def step(s):
        wanted = s["held"] + 1
        length, cu, slots, positions, state = B.odb_page_tables(s["held"], wanted, s["tables"], s["free"], s["n_free"], page, n_pages, slots=s["slots"],
                                                                positions=s["positions"])
        q = B.odb_qk_norm_rope(s["qkv"][:, :heads], s["qkv"][:, heads:heads + kv], s["qkv"][:, heads + kv:], *s["pools"], table, positions, slots)
        out = B.odb_paged_attention(q, *s["pools"], s["tables"], length, causal=True, cu_rows=cu)
        return out, length, slots, state

    sides = [make(), make()]
    for s in sides:
        step(s)
    torch.cuda.synchronize()
    graphs = []
    for s in sides:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            s["out"] = step(s)
        graphs.append(gr)
    for turn in range(4):
        for s in sides:
            s["qkv"].copy_(torch.randn(s["qkv"].shape, generator=g, device="cuda"))
            s["held"].copy_(ints([[7, 100, 900, 1300], [8, 15, 16, 17], [1400, 1, 0, 31], [64, 63, 62, 1000]][turn]))
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        for s in sides:
            got = [x.clone() for x in s["out"]]
            for x, y in zip(got, step(s)):
                assert torch.equal(x, y), turn


def test_two_streams_at_once():
    """Two calls with keys split over workgroups overlap on two streams: each has a workspace of its own."""
    sets = [Requests(29 + i, [1, 1], [4000 + 100 * i, 3000], 8, 2, 128, "f16", 16) for i in range(2)]
    args = [(r.q.cuda(), r.k.cuda(), r.v.cuda(), ints(r.tables), ints(r.lens)) for r in sets]
    alone = [B.odb_paged_attention(*a, causal=True) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[], []]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                outs[i].append(B.odb_paged_attention(*args[i], causal=True))
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            assert torch.equal(o, alone[i])
        sets[i].check(alone[i], causal=True)
