"""Attention over pages of 8-bit codes against a plain implementation in 64 bits (tests/paged_plain.py), element by element.

Tolerances count roundings.  u is half a step of the result's type (2^-11 binary16, 2^-8 bfloat16), f = 2^-24 that of 32 bits.
"""
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paged_plain as plain                                          # noqa: E402
import quant_plain as quant                                          # noqa: E402
from paper_2511_21759_amd import binding as B                        # noqa: E402

pytestmark = pytest.mark.gpu
F, U16 = 2.0 ** -24, 2.0 ** -11
DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def ints(x, device="cuda"):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=device)


class Requests:
    """Random requests over a pool whose unused places hold what must not count: codes that are no numbers, scales that are none."""

    def __init__(self, seed, rows, lens, heads, kv, dim, dtype, kind, group, page, extra_columns=1, poison=True, sharp=1.5, spread=0.5):
        g = self.g = torch.Generator().manual_seed(seed)
        self.rows, self.lens, self.page, self.kind, self.group = rows, lens, page, kind, group
        need = [-(-max(length, 0) // page) for length in lens]
        n_pages, most = sum(need) + 2, quant.MOST[kind]
        self.codes = []
        for _ in range(2):
            x = (torch.randn(n_pages, kv, page, dim, generator=g) * most / 4).clamp(-most, most)
            self.codes.append(x.round().to(torch.int8) if kind == "int8" else x.to(torch.float8_e4m3fn))
        self.scales = [4 / most * torch.exp(spread * torch.randn(n_pages, kv, page // group, generator=g)) for _ in range(2)]
        self.q = (sharp * torch.randn(sum(rows), heads, dim, generator=g)).to(DT[dtype])
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
            hide = ~used[:, None, :, None].expand_as(self.codes[0])
            for c, bad in zip(self.codes, (float("nan"), float("inf"))):
                c.view(torch.int8)[hide] = 0x7f
            nobody = ~used.view(n_pages, 1, page // group, group).any(-1).expand_as(self.scales[0])
            self.scales[0][nobody], self.scales[1][nobody] = float("nan"), float("inf")

    def run(self, first=None, cu=True, **kw):
        cu_rows = ints(np.r_[0, np.cumsum(self.rows)]) if cu else None
        return B.odb_paged_attention_quant(self.q.cuda(), *(t.cuda() for t in self.codes + self.scales), ints(self.tables), ints(self.lens),
                                           cu_rows=cu_rows, first_pos=None if first is None else ints(first), **kw)

    def values(self):
        return [quant.values(c, s) for c, s in zip(self.codes, self.scales)]

    def check(self, got, first=None, causal=False, window=0, sinks=0, scale=None, oracle=plain.attention):
        dim, dt = self.q.shape[2], self.q.dtype
        scale = dim ** -0.5 if scale is None else scale
        k, v = self.values()
        want, size, big = oracle(self.q.double(), k, v, self.tables, self.lens, self.rows, first, scale, causal, window, sinks)
        u, n = torch.finfo(dt).eps / 2, max(self.lens + [1])
        finite = lambda x: x[torch.isfinite(x)].abs().max().item() if torch.isfinite(x).any() else 0.0        # noqa: E731
        # a probability is off by its rounding to binary16, in the sum or, times V's scale, in the product, U16 and F; by the score's sum,
        # dim F of sum |q||k|, and 6 F more for its products with scales; and by exp2, 4 F; numerator and denominator both.  Below 2^-14 binary16
        # has steps of 2^-24: the largest probability is 2^8 or more and V's largest scale a quarter of its unit, so that a key is off by
        # 2^-25 * 4 / 2^8 of the largest |v|, and of the denominator's 2^-33.  bfloat16 queries are off by 2^-33 of their row's largest, per channel.
        # The sums over the keys add their number times F times the largest (made in 16s: a quarter of that).  Then the result is rounded.
        fine = 2.0 ** -33 * dim * finite(self.q.double()) * finite(k) * scale
        off = U16 + (dim + 6) * F * big[..., None] + fine + 10 * F + n * F / 4 + n * 2.0 ** -33
        bound = 2 * off * size * (1 + 4 * off) + n * 2.0 ** -31 * finite(v) + u * want.abs() * (1 + u) + torch.finfo(dt).tiny * torch.finfo(dt).eps
        got = got.cpu().double()
        assert got.shape == want.shape and torch.isfinite(got).all()
        err = (got - want).abs()
        assert (err <= bound).all(), ((err / bound).max().item(), torch.nonzero(err > bound)[:3].tolist())


KINDS = [("int8", 16), ("int8", 1), ("e4m3", 32), ("e4m3", 1)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("kind,group", KINDS)
@pytest.mark.parametrize("heads,kv,dim", [(1, 1, 64), (8, 2, 128), (6, 6, 64), (7, 1, 128), (4, 2, 256), (33, 1, 128), (70, 1, 256)])
def test_single_tokens(heads, kv, dim, kind, group, dtype):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 47, 64, 100, 129, 0, 257]
    rq = Requests(heads * dim, [1] * len(lens), lens, heads, kv, dim, dtype, kind, group, 32)
    for causal in (False, True):
        got = rq.run(causal=causal, cu=not causal)
        rq.check(got, causal=causal)
        assert (got[12] == 0).all()                       # no keys at all


@pytest.mark.parametrize("kind,group", KINDS)
@pytest.mark.parametrize("page", [32, 256, 4096])
@pytest.mark.parametrize("max_len", [0, 600, 5])
def test_long_keys_split_over_workgroups(page, max_len, kind, group):
    lens = [5000, 3, 1700, 0, 513]
    rq = Requests(page, [1] * 5, lens, 8, 2, 64, "bf16", kind, group, page, extra_columns=3)
    rq.check(rq.run(causal=True, cu=False, max_len=max_len), causal=True)


@pytest.mark.parametrize("n,kv", [(64, 1), (65, 1), (300, 2), (700, 4), (4096, 1)])
@pytest.mark.parametrize("max_len", [0, 64])
def test_many_requests(n, kv, max_len):
    rng = random.Random(n)
    lens = [rng.choice([0, 1, 17, 40, rng.randint(1, 60), 700 if rng.random() < 0.05 else 33]) for _ in range(n)]
    rows = [rng.choice([0, 1, 1, 1, min(3, max(1, length))]) for length in lens]
    rq = Requests(n + kv, rows, lens, 2 * kv, kv, 64, "f16", "e4m3", 16, 16)
    rq.check(rq.run(causal=True, max_len=max_len), causal=True)


MASKS = [(False, 0, 0), (True, 0, 0), (True, 1, 0), (True, 20, 3), (False, 20, 3), (True, 70, 40), (False, 300, 17), (True, 64, 2000)]


@pytest.mark.parametrize("dtype,dim", [("f16", 64), ("bf16", 128), ("f16", 256)])
@pytest.mark.parametrize("kind,group", KINDS)
@pytest.mark.parametrize("causal,window,sinks", MASKS)
def test_ragged_rows_masks_and_sinks(dtype, dim, kind, group, causal, window, sinks):
    rows, lens = [5, 1, 33, 0, 70, 16], [40, 17, 210, 30, 70, 601]
    rq = Requests(dim + window, rows, lens, 6, 2, dim, dtype, kind, group, 32)
    rq.check(rq.run(causal=causal, window=window, sinks=sinks), causal=causal, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,dim,kind,group", [("f16", 64, "int8", 1), ("bf16", 128, "e4m3", 32), ("f16", 128, "int8", 1), ("f16", 256, "e4m3", 16)])
@pytest.mark.parametrize("rows", [[2, 1, 5, 0, 3, 4], [9, 1, 10, 0, 4, 7], [5, 1, 21, 0, 20, 16], [5, 1, 33, 0, 70, 16]])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 1700, 3), (False, 1700, 40), (True, 2000, 700)])
def test_ragged_rows_whose_keys_are_split_over_workgroups(dtype, dim, kind, group, rows, causal, window, sinks):
    lens = [40, 17, 210, 30, 2300, 601]
    rq = Requests(dim + window + sum(rows), rows, lens, 6, 2, dim, dtype, kind, group, 32, extra_columns=300)
    rq.check(rq.run(causal=causal, window=window, sinks=sinks), causal=causal, window=window, sinks=sinks, oracle=plain.attention_many)


@pytest.mark.parametrize("dtype,dim,heads,kv,kind,group", [("f16", 64, 64, 64, "int8", 16), ("bf16", 128, 64, 64, "e4m3", 1), ("bf16", 128, 96, 32, "int8", 1),
                                                            ("f16", 256, 40, 40, "e4m3", 16), ("f16", 64, 120, 24, "e4m3", 1), ("bf16", 256, 40, 40, "int8", 1),
                                                            ("f16", 128, 64, 64, "int8", 16)])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 33, 5), (False, 100, 70), (True, 1, 0)])
def test_many_rows(dtype, dim, heads, kv, kind, group, causal, window, sinks):
    rows, lens = [260, 1, 0, 131, 64], [301, 1, 70, 131, 530]
    rq = Requests(dim + window + heads, rows, lens, heads, kv, dim, dtype, kind, group, 16)
    rq.check(rq.run(causal=causal, window=window, sinks=sinks), causal=causal, window=window, sinks=sinks, oracle=plain.attention_many)


@pytest.mark.parametrize("dtype,dim,heads,kv,kind,group", [("f16", 64, 16, 16, "e4m3", 16), ("bf16", 128, 32, 32, "int8", 64), ("bf16", 128, 32, 32, "e4m3", 1),
                                                            ("f16", 256, 16, 16, "int8", 32)])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 900, 5), (False, 300, 70)])
def test_many_rows_whose_keys_are_split_over_workgroups(dtype, dim, heads, kv, kind, group, causal, window, sinks):
    rows, lens = [150, 0, 1, 129], [3500, 20, 1, 9000]
    rq = Requests(dim + window + heads, rows, lens, heads, kv, dim, dtype, kind, group, 64)
    cu = ints([0, 150, 150, 151, 280])                                     # rows that belong to no request stay
    q = torch.cat([rq.q, rq.q[:20]]).cuda()
    out = torch.full_like(q, 3.0)
    B.odb_paged_attention_quant(q, *(t.cuda() for t in rq.codes + rq.scales), ints(rq.tables), ints(rq.lens), causal=causal, window=window, sinks=sinks,
                                cu_rows=cu, out=out)
    rq.check(out[:280], causal=causal, window=window, sinks=sinks, oracle=plain.attention_many)
    assert (out[280:] == 3.0).all()


@pytest.mark.parametrize("dtype,dim,kind,group", [("f16", 64, "int8", 16), ("bf16", 128, "e4m3", 1), ("f16", 256, "e4m3", 16)])
@pytest.mark.parametrize("window,sinks", [(1, 50), (3, 700), (40, 45), (64, 2000)])
def test_positions_that_stay_visible_beyond_the_window(dtype, dim, kind, group, window, sinks):
    """... which, where rows see what lies behind them, are not the first of what a row sees: single tokens, few rows, keys split over workgroups, many
    rows, pieces of them."""
    for heads, kv, rows, lens, first, columns in ((4, 2, [1, 1, 5], [300, 40, 1000], [2, 39, 100], 1), (6, 2, [5, 1, 33], [40, 17, 2300], [0, 3, 9], 300),
                                                  (40, 40, [220, 130, 3], [220, 1000, 60], [0, 200, 1], 1), (16, 16, [150, 129], [3500, 9000], [7, 400], 1)):
        rq = Requests(dim + window + sum(rows), rows, lens, heads, kv, dim, dtype, kind, group, 16, extra_columns=columns)
        rq.check(rq.run(first=first, causal=False, window=window, sinks=sinks), first=first, window=window, sinks=sinks, oracle=plain.attention_many)


@pytest.mark.parametrize("kind,group", KINDS)
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 9, 2), (False, 9, 2)])
def test_rows_at_given_positions(kind, group, causal, window, sinks):
    rows, lens, first = [32, 32, 8, 8, 8], [300, 64, 50, 50, 50], [100, 0, -4, 46, 2 ** 31 - 40]
    rq = Requests(3, rows, lens, 4, 4, 128, "f16", kind, group, 32)
    rq.check(rq.run(first=first, causal=causal, window=window, sinks=sinks), first=first, causal=causal, window=window, sinks=sinks)


@pytest.mark.parametrize("heads,kv,rows,lens", [(4, 2, [40], [100]), (64, 64, [200, 70], [300, 90])])
@pytest.mark.parametrize("group", [1, 16])
def test_codes_and_scales_that_some_rows_do_not_see(heads, kv, rows, lens, group):
    """Causal rows: a code that is no number and scales that are none, at a position that half of a tile's rows see: the others stay as they were."""
    rq = Requests(9, rows, lens, heads, kv, 64, "f16", "e4m3", group, 16)
    clean = rq.run(causal=True)
    rq.check(clean, causal=True)
    clean = clean.cpu()
    key = lens[0] - 16
    page_id, at, sees = int(rq.tables[0, key // 16]), key % 16, key - (lens[0] - rows[0])
    scaled = key // group * group - (lens[0] - rows[0])                     # a scale is seen by the rows that see any position of its group
    keep = rq.codes[1].clone()
    rq.codes[1].view(torch.int8)[page_id, :, at, :32] = 0x7f
    got = rq.run(causal=True).cpu()
    assert torch.equal(got[:sees], clean[:sees]) and torch.isnan(got[sees:rows[0], :, :32]).all() and torch.isfinite(got[sees:rows[0], :, 32:]).all()
    assert torch.equal(got[rows[0]:], clean[rows[0]:])
    rq.codes[1] = keep
    keep = rq.codes[0].clone()
    rq.codes[0].view(torch.int8)[page_id, :, at] = -1                        # 0xff
    got = rq.run(causal=True).cpu()
    assert torch.equal(got[:sees], clean[:sees]) and torch.isnan(got[sees:rows[0]]).all() and torch.equal(got[rows[0]:], clean[rows[0]:])
    rq.codes[0] = keep
    for s in rq.scales:
        was = s[page_id, :, at // group].clone()
        s[page_id, :, at // group] = float("nan")
        got = rq.run(causal=True).cpu()
        assert torch.equal(got[:scaled], clean[:scaled]) and torch.isnan(got[scaled:rows[0]]).all() and torch.equal(got[rows[0]:], clean[rows[0]:])
        s[page_id, :, at // group] = was


@pytest.mark.parametrize("kind,group", KINDS)
def test_pages_outside_the_pool_are_seen_by_nobody(kind, group):
    rq = Requests(11, [1, 3, 20], [200, 90, 333], 8, 2, 128, "bf16", kind, group, 32)
    rq.tables[0, 2], rq.tables[1, 0], rq.tables[2, 5], rq.tables[2, 10] = -1, rq.codes[0].shape[0], 2 ** 31 - 1, -2 ** 31
    for causal in (True, False):
        rq.check(rq.run(causal=causal), causal=causal)
    rq.tables[:] = -1
    assert (rq.run(causal=False) == 0).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("kind,group", KINDS)
def test_scales_far_apart_and_zero(kind, group, dtype):
    """V's scales rise over the keys by a factor of 2^40, fall again, and are zero; K's are zero for some keys."""
    rq = Requests(31, [1, 1, 1, 200], [900, 900, 900, 700], 4, 2, 64, dtype, kind, group, 32)
    for r in range(3):
        for j, page_id in enumerate(rq.tables[r, :29]):
            if r < 2:
                rq.scales[1][page_id] = 2.0 ** (40 * (j if r == 0 else 28 - j) / 28 - 30)
            else:
                rq.scales[1][page_id] = 0 if j % 3 else 1e-3
                rq.scales[0][page_id] = 0 if j % 2 else 0.02
    rq.scales[1][rq.tables[3, :22]] = 0
    got = rq.run(causal=True)
    rq.check(got, causal=True, oracle=plain.attention_many)
    assert (got[3:] == 0).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("kind,group", KINDS)
def test_scores_far_apart_rising_and_equal(kind, group, dtype):
    rq = Requests(17, [1, 1, 1], [900, 900, 900], 2, 1, 64, dtype, kind, group, 32)
    for j, page_id in enumerate(rq.tables[0, :29]):
        rq.codes[0][page_id] = torch.zeros(1, 32, 64).to(rq.codes[0].dtype)
        rq.codes[0][page_id, :, :, 0] = 8 if j > 14 else -8
        rq.scales[0][page_id] = abs(j - 14) / 3
    for page_id in rq.tables[1, :29]:
        rq.codes[0][page_id], rq.scales[0][page_id] = torch.full((1, 32, 64), 4).to(rq.codes[0].dtype), 1 / 16
    rq.q[0] = 0
    rq.q[0, :, 0] = torch.tensor([30.0, -30.0]).to(DT[dtype])
    rq.codes[0][rq.tables[2, 11], :, 3] = (20 * rq.q[2, 0].float()).round().clamp(-120, 120).to(rq.codes[0].dtype)
    rq.scales[0][rq.tables[2, 11]] = 1
    rq.check(rq.run(causal=False, scale=1.0), scale=1.0)


def test_queries_of_any_size():
    """bfloat16 queries far beyond binary16, tiny ones and rows of zeros."""
    rq = Requests(41, [6, 200], [300, 400], 4, 2, 128, "bf16", "int8", 16, 16, sharp=1.0)
    rq.q[0] = rq.q[0] * 2.0 ** 60
    rq.q[1] = rq.q[1] * 2.0 ** -90
    rq.q[2] = 0
    rq.q[3, :, 1:] = rq.q[3, :, 1:] * 2.0 ** -20
    low = rq.run(causal=True, scale=2.0 ** -64)                              # row 0's scores are of an ordinary size, the others' are nought
    rq.check(low, causal=True, scale=2.0 ** -64, oracle=plain.attention_many)
    rq.q[0] = 1
    rq.check(rq.run(causal=True), causal=True, oracle=plain.attention_many)


@pytest.mark.parametrize("score,ok", [(2.0 ** 20, True), (2.0 ** 26, True), (2.0 ** 28, False)])
@pytest.mark.parametrize("rows", [1, 200])
def test_scores_far_from_zero(score, ok, rows):
    """All keys equal: any size of score gives the mean of the values up to its limit, and no numbers beyond."""
    rq = Requests(43, [rows], [300], 2, 2, 64, "f16", "int8", 16, 16, poison=False)
    rq.q[:] = 1
    rq.codes[0][:] = 1
    rq.scales[0][:] = score / 64 / 1.4426950408889634
    got = rq.run(causal=False, scale=1.0)
    if not ok:
        assert torch.isnan(got).all()
        return
    k, v = rq.values()
    ids = torch.tensor(rq.tables[0, :19].astype(np.int64))
    mean = v[ids].permute(1, 0, 2, 3).reshape(2, -1, 64)[:, :300].mean(1)
    size = v[ids].permute(1, 0, 2, 3).reshape(2, -1, 64)[:, :300].abs().mean(1)
    # equal scores, equal probabilities: their roundings to binary16, one of them times the scale
    assert ((got.cpu().double() - mean).abs() <= 2.1 * U16 * size + U16 * mean.abs() + 300 * 2.0 ** -31 * size.max()).all()


def test_strided_rows_and_pools_and_a_given_workspace():
    rq = Requests(13, [2, 30, 1], [700, 65, 1200], 6, 3, 128, "bf16", "e4m3", 32, 32, poison=False)
    want = rq.run(causal=True)
    rq.check(want, causal=True)
    wide = torch.zeros(33, 10, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:8] = rq.q.cuda()
    codes = [x.view(torch.int8).permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3).view(torch.float8_e4m3fn) for x in rq.codes]
    scales = [x.permute(1, 0, 2).contiguous().cuda().permute(1, 0, 2) for x in rq.scales]
    out = torch.full((33, 9, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    work = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    args = (wide[:, 2:8], *codes, *scales, ints(rq.tables), ints(rq.lens))
    got = B.odb_paged_attention_quant(*args, causal=True, cu_rows=ints([0, 2, 32, 33]), out=out[:, 3:], workspace=work)
    assert torch.equal(got, want) and (out[:, :3] == 5.0).all()
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.OdbError, match="workspace"):
        B.odb_paged_attention_quant(*args, causal=True, cu_rows=ints([0, 2, 32, 33]), workspace=small)


def test_offsets_beyond_32_bits():
    """Pages more than 2^32 bytes from the pool's start (the pools overlap in one buffer of 17 GB)."""
    page, stride = 16, 1 << 32
    buf = torch.empty(4 * stride + (1 << 20), dtype=torch.int8, device="cuda")
    k = buf.as_strided((5, 1, page, 64), (stride, page * 64, 64, 1))
    v = buf[1 << 19:].as_strided((5, 1, page, 64), (stride, page * 64, 64, 1))
    rq = Requests(19, [1, 4], [30, 45], 2, 1, 64, "f16", "int8", 16, 16, poison=False)
    ids, at = [4, 2, 0, 3, 1], 0
    tables, scales = np.full_like(rq.tables, -1), [torch.zeros(5, 1, 1, device="cuda") for _ in range(2)]
    for r, need in enumerate((2, 3)):
        for j in range(need):
            was = rq.tables[r, j]
            k[ids[at]], v[ids[at]] = rq.codes[0][was].cuda(), rq.codes[1][was].cuda()
            for s, t in zip(scales, rq.scales):
                s[ids[at]] = t[was].cuda()
            tables[r, j] = ids[at]
            at += 1
    got = B.odb_paged_attention_quant(rq.q.cuda(), k, v, *scales, ints(tables), ints(rq.lens), causal=True, cu_rows=ints([0, 1, 5]))
    rq.check(got, causal=True)
    qkv = torch.randn(1, 3, 64, device="cuda").half()
    B.odb_qk_norm_rope_quant(qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], k, v, *scales, B.odb_rope_table(64, 64, 10000.0), ints([0]), ints([[4]]), ints([6]), first_pos=ints([5]))
    back = B.odb_paged_read_quant(k, v, *scales, ints([4 * 16 + 5]))
    for x, y, s in zip(back, (qkv[:, 1:2], qkv[:, 2:]), scales):
        assert ((x.float() - y.float()).abs() <= 0.501 * s[4, 0, 0] + 2.0 ** -11 * y.float().abs()).all()
