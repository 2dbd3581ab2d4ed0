"""Paged K/V in 8 bits against plain implementations in 64 bits (tests/quant_plain.py, tests/paged_plain.py), element by element.

Tolerances count roundings.  u is half a step of the result's type (2^-11 binary16, 2^-8 bfloat16), f = 2^-24 that of 32 bits.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paged_plain as plain                                          # noqa: E402
import quant_plain as quant                                          # noqa: E402
from paper_2511_21759_amd import binding as B                        # noqa: E402

pytestmark = pytest.mark.gpu
F = 2.0 ** -24
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def half_step(dt):
    return torch.finfo(dt).eps / 2


def ints(x, device="cuda"):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=device)


def pools(g, kind, n_pages, kv, page, dim, group, size=4.0):
    """Codes of a normal distribution and scales that differ: (k, v, k_scale, v_scale)."""
    most, out = quant.MOST[kind], []
    for _ in range(2):
        x = (torch.randn(n_pages, kv, page, dim, generator=g) * most / size).clamp(-most, most)
        out.append(x.round().to(torch.int8) if kind == "int8" else x.to(torch.float8_e4m3fn))
    return out + [size / most * torch.exp(0.5 * torch.randn(n_pages, kv, page // group, generator=g)) for _ in range(2)]


def some_tables(g, lens, page, extra=1):
    need = [-(-max(length, 0) // page) for length in lens]
    n_pages = sum(need) + 2
    ids, at = torch.randperm(n_pages, generator=g).tolist(), 0
    tables = np.full((len(lens), max(need + [1]) + extra), -1, np.int32)
    for r, count in enumerate(need):
        tables[r, :count] = ids[at:at + count]
        at += count
    return tables, n_pages


# ---- rows to codes ----------------------------------------------------------------------------------------------------

class Rows:
    """Rows of requests, with norms and rotation or with angles of nought."""

    def __init__(self, seed, kind, rows, lens, first, heads, kv, dim, rot, given, dtype, inter, norms, group, page, turning=True):
        g = self.g = torch.Generator().manual_seed(seed)
        self.kind, self.rows, self.lens, self.first, self.group, self.page = kind, rows, lens, first, group, page
        self.heads, self.kv, self.dim, self.rot, self.inter, self.dtype = heads, kv, dim, rot, inter, DT[dtype]
        self.tables, n_pages = some_tables(g, lens, page)
        self.before = pools(g, kind, n_pages, kv, page, dim, group)
        self.qkv = torch.randn(sum(rows), heads + 2 * kv, dim, generator=g).to(DT[given])
        self.n_pos = 6000
        self.table = torch.from_numpy(plain.rope_table(self.n_pos, rot, 10000.0).astype(np.float32))
        if not turning:
            self.table[..., 0], self.table[..., 1] = 1, 0
        starts = [length - m if first is None else first[r] for r, (m, length) in enumerate(zip(rows, lens))]
        self.positions = torch.tensor([s + i for s, m in zip(starts, rows) for i in range(m)], dtype=torch.int32).clamp(0, self.n_pos - 1)
        self.gains = [1 + 0.3 * torch.randn(dim, generator=g) for _ in range(2)] if norms else [None, None]

    def run(self, dev=None, before=None, cu=True, **kw):
        """-> (queries, after) on the CPU."""
        dev = self.qkv.cuda() if dev is None else dev
        after = [t.cuda() for t in (self.before if before is None else before)]
        gains = [None if t is None else t.cuda() for t in self.gains]
        h, kv = self.heads, self.kv
        out = B.odb_qk_norm_rope_quant(dev[:, :h], dev[:, h:h + kv], dev[:, h + kv:], *after, self.table.cuda(), self.positions.cuda(), ints(self.tables),
                                       ints(self.lens), cu_rows=ints(np.r_[0, np.cumsum(self.rows)]) if cu else None,
                                       first_pos=None if self.first is None else ints(self.first), q_gain=gains[0], k_gain=gains[1], eps=1e-5,
                                       interleaved=self.inter, dtype=self.dtype, **kw)
        return out.cpu(), [t.cpu() for t in after]

    def check(self, out, after, before=None):
        before, h, kv = self.before if before is None else before, self.heads, self.kv
        live = (self.positions >= 0) & (self.positions < self.n_pos)
        angles = self.table.double()[self.positions.long().clamp(0, self.n_pos - 1)]
        gains = [None if t is None else t.double() for t in self.gains]
        # as for 16-bit pages: mean of squares, root, division, two products, two products and a sum - fewer than 24 roundings
        q, size = plain.rotate(self.qkv[:, :h].double(), gains[0], 1e-5, angles, self.rot, self.inter)
        q[~live], size[~live] = 0, 0
        u, tiny = half_step(self.dtype), torch.finfo(self.dtype).tiny * half_step(self.dtype)
        assert ((out.double() - q).abs() <= u * q.abs() + (1 + u) * 24 * F * size + tiny).all()
        k, size = plain.rotate(self.qkv[:, h:h + kv].double(), gains[1], 1e-5, angles, self.rot, self.inter)
        v = self.qkv[:, h + kv:].double()
        args = (self.rows, self.first, self.lens, self.tables, live)
        quant.check_store(self.kind, self.group, (before[0], before[2]), (after[0], after[2]), k, 24 * F * size, *args, "k")
        quant.check_store(self.kind, self.group, (before[1], before[3]), (after[1], after[3]), v, torch.zeros_like(v), *args, "v")


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("rows,lens,first,heads,kv,dim,rot,given,dtype,inter,norms,group,page", [
    ([1], [1], None, 1, 1, 64, 64, "f16", "f16", False, True, 16, 16),
    ([1, 1, 1], [17, 32, 40], None, 32, 8, 128, 128, "bf16", "bf16", False, True, 16, 16),
    ([1, 1, 1, 1], [1, 2, 700, 33], None, 5, 5, 128, 16, "bf16", "bf16", True, False, 1, 32),
    ([17, 0, 5], [50, 9, 5], None, 7, 1, 256, 256, "f32", "bf16", False, True, 64, 64),
    ([33, 32], [200, 70], [5, 38], 4, 2, 64, 32, "f32", "f16", True, True, 64, 4096),
    ([32, 32, 7], [300, 64, 90], [100, 0, 83], 12, 3, 128, 64, "f16", "f16", False, True, 32, 32),
    ([100, 1, 64], [101, 1, 164], None, 12, 3, 256, 48, "f16", "f16", True, True, 16, 16),
    ([300, 129], [400, 130], [77, 1], 3, 1, 128, 112, "bf16", "bf16", False, True, 64, 128),
    ([65, 200], [65, 200], [0, 0], 3, 1, 64, 48, "bf16", "bf16", False, True, 1, 16),
    ([40, 3], [45, 300], [5, 200], 2, 2, 256, 256, "bf16", "bf16", False, True, 32, 32),
])
def test_norm_rotation_and_codes(kind, rows, lens, first, heads, kv, dim, rot, given, dtype, inter, norms, group, page):
    c = Rows(sum(rows) + dim, kind, rows, lens, first, heads, kv, dim, rot, given, dtype, inter, norms, group, page)
    out, after = c.run()
    c.check(out, after)
    # the same call again writes the same
    again, twice = c.run(before=after)
    assert torch.equal(out, again) and all(torch.equal(a.view(torch.int8), b.view(torch.int8)) for a, b in zip(after, twice))


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dim,group", [(64, 16), (128, 1), (128, 64), (256, 64)])
def test_padding_rows_rows_beyond_lengths_and_pages_that_are_not_there(kind, dim, group):
    rows, lens, first = [70, 40, 30, 20], [100, 60, 300, 10], [40, 30, -9, 4]       # rows before the start and behind the length
    c = Rows(3 + dim, kind, rows, lens, first, 4, 2, dim, 32, "f16", "f16", False, True, group, 64)
    c.positions[3], c.positions[71], c.positions[90] = -1, c.n_pos, -2 ** 31
    c.tables[1, 0] = c.before[0].shape[0]
    out, after = c.run()
    c.check(out, after)
    assert (out[[3, 71, 90]] == 0).all()
    c.tables[:] = -1
    _, after = c.run()
    assert all(torch.equal(a.view(torch.int8), b.view(torch.int8)) for a, b in zip(after, c.before))


def test_rows_of_no_request_become_zero_queries_and_store_nothing():
    c = Rows(8, "int8", [5, 4], [20, 30], None, 4, 2, 64, 64, "f16", "f16", False, False, 16, 16)
    extra = torch.randn(3, 8, 64).half()
    c2 = Rows(8, "int8", [5, 4], [20, 30], None, 4, 2, 64, 64, "f16", "f16", False, False, 16, 16)
    c2.qkv, c2.positions = torch.cat([c.qkv, extra]), torch.cat([c.positions, torch.tensor([1, 2, 3], dtype=torch.int32)])
    (out, after), (out2, after2) = c.run(), c2.run()
    assert torch.equal(out, out2[:9]) and (out2[9:] == 0).all()
    assert all(torch.equal(a, b) for a, b in zip(after, after2))


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_one_row_per_request_without_cu_rows(kind):
    lens = [1, 16, 17, 100, 33, 48] * 15                                          # more than 64 requests
    a = Rows(5, kind, [1] * 90, lens, None, 4, 2, 128, 128, "bf16", "bf16", False, True, 16, 32)
    (out, after), (out2, after2) = a.run(cu=False), a.run()
    a.check(out, after)
    assert torch.equal(out, out2) and all(torch.equal(x.view(torch.int8), y.view(torch.int8)) for x, y in zip(after, after2))


@pytest.mark.parametrize("n", [65, 700, 4096])
def test_many_requests_of_few_rows(n):
    rng = np.random.default_rng(n)
    rows = rng.choice([0, 1, 1, 1, 2, 20], n).tolist()
    lens = [int(m + rng.integers(0, 30)) for m in rows]
    c = Rows(n, "e4m3", rows, lens, None, 1, 1, 64, 32, "f16", "f16", False, False, 16, 16)
    c.check(*c.run())


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_values_between_two_codes_go_to_the_even_one(kind):
    """Angles of nought: quotients that lie exactly between two codes, which a rounded scale must not move."""
    c = Rows(2, kind, [48], [48], None, 1, 1, 128, 16, "f32", "f16", False, False, 16, 16, turning=False)
    most = quant.MOST[kind]
    q = (torch.arange(128) - 64) * 0.5 if kind == "int8" else torch.tensor([17.0, 19.0, 2.125, -1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, 34.0] * 16)
    for i, a in enumerate([3.0, 0.7001953125, 1e-3]):
        c.qkv[16 * i:16 * i + 16] = (q.double() * float(np.float32(a)) / most).float()
        c.qkv[16 * i:16 * i + 16, :, 0] = float(np.float32(a))
    out, after = c.run()
    c.check(out, after)
    want = q.round() if kind == "int8" else q.to(torch.float8_e4m3fn).float()
    # (1 / 127 and 1 / 448 are rounded where the values are made, by half a step of 32 bits: only a = 3 * 448 / 448 ... is exact)
    exact = Rows(2, kind, [16], [16], None, 1, 1, 128, 16, "f32", "f16", False, False, 16, 16, turning=False)
    exact.qkv[:] = q * 0.75                                                      # the largest: 0.75 * most, so every quotient is q
    exact.qkv[:, :, 0] = 0.75 * most
    _, after = exact.run()
    pg = int(exact.tables[0, 0])
    for pool, scale in ((after[0], after[2]), (after[1], after[3])):
        assert (quant.numbers(pool)[pg, 0, :, 1:] == want[1:].double()).all() and scale[pg, 0, 0] == 0.75


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("group", [1, 16])
def test_values_that_are_not_finite_are_reported(kind, group):
    c = Rows(6, kind, [20, 3], [20, 40], None, 2, 2, 64, 64, "f32", "bf16", False, False, group, 16, turning=False)
    odd = ints([0])
    _, clean = c.run(odd=odd)
    assert odd.item() == 0
    c.qkv[4, 4, 3], c.qkv[4, 4, 5], c.qkv[5, 5, 9] = float("inf"), float("-inf"), float("nan")     # values of head 0, of head 1
    _, after = c.run(odd=odd)
    assert odd.item() == 1
    pg = int(c.tables[0, 0])
    n, most = quant.numbers(after[1]), quant.MOST[kind]
    assert n[pg, 0, 4, 3] == most and n[pg, 0, 4, 5] == -most and n[pg, 1, 5, 9] == 0
    want = c.qkv[:, 4:].double()
    want[5, 1, 9] = 0
    args = (c.rows, c.first, c.lens, c.tables, torch.ones(23, dtype=torch.bool))
    quant.check_store(kind, group, (c.before[1], c.before[3]), (after[1], after[3]), want, torch.zeros_like(want), *args, "v")
    assert torch.equal(clean[0].view(torch.int8), after[0].view(torch.int8)) and torch.equal(clean[2], after[2])
    c.run()                                                                       # nowhere to report to


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_very_small_and_very_large_values(kind):
    c = Rows(7, kind, [64], [64], None, 1, 1, 128, 16, "f32", "bf16", False, False, 16, 16, turning=False)
    for i, size in enumerate([2.0 ** -101, 2.0 ** -98, 2.0 ** 120, 0.0]):
        c.qkv[16 * i:16 * i + 16] = c.qkv[16 * i:16 * i + 16].clamp(-1, 1) * size
    out, after = c.run()
    live = torch.ones(64, dtype=torch.bool)
    v = c.qkv[:, 2:].double()
    quant.check_store(kind, 16, (c.before[1], c.before[3]), (after[1], after[3]), v, torch.zeros_like(v), c.rows, c.first, c.lens, c.tables, live, "v")
    assert after[3][int(c.tables[0, 0])].item() == 0 and after[3][int(c.tables[0, 3])].item() == 0


def test_codes_in_place_and_through_strided_pools():
    """out = q inside a fused buffer; pools stored [page, position, head, channel], scales [head, page, group]."""
    c = Rows(4, "int8", [40], [40], None, 8, 4, 128, 128, "bf16", "bf16", False, False, 16, 16)
    want, after = c.run()
    dev = c.qkv.cuda()
    codes = [t.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3) for t in c.before[:2]]
    scales = [t.permute(1, 0, 2).contiguous().cuda().permute(1, 0, 2) for t in c.before[2:]]
    got = B.odb_qk_norm_rope_quant(dev[:, :8], dev[:, 8:12], dev[:, 12:], *codes, *scales, c.table.cuda(), c.positions.cuda(), ints(c.tables),
                                   ints(c.lens), cu_rows=ints([0, 40]), out=dev[:, :8])
    assert got.data_ptr() == dev.data_ptr() and torch.equal(got.cpu(), want)
    for a, b in zip(codes + scales, after):
        assert torch.equal(a.cpu(), b)
    assert torch.equal(dev[:, 8:].cpu(), c.qkv[:, 8:])
    back = B.odb_paged_read_quant(*codes, *scales, ints(range(32)))
    for x, y in zip(back, B.odb_paged_read_quant(*(t.cuda() for t in after), ints(range(32)))):
        assert torch.equal(x, y)


# ---- values read back -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,kv,dim,page,group", [(1, 1, 64, 16, 16), (3, 8, 128, 32, 1), (70, 3, 256, 64, 32), (1000, 2, 128, 64, 64), (257, 5, 64, 16, 1)])
def test_read_back(kind, dtype, rows, kv, dim, page, group):
    g = torch.Generator().manual_seed(rows)
    n_pages = -(-rows // page) + 2
    p = pools(g, kind, n_pages, kv, page, dim, group)
    p[2][0], p[3][0] = 1e-6, 3e4                                                 # beyond what binary16 holds, on both sides
    slots = torch.randint(0, n_pages * page, (rows,), generator=g).int()
    if rows > 3:
        slots[1], slots[2], slots[3] = -1, n_pages * page, -2 ** 31
    got = B.odb_paged_read_quant(*(t.cuda() for t in p), slots.cuda(), dtype=DT[dtype])
    there = (slots >= 0) & (slots < n_pages * page)
    at = slots.long().clamp(0, n_pages * page - 1)
    for x, pool, scale in ((got[0], p[0], p[2]), (got[1], p[1], p[3])):
        want = (pool.float() * scale.repeat_interleave(group, 2)[..., None])[at // page, :, at % page].to(DT[dtype])     # one product of 32 bits, rounded once
        want[~there] = 0
        assert x.dtype == DT[dtype] and torch.equal(x.cpu(), want)


def test_read_back_into_parts_of_a_buffer():
    g = torch.Generator().manual_seed(1)
    p = [t.cuda() for t in pools(g, "int8", 5, 2, 16, 128, 16)]
    slots = ints([3, 70, 17, 18, 200, 40])
    want = B.odb_paged_read_quant(*p, slots)
    buf = torch.full((6, 5, 128), 9.0, dtype=torch.float16, device="cuda")
    k, v = B.odb_paged_read_quant(*p, slots, out=(buf[:, 1:3], buf[:, 3:]))
    assert torch.equal(k, want[0]) and torch.equal(v, want[1]) and (buf[:, 0] == 9).all() and k.data_ptr() == buf[:, 1:].data_ptr()
    with pytest.raises(B.OdbError, match="overlap"):
        B.odb_paged_read_quant(*p, slots, out=(buf[:, 1:3], buf[:, 2:4]))
