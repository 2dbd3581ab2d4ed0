"""Paged K/V in 8 bits as its calls are used: together, captured, on two streams, over the same buffers again."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import quant_plain as quant                                          # noqa: E402
from paper_2511_21759_amd import binding as B                        # noqa: E402

pytestmark = pytest.mark.gpu
F = 2.0 ** -24


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Serving:
    """Requests that grow, are cut and start anew over one pool; tables, rotation and codes, attention in every step."""

    def __init__(self, n, kind, group, page=16, heads=8, kv=2, dim=128, n_pages=64, columns=20, dtype=torch.bfloat16, seed=23):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.n, self.page, self.heads, self.kv, self.n_pages, self.dtype = n, page, heads, kv, n_pages, dtype
        self.table = B.odb_rope_table(page * columns, dim, 10000.0)
        codes = [torch.randint(-128, 127, (n_pages, kv, page, dim), generator=self.g, device="cuda").to(torch.int8).view(quant.CODES[kind]) for _ in range(2)]
        self.pools = codes + [torch.full((n_pages, kv, page // group), float("nan"), device="cuda") for _ in range(2)]
        self.tables, self.free, self.n_free = ints(np.full((n, columns), -1)), ints(np.arange(n_pages)[::-1].copy()), ints([n_pages])
        self.held = ints([0] * n)

    def rows(self, count):
        return torch.randn(count, self.heads + 2 * self.kv, 128, generator=self.g, device="cuda").to(self.dtype)

    def step(self, wanted, qkv, causal=True, **kw):
        h, kv = self.heads, self.kv
        length, cu, slots, positions, state = B.odb_page_tables(self.held, wanted, self.tables, self.free, self.n_free, self.page, self.n_pages, rows_cap=qkv.shape[0])
        q = B.odb_qk_norm_rope_quant(qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:], *self.pools, self.table, positions, self.tables, length, cu_rows=cu)
        out = B.odb_paged_attention_quant(q, *self.pools, self.tables, length, causal=causal, cu_rows=cu, **kw)
        self.held, self.n_free = length, state[:1].clone()
        return q, out, cu


@pytest.mark.parametrize("kind,group", [("int8", 16), ("e4m3", 16), ("int8", 1), ("e4m3", 1)])
def test_steps_of_growing_and_cut_requests(kind, group):
    """Pages go from request to request, so codes and scales of others lie in them first.  A value is off by half a code of its group's scale for
    every time that it was rounded: once when stored, and again when its group's scale grew (at most 15 times in 16 positions); here the
    largest value of a group is below 8 times its standard deviation, and the answer is compared with values of 64 bits."""
    s = Serving(3, kind, group)
    plan = [[40, 3, 100], [41, 4, 101], [42, 5, 80], [43, 60, 81], [20, 61, 82], [21, 62, 83], [0, 63, 84], [90, 64, 85]]
    held, history = [0, 0, 0], [[torch.zeros(0, 2, 128, dtype=torch.float64)] * 2 for _ in range(3)]
    for want in plan:
        rows = [max(0, w - h) for w, h in zip(want, held)]
        qkv = s.rows(max(1, sum(rows)))
        q, out, cu = s.step(ints(want), qkv)
        assert cu.tolist() == np.r_[0, np.cumsum(rows)].tolist() and s.held.tolist() == want
        at = 0
        for r in range(3):
            # the same rows in 64 bits: keys as q's rotation has them, by the other operator, over pages of its own
            new = qkv[at:at + rows[r]]
            if rows[r]:
                k16, v16 = (torch.zeros(rows[r] // 16 + 1, 2, 16, 128, dtype=s.dtype, device="cuda") for _ in range(2))
                pos = torch.arange(held[r], held[r] + rows[r], dtype=torch.int32, device="cuda")
                B.odb_qk_norm_rope(new[:, :8], new[:, 8:10], new[:, 10:], k16, v16, s.table, pos, torch.arange(rows[r], dtype=torch.int32, device="cuda"))
                turned = k16.transpose(1, 2).flatten(0, 1)[:rows[r]].double().cpu()
                history[r] = [torch.cat([history[r][0][:held[r]], turned]), torch.cat([history[r][1][:held[r]], new[:, 10:].double().cpu()])]
            history[r] = [x[:want[r]] for x in history[r]]
            if want[r]:
                slots = s.tables[r, torch.arange(want[r], device="cuda") // 16] * 16 + torch.arange(want[r], device="cuda").int() % 16
                held_values = [x.double().cpu() for x in B.odb_paged_read_quant(*s.pools, slots, dtype=torch.float32)]
                for x, y in zip(held_values, history[r]):
                    top = y.abs().amax()
                    # (E4M3: half a step is 2^-4 of a value, and of the group's 448th part below 2^-6 of a code; keys come rounded to bfloat16 here)
                    once = top / 254 if kind == "int8" else y.abs() / 16 + top / 448 * 2.0 ** -10
                    times = 1 if group == 1 else 3
                    assert ((x - y).abs() <= times * 1.1 * once + 2.0 ** -8 * y.abs()).all()
                # attention over the values that the pages hold
                q64 = q[at:at + rows[r]].double().cpu()
                for i in range(rows[r]):
                    m = held[r] + i + 1
                    for h in range(8):
                        k, v = held_values[0][:m, h // 4], held_values[1][:m, h // 4]
                        w = torch.softmax(k @ q64[i, h] * 128 ** -0.5, 0)
                        off = 2.0 ** -11 + 150 * F * (q64[i, h].abs() @ k.abs().t()).max() * 128 ** -0.5 + 1e-6
                        bound = 2.1 * off * (w @ v.abs()) + 1.01 * 2.0 ** -8 * (w @ v).abs() + 1e-6
                        assert ((out[at + i, h].double().cpu() - w @ v).abs() <= bound).all()
            at += rows[r]
        held = list(want)


@pytest.mark.parametrize("kind,group", [("int8", 16), ("e4m3", 1)])
def test_captured_steps_equal_eager_ones_and_two_graphs_do_not_meet(kind, group):
    """A captured step of single tokens is replayed with new lengths and rows; another graph of the same pool of memory runs in between."""
    heads, kv, dim, page, n_pages, n = 8, 2, 128, 16, 400, 4
    g = torch.Generator(device="cuda").manual_seed(3)
    table = B.odb_rope_table(2048, dim, 10000.0)
    tables = torch.randperm(n_pages, generator=g, device="cuda").int()[:n * 90].view(n, 90).contiguous()

    def make():
        # (numbers all: bytes of any kind would hold 0xff, which is none in E4M3)
        codes = [(30 * torch.randn(n_pages, kv, page, dim, generator=g, device="cuda")).clamp(-120, 120).to(quant.CODES[kind]) for _ in range(2)]
        pools = codes + [torch.rand(n_pages, kv, page // group, generator=g, device="cuda") * 0.02 for _ in range(2)]
        return dict(pools=pools, qkv=torch.randn(n, heads + 2 * kv, dim, generator=g, device="cuda").half(), held=ints([7, 100, 900, 1300]), tables=tables.clone(),
                    free=ints(np.arange(n_pages)), n_free=ints([40]), slots=ints([-1] * n), positions=ints([0] * n), odd=ints([0]))

    def step(s):
        wanted = s["held"] + 1
        length, cu, slots, positions, state = B.odb_page_tables(s["held"], wanted, s["tables"], s["free"], s["n_free"], page, n_pages, slots=s["slots"],
                                                                positions=s["positions"])
        qkv = s["qkv"]
        q = B.odb_qk_norm_rope_quant(qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:], *s["pools"], table, positions, s["tables"], length,
                                     cu_rows=cu, odd=s["odd"])
        out = B.odb_paged_attention_quant(q, *s["pools"], s["tables"], length, causal=True, cu_rows=cu)
        return out, length, slots, state, *B.odb_paged_read_quant(*s["pools"], slots)

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
            assert s["odd"].item() == 0


def long_call(seed, rows, lens, heads=8, kv=2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-x // 64) for x in lens]
    codes = [torch.randint(-127, 128, (sum(need), kv, 64, 128), generator=g, device="cuda").to(torch.int8) for _ in range(2)]
    scales = [torch.rand(sum(need), kv, 4, generator=g, device="cuda") * 0.02 for _ in range(2)]
    tables, at = np.full((len(lens), max(need)), -1, np.int32), 0
    for r, c in enumerate(need):
        tables[r, :c], at = np.arange(at, at + c), at + c
    q = torch.randn(sum(rows), heads, 128, generator=g, device="cuda").half()
    return dict(q=q, k_pages=codes[0], v_pages=codes[1], k_scale=scales[0], v_scale=scales[1], tables=ints(tables), kv_len=ints(lens), causal=True,
                cu_rows=ints(np.r_[0, np.cumsum(rows)]), max_rows=max(rows))


@pytest.mark.parametrize("rows,lens", [([1, 1], [4000, 3000]), ([300, 200], [9000, 700])])
def test_two_streams_at_once(rows, lens):
    """Calls with keys split over workgroups overlap on two streams: each has a workspace of its own."""
    sets = [long_call(29 + i, rows, lens, *((8, 2) if rows[0] == 1 else (16, 16))) for i in range(2)]
    alone = [B.odb_paged_attention_quant(**a) for a in sets]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                outs[i].append(B.odb_paged_attention_quant(**sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for x in outs[i]:
            assert torch.equal(x, alone[i])


@pytest.mark.parametrize("rows", [[1, 1, 1], [40, 3, 17], [600, 100, 300]])
def test_both_ways_of_the_binding_are_the_same(rows, monkeypatch):
    """The packed path and the one in Python, which takes what the other does not."""
    a = long_call(7, rows, [900, 333, 5000], 32, 8)
    g = torch.Generator(device="cuda").manual_seed(1)
    table, qkv = B.odb_rope_table(6000, 128, 10000.0), torch.randn(sum(rows), 48, 128, generator=g, device="cuda")
    positions = torch.cat([torch.arange(n - m, n, dtype=torch.int32) for m, n in zip(rows, [900, 333, 5000])]).cuda()

    def all_three():
        pools = [a[x].clone() for x in ("k_pages", "v_pages", "k_scale", "v_scale")]
        gains = [torch.ones(128, device="cuda"), torch.full((128,), 0.5, device="cuda")]
        q = B.odb_qk_norm_rope_quant(qkv[:, :32], qkv[:, 32:40], qkv[:, 40:], *pools, table, positions, a["tables"], a["kv_len"], cu_rows=a["cu_rows"],
                                     q_gain=gains[0], k_gain=gains[1], eps=1e-5, interleaved=True, dtype=torch.bfloat16, odd=ints([0]))
        out = torch.empty_like(q)
        same = B.odb_paged_attention_quant(q, *pools, a["tables"], a["kv_len"], causal=True, cu_rows=a["cu_rows"], out=out, window=700, sinks=3, scale=0.1,
                                           max_rows=max(rows), max_len=5000, workspace=torch.empty(256 << 20, dtype=torch.uint8, device="cuda"))
        assert same is out
        return q, out, *pools, *B.odb_paged_read_quant(*pools, ints([5, -1, 700, 64 * 98]), dtype=torch.float32)

    fast = all_three()
    monkeypatch.setattr(B, "_here", lambda index: None)
    for x, y in zip(fast, all_three()):
        assert torch.equal(x, y)
    monkeypatch.undo()
    bad_room = [dict(workspace=torch.empty(0, dtype=torch.uint8, device="cuda"), tables=a["tables"].repeat(1, 40))] if max(rows) == 1 else []      # (whole tiles need none)
    for bad in (dict(window=-1), dict(scale=0.0), dict(max_len=-2), *bad_room):
        with pytest.raises(B.OdbError, match="paged_attention_quant"):
            B.odb_paged_attention_quant(**dict(a, **bad))
    for bad in (dict(kv_len=a["kv_len"].long()), dict(tables=a["tables"].cpu()), dict(q=a["q"].float()), dict(k_scale=a["k_scale"][:, :1]), dict(out=torch.empty(3))):
        with pytest.raises(TypeError):
            B.odb_paged_attention_quant(**dict(a, **bad))


def test_rows_of_a_cut_last_round_and_longest_first():
    """Many whole tiles in a round that is not full: some are cut and joined; requests lie in any order of their lengths."""
    for rows, lens in (([700, 2400, 1100], [900, 2500, 1500]), ([1300, 900, 2100], [3000, 901, 2200])):
        a = long_call(11, rows, lens, 32, 8)
        got = B.odb_paged_attention_quant(**a)
        first = 0
        for r, m in enumerate(rows):                       # each request alone is another way of computing
            alone = dict(a, q=a["q"][first:first + m].contiguous(), tables=a["tables"][r:r + 1].contiguous(), kv_len=a["kv_len"][r:r + 1], cu_rows=ints([0, m]), max_rows=m)
            want = B.odb_paged_attention_quant(**alone)
            # two roundings of probabilities and of the result each (values up to 127 * 0.02)
            assert ((got[first:first + m].double() - want.double()).abs() <= 6 * 2.0 ** -11 * 1.3 + 2.0 ** -10 * want.double().abs()).all()
            first += m
