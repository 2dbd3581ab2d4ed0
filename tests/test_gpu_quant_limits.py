"""Attention over pages of 8-bit codes at the ends of what scales and queries can be, on every way that sizes lead to.  Tolerances are those of
test_gpu_quant_attention.py."""
import pytest

torch = pytest.importorskip("torch")

import paged_plain as plain                                          # noqa: E402
import quant_plain as quant                                          # noqa: E402
from test_gpu_quant_attention import F, KINDS, U16, Requests         # noqa: E402

pytestmark = pytest.mark.gpu

# heads, K/V heads, rows, lengths, further columns of the tables: single tokens, few rows, keys split over workgroups, many rows, pieces of them
WAYS = [(8, 2, [1, 1, 1], [100, 33, 700], 1), (6, 2, [5, 33], [90, 333], 1), (8, 2, [1, 1], [5000, 900], 3), (6, 2, [9, 40], [2300, 601], 300),
        (64, 64, [260, 131], [301, 131], 1), (16, 16, [150, 129], [3500, 9000], 1)]


@pytest.mark.parametrize("heads,kv,rows,lens,columns", WAYS)
@pytest.mark.parametrize("dtype,dim", [("f16", 64), ("bf16", 128), ("bf16", 256)])
@pytest.mark.parametrize("kind,group", KINDS)
def test_scales_of_v_below_the_smallest_normal_number(kind, group, dtype, dim, heads, kv, rows, lens, columns):
    """The first scales of V that a row sees are subnormal: whatever follows, and where nothing does, results are numbers.  (The unit of probabilities times
    scales is then 2^-124: a key's part of a row is off by 2^-157 of its code, below the last place of any result.)"""
    rq = Requests(dim + sum(rows) + group, rows, lens, heads, kv, dim, dtype, kind, group, 32, extra_columns=columns)
    v_scale = rq.scales[1]
    for r, first in enumerate((2.0 ** -140, 2.0 ** -149, 2.0 ** -130)[:len(rows)]):
        pages = rq.tables[r, :-(-lens[r] // 32)]
        v_scale[pages[0]] = first
        if len(pages) > 2:
            v_scale[pages[1]] = 1.5 * 2.0 ** -127
            v_scale[pages[2]] = 0.0
    first = [0] * len(rows) if rows[0] == 260 else None                     # (rows that see nothing else)
    rq.check(rq.run(causal=True, first=first), causal=True, first=first, oracle=plain.attention_many)
    for r in range(len(rows)):
        v_scale[rq.tables[r, :-(-lens[r] // 32)]] = 2.0 ** -130
    rq.check(rq.run(causal=False), causal=False, oracle=plain.attention_many)


@pytest.mark.parametrize("heads,kv,rows,lens,columns", WAYS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind,group", KINDS)
def test_small_channels_of_bfloat16_queries(kind, group, dim, heads, kv, rows, lens, columns):
    """bfloat16 queries are kept within 2^-33 of their row's largest: multiples of 2^-32 beside a channel of 1.5, which alone meet codes that are not zero, are
    whole multiples of binary16's smallest number then, and come through exactly."""
    rq = Requests(dim + sum(rows) + group, rows, lens, heads, kv, dim, "bf16", kind, group, 32, extra_columns=columns)
    odd = torch.randint(-4, 4, rq.q.shape, generator=rq.g) * 2 + 1
    rq.q = (odd * 2.0 ** -32).bfloat16()
    rq.q[..., 0] = 1.5
    rq.codes[0].view(torch.int8)[..., 0] = 0
    rq.scales[0] = torch.where(rq.scales[0].isnan(), rq.scales[0], 2.0 ** 26 / quant.MOST[kind])
    scale = 2.0 ** 4 * dim ** -0.5
    got, (k, v), u = rq.run(causal=True, scale=scale).cpu().double(), rq.values(), 2.0 ** -8
    want, size, big = plain.attention_many(rq.q.double(), k, v, rq.tables, lens, rows, None, scale, True, 0, 0)
    assert 0.5 < big.max() < 2.0 ** 6                                       # (scores that tell whether the channels were there)
    n = max(lens)
    # as Requests.check, whose part for what queries lose is nought here
    off = U16 + (dim + 6) * F * big[..., None] + 10 * F + n * F / 4 + n * 2.0 ** -33
    bound = 2 * off * size * (1 + 4 * off) + n * 2.0 ** -31 * v[v.isfinite()].abs().max() + u * want.abs() * (1 + u) + torch.finfo(torch.bfloat16).tiny
    assert ((got - want).abs() <= bound).all(), ((got - want).abs() / bound).max().item()
