"""Plain forms of the paged K/V operators in 8 bits for the tests: in 64 bits, on the CPU, one group of positions after the other."""
import torch

MOST = {"int8": 127.0, "e4m3": 448.0}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
F = 2.0 ** -24


def numbers(pool):
    """The numbers that codes are, 64 bits."""
    return pool.float().double()


def values(pool, scale):
    """[n_pages, heads, page, dim] of 64 bits."""
    return numbers(pool) * scale.double().repeat_interleave(pool.shape[2] // scale.shape[2], 2)[..., None]


def step_at(q, kind):
    """The distance of codes around numbers q."""
    if kind == "int8":
        return torch.ones_like(q)
    _, e = torch.frexp(q.abs().clamp(min=1e-30))
    return torch.pow(2.0, (e - 1).clamp(min=-6).double() - 3)


def check_store(kind, group, before, after, x, delta, rows, first, lens, tables, live, what):
    """before, after: (codes, scales) of a pool, K or V; x [rows, heads, dim] the new values, known to within delta; live [rows]: not padding.
    Checks scales and codes of every group that a row falls into against the definition, and that nothing else has changed."""
    (codes0, scale0), (codes1, scale1) = before, after
    n_pages, heads, page, dim = codes0.shape
    most, n0, n1 = MOST[kind], numbers(codes0), numbers(codes1)
    raw0, raw1 = codes0.view(torch.int8).clone(), codes1.view(torch.int8).clone()
    same_scale = torch.ones_like(scale0, dtype=torch.bool)
    row = 0
    for r, m in enumerate(rows):
        length = min(max(lens[r], 0), tables.shape[1] * page)
        f = length - m if first is None else first[r]
        new = {}
        for i in range(m):
            p = f + i
            if bool(live[row + i]) and 0 <= p < length and 0 <= tables[r, p // page] < n_pages:
                new[p] = row + i
        for g in sorted({p // group for p in new}):
            here = [p for p in range(g * group, (g + 1) * group) if p < length]
            fresh = [p for p in here if p in new]
            stay = [p for p in here if p not in new]
            pg, at = int(tables[r, g * group // page]), (g * group % page) // group
            xs, ds = x[[new[p] for p in fresh]], delta[[new[p] for p in fresh]]           # [fresh, heads, dim]
            finite = torch.isfinite(xs)
            top = xs.abs().where(finite, torch.zeros(())).amax((0, 2))
            slack = ds.amax((0, 2))
            mine = torch.where(top < 2.0 ** -100, torch.zeros_like(top), top / most)
            old = scale0[pg, :, at].double() if stay else torch.zeros(heads, dtype=torch.float64)
            want = torch.maximum(mine, old)
            got = scale1[pg, :, at].double()
            assert ((got - want).abs() <= slack / most + 2 * F * want).all(), (what, r, g, got, want)
            kept_scale = old > mine + slack / most + 2 * F * mine
            assert (got[kept_scale] == old[kept_scale]).all(), (what, "a scale that stays", r, g)
            s = got[None, :, None]
            # new values: the nearest code, up to the roundings of value and quotient
            c = torch.stack([n1[pg, :, p % page] for p in fresh])
            q = torch.where(s > 0, torch.where(finite, xs, torch.sign(xs).nan_to_num(0.0) * most * s) / s, 0.0)
            half = step_at(torch.maximum(q.abs(), c.abs()), kind) / 2
            assert ((c - q.clamp(-most, most)).abs() * s <= half * s + ds + 4 * F * q.abs() * s).all(), (what, "codes", r, g)
            assert (c[(s == 0).expand_as(c)] == 0).all()
            # those that stay: untouched, or rounded to the scale that has grown
            for p in stay:
                a, b = n0[pg, :, p % page], n1[pg, :, p % page]
                grown = got > old
                assert torch.equal(raw0[pg, ~grown, p % page], raw1[pg, ~grown, p % page]), (what, "what stays", r, p)
                q = (a * old[:, None] / got[:, None].clamp(min=1e-300))[grown]
                half = step_at(torch.maximum(q.abs(), b[grown].abs()), kind) / 2
                assert ((b[grown] - q).abs() <= half + 6 * F * q.abs()).all(), (what, "rounded anew", r, p)
            for p in here:
                raw1[pg, :, p % page] = raw0[pg, :, p % page]
            same_scale[pg, :, at] = False
        row += m
    assert torch.equal(raw0, raw1), (what, "other positions")
    assert torch.equal(scale0.view(torch.int32)[same_scale], scale1.view(torch.int32)[same_scale]), (what, "other scales")        # (no numbers among them)
