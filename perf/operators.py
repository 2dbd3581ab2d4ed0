"""The operators of a paged K/V cache that are timed, and what they have to return.

Requests of different lengths share a pool of pages.  A page holds `page` positions of every K/V head; a request's
table names its pages in order.  The operators, in the order in which a serving step calls them:

  tables      page tables, slot maps and row offsets of a step, built on the GPU from the requests' lengths; pages are
              taken from, and given back to, a stack of free ones
  angles      the table of rotary cosines and sines, plain or scaled for long contexts
  rotate      norms of queries and keys for each head, the rotation of both, and K/V stored where the slot map says
  attend      attention of one or more new rows of every request over its pages, causal or bidirectional, with a
              sliding window and a few first positions that stay visible

`own` says whether run() calls the framework or computes the plain form.  Sizes are generic, or those of the package's own
models ("8b": 32 heads of 128, blocks of 32 rows; "tiny": 4 heads of 64).
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one step of 24 running requests that each get one more token: latency only
        dict(name="tables-append-24", kind="tables", mode="append", requests=24, page=16, columns=256, lo=5, hi=4000, lens=1, share=1.0),
        # a step in which 700 requests arrive, decode blocks of 32 rows, or have been cut behind a predicted end
        dict(name="tables-mixed-700", kind="tables", mode="mixed", requests=700, page=32, columns=300, lo=3, hi=9000, lens=2, share=1.0),
        # the table of a short context, made when a model is loaded
        dict(name="angles-4096", kind="angles", positions=4096, rot=64, scaling="plain", factor=1.0, original=0),
        # the table of a context stretched from 32768 positions to four times as many
        dict(name="angles-131072", kind="angles", positions=131072, rot=128, scaling="yarn", factor=4.0, original=32768),
        # single tokens of nine requests, grouped heads with norms of queries and keys
        dict(name="rotate-9", kind="rotate", rows=9, heads=32, kv_heads=8, dim=128, rot=128, given="bf16", cache="bf16",
             interleaved=False, norms=True, page=16, positions=8192),
        # blocks of 32 rows of seven requests of the 8b shape, from 32-bit sums of the projection
        dict(name="rotate-224-f32", kind="rotate", rows=224, heads=32, kv_heads=32, dim=128, rot=128, given="f32", cache="f16",
             interleaved=True, norms=False, page=32, positions=4096),
        # a long prefill, half of each head rotated
        dict(name="rotate-16411", kind="rotate", rows=16411, heads=32, kv_heads=8, dim=128, rot=64, given="bf16", cache="bf16",
             interleaved=False, norms=True, page=16, positions=32768),
        # the tiny shape, one request, one token
        dict(name="attend-1x1", kind="attend", requests=1, rows_lo=1, rows_hi=1, lo=333, hi=333, lens=3, heads=4, kv_heads=4, dim=64,
             cache="f16", page=16, causal=True, window=0, sinks=0),
        # 64 requests decode one token each, lengths from a few positions to 16384
        dict(name="attend-64x1", kind="attend", requests=64, rows_lo=1, rows_hi=1, lo=17, hi=16384, lens=4, heads=32, kv_heads=8, dim=128,
             cache="bf16", page=16, causal=True, window=0, sinks=0),
        # two requests at a very long context
        dict(name="attend-2x1-long", kind="attend", requests=2, rows_lo=1, rows_hi=1, lo=100001, hi=131072, lens=5, heads=32, kv_heads=8,
             dim=128, cache="f16", page=64, causal=True, window=0, sinks=0),
        # block decoding at the 8b shape: 32 rows of each of eight requests see the whole sequence
        dict(name="attend-8x32", kind="attend", requests=8, rows_lo=32, rows_hi=32, lo=500, hi=3000, lens=6, heads=32, kv_heads=32, dim=128,
             cache="f16", page=32, causal=False, window=0, sinks=0),
        # pieces of long prompts with a sliding window and four first positions that stay visible
        dict(name="attend-3x2048-window", kind="attend", requests=3, rows_lo=700, rows_hi=2048, lo=3500, hi=8192, lens=7, heads=32, kv_heads=8,
             dim=128, cache="bf16", page=16, causal=True, window=1024, sinks=4),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "angles", "rotate", "rotate", "attend", "attend", "attend", "attend"])
    lens = rng.randrange(1 << 20)
    if kind == "tables":
        page = rng.choice([16, 32, 64, 128])
        hi = _spread(rng, 200, 9000)
        return dict(kind=kind, mode=rng.choice(["append", "mixed", "mixed", "prefill"]), requests=_spread(rng, 1, 700), page=page,
                    columns=-(-hi // page) + rng.randint(3, 9), lo=3, hi=hi, lens=lens, share=rng.choice([1.0, 1.0, 0.6]))
    if kind == "angles":
        scaling = rng.choice(["plain", "linear", "ntk", "yarn"])
        return dict(kind=kind, positions=_spread(rng, 1, 131072), rot=2 * rng.randint(8, 64), scaling=scaling,
                    factor=1.0 if scaling == "plain" else rng.uniform(1.5, 16.0), original=rng.choice([2048, 4096, 8192]))
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (32, 32, 128), (4, 4, 64), (8, 8, 128), (28, 4, 128), (64, 8, 64), (16, 2, 128), (8, 1, 256)])
    if kind == "rotate":
        cache = rng.choice(["f16", "bf16"])
        return dict(kind=kind, rows=_spread(rng, 1, 12000), heads=heads, kv_heads=kv_heads, dim=dim,
                    rot=rng.choice([dim, dim, dim // 2, dim // 4]), given=rng.choice([cache, cache, "f32"]), cache=cache,
                    interleaved=rng.random() < 0.4, norms=rng.random() < 0.6, page=rng.choice([16, 32, 64]), positions=16384)
    use = rng.choice(["token", "token", "block", "prefill"])
    cache, page = rng.choice(["f16", "bf16"]), rng.choice([16, 32, 64, 128])
    window = rng.choice([0, 0, rng.randint(1, 2000)])
    common = dict(kind=kind, lens=lens, heads=heads, kv_heads=kv_heads, dim=dim, cache=cache, page=page, window=window,
                  sinks=rng.randint(0, 40) if window else 0)
    if use == "token":
        requests = _spread(rng, 1, 48)
        hi = min(60000, max(40, _spread(rng, 40, 2e7 / (requests * kv_heads * (dim / 128)))))
        return dict(common, requests=requests, rows_lo=1, rows_hi=rng.choice([1, 1, 1, 4]), lo=max(4, hi // rng.choice([1, 4, 50])), hi=hi, causal=True)
    if use == "block":
        hi = _spread(rng, 200, 3000)
        rows = rng.choice([7, 16, 32, 32, 48, 64])
        return dict(common, requests=rng.randint(1, 8), rows_lo=rows, rows_hi=rows, lo=max(rows, hi // 4), hi=hi, causal=False)
    hi = _spread(rng, 300, 6000)
    rows = min(hi, _spread(rng, 100, 1500))
    return dict(common, requests=rng.randint(1, 3), rows_lo=max(1, rows // 5), rows_hi=rows, lo=rows, hi=hi, causal=rng.random() < 0.7)


# ---- sizes that follow from a case -------------------------------------------------------------------------------

def _between(rng, lo, hi):
    return lo if hi <= lo else min(hi, max(lo, _spread(rng, lo, hi)))


def _step(case):
    """(held, wanted, first row, rows) of every request of a tables case."""
    rng, out = random.Random(case["lens"]), []
    for _ in range(case["requests"]):
        held = _between(rng, case["lo"], case["hi"])
        use = case["mode"] if case["mode"] != "mixed" else rng.choice(["append", "prefill", "block", "cut"])
        if use == "append":
            out.append((held, held + 1, held, 1))
        elif use == "prefill":
            out.append((0, held, 0, held))
        elif use == "block":           # the block's rows are computed anew, the sequence stays as long as it is
            first = rng.randint(0, max(0, held - 32))
            out.append((held, max(held, first + 32), first, 32))
        else:                          # cut behind a predicted end, no rows
            wanted = rng.randint(1, held)
            out.append((held, wanted, wanted, 0))
    return out


def _lengths(case):
    """(rows, positions) of every request of an attend case; the rows are the last positions, those of a block lie anywhere."""
    rng, out = random.Random(case["lens"]), []
    for _ in range(case["requests"]):
        length = _between(rng, case["lo"], case["hi"])
        rows = min(length, _between(rng, case["rows_lo"], case["rows_hi"]))
        first = length - rows if case["causal"] else rng.randint(0, length - rows)
        out.append((rows, length, first))
    return out


def _seen(case, position, length):
    """How many positions a row sees, and the first and last of its window."""
    hi = min(length, position + 1) if case["causal"] else length
    if not case["window"]:
        return hi, 0, hi
    lo = max(0, position - case["window"] + 1)
    hi = min(hi, position + case["window"])
    return max(0, hi - lo) + min(case["sinks"], lo), lo, hi


# ---- inputs -------------------------------------------------------------------------------------------------------

def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _prepare_tables(case, seed):
    step, page, g = _step(case), case["page"], _generator(seed)
    n, columns = case["requests"], case["columns"]
    held = [-(-h // page) for h, _, _, _ in step]
    more = sum(max(0, -(-w // page) - h) for (_, w, _, _), h in zip(step, held))
    spare = int(case["share"] * more) + 5
    n_pages = sum(held) + spare
    ids = torch.randperm(n_pages, generator=g, device="cuda").int()
    tables = torch.full((n, columns), -1, dtype=torch.int32, device="cuda")
    counts = torch.tensor(held, device="cuda")
    tables[torch.arange(columns, device="cuda") < counts[:, None]] = ids[:sum(held)]
    free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free[:spare] = ids[sum(held):]
    rows = sum(r for _, _, _, r in step)
    cap = -(-max(rows, 1) // 64) * 64
    return dict(case=case, n_pages=n_pages, held=_ints([s[0] for s in step]), wanted=_ints([s[1] for s in step]),
                first=_ints([s[2] for s in step]), count=_ints([s[3] for s in step]), tables=tables, free=free, n_free=_ints([spare]),
                slots=torch.full((cap,), -1, dtype=torch.int32, device="cuda"),
                positions=torch.full((cap,), -1, dtype=torch.int32, device="cuda"))


def _prepare_rotate(case, seed):
    g, rows, dim = _generator(seed), case["rows"], case["dim"]
    heads, kv = case["heads"], case["kv_heads"]
    # the projection's output: queries, keys and values of a row beside each other
    qkv = torch.randn(rows, heads + 2 * kv, dim, generator=g, device="cuda").to(DTYPES[case["given"]])
    n_pages = -(-rows // case["page"]) + 7
    shape = (n_pages, kv, case["page"], dim)
    pools = [torch.randn(shape, generator=g, device="cuda").to(DTYPES[case["cache"]]) for _ in range(2)]
    # consecutive rows fill a page, the pages lie anywhere; some rows are stored nowhere
    at = torch.arange(rows, device="cuda")
    pages = torch.randperm(n_pages, generator=g, device="cuda")
    slots = pages[at // case["page"]] * case["page"] + at % case["page"]
    slots = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.03, torch.full_like(slots, -1), slots)
    start = torch.randint(0, max(1, case["positions"] - rows), (1,), generator=g, device="cuda")
    positions = (at + start) % case["positions"]
    gains = [1 + 0.2 * torch.randn(dim, generator=g, device="cuda") for _ in range(2)] if case["norms"] else [None, None]
    angles = torch.arange(case["positions"], device="cuda").double()[:, None] * 10000.0 ** (
        -torch.arange(0, case["rot"], 2, device="cuda").double() / case["rot"])
    return dict(case=case, q=qkv[:, :heads], k=qkv[:, heads:heads + kv], v=qkv[:, heads + kv:], k_pages=pools[0], v_pages=pools[1],
                slots=slots.int(), positions=positions.int(), q_gain=gains[0], k_gain=gains[1],
                table=torch.stack([angles.cos(), angles.sin()], -1).float())


def _prepare_attend(case, seed):
    g, page, dt = _generator(seed), case["page"], DTYPES[case["cache"]]
    lengths = _lengths(case)
    n, rows = len(lengths), sum(r for r, _, _ in lengths)
    counts = [-(-length // page) for _, length, _ in lengths]
    n_pages, columns = sum(counts) + 3, max(counts) + 2
    shape = (n_pages, case["kv_heads"], page, case["dim"])
    k, v = (torch.randn(shape, dtype=dt, generator=g, device="cuda") for _ in range(2))
    q = (1.5 * torch.randn(rows, case["heads"], case["dim"], generator=g, device="cuda")).to(dt)
    tables = torch.full((n, columns), -1, dtype=torch.int32, device="cuda")
    ids = torch.randperm(n_pages, generator=g, device="cuda").int()
    tables[torch.arange(columns, device="cuda") < torch.tensor(counts, device="cuda")[:, None]] = ids[:sum(counts)]
    return dict(case=case, q=q, k_pages=k, v_pages=v, tables=tables, kv_len=_ints([length for _, length, _ in lengths]),
                first=_ints([f for _, _, f in lengths]), cu_rows=_ints([0] + list(np.cumsum([r for r, _, _ in lengths]))),
                max_rows=max(r for r, _, _ in lengths), max_len=max(length for _, length, _ in lengths),
                scale=1.0 / math.sqrt(case["dim"]))


def prepare(case, seed):
    if case["kind"] == "tables":
        return _prepare_tables(case, seed)
    if case["kind"] == "angles":
        # a table is made from numbers alone: the base is the input (models use 10000 to a few millions)
        return dict(case=case, base=float(random.Random(seed).choice([10000, 500000, 1000000]) + seed % 97))
    return _prepare_rotate(case, seed) if case["kind"] == "rotate" else _prepare_attend(case, seed)


# ---- one pass -----------------------------------------------------------------------------------------------------

def _tables_plain(s):
    case, cap, n_pages = s["case"], s["slots"].numel(), s["n_pages"]
    page, n, columns = case["page"], *s["tables"].shape
    held, wanted = s["held"].long().clamp(0, columns * page), s["wanted"].long()
    fits = (wanted >= 0) & (wanted <= columns * page)
    had = (held + page - 1) // page
    need = torch.where(fits, (wanted + page - 1) // page, had)
    take, give = (need - had).clamp(min=0), (had - need).clamp(min=0)
    taken, given = take.cumsum(0), give.cumsum(0)
    n_free = s["n_free"].long().clamp(0, n_pages)
    have = n_free + given[-1]
    granted = fits & ((take == 0) | (taken <= have))
    # pages given back go on top of the stack, then those that are granted come off it
    j = torch.arange(columns, device="cuda")[None, :]
    stack = torch.cat([s["free"], s["free"].new_zeros(1)])
    back = (j >= need[:, None]) & (j < had[:, None])
    to = n_free + (given - give)[:, None] + j - need[:, None]
    stack[torch.where(back, to, n_pages)] = s["tables"]
    gets = granted[:, None] & (j >= had[:, None]) & (j < need[:, None])
    at = have - 1 - ((taken - take)[:, None] + j - had[:, None])
    s["tables"].copy_(torch.where(gets, stack[torch.where(gets, at, n_pages)], s["tables"]))
    s["free"].copy_(stack[:n_pages])
    length = torch.where(granted, wanted, held)
    used = torch.where(granted, take, 0).sum()
    state = torch.stack([(have - used)[0], used, given[-1], (~granted).sum()])
    cu = torch.cat([taken.new_zeros(1), s["count"].long().clamp(0, cap).cumsum(0).clamp(max=cap)])
    i = torch.arange(cap, device="cuda")
    r = torch.searchsorted(cu[1:].contiguous(), i, right=True).clamp(max=n - 1)
    live = i < cu[n]
    p = s["first"].long()[r] + i - cu[r]
    ids = s["tables"][r, (p // page).clamp(0, columns - 1)].long()
    stored = (p >= 0) & (p < length[r]) & (ids >= 0) & (ids < n_pages)
    s["slots"].copy_(torch.where(live, torch.where(stored, ids * page + p % page, -1), s["slots"]))
    s["positions"].copy_(torch.where(live, p, s["positions"]))
    return length.int(), s["tables"], s["free"], state.int(), cu.int(), s["slots"], s["positions"]


def _frequencies(case, base):
    """Angle per position of every pair, 64 bits, and what cosines and sines are multiplied by."""
    rot, factor = case["rot"], case["factor"]
    if case["scaling"] == "ntk" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] != "yarn":
        return f, 1.0
    # pairs that turn more than 32 times in the original context stay, those that turn less than once are stretched
    turns = case["original"] * f / (2 * math.pi)
    keep = ((turns - 1.0) / 31.0).clamp(0, 1)
    return f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1.0


def _angles_plain(s):
    f, size = _frequencies(s["case"], s["base"])
    a = torch.arange(s["case"]["positions"], device="cuda", dtype=torch.float64)[:, None] * f
    return (torch.stack([a.cos(), a.sin()], -1) * size).float()


def _turned(x, cos, sin, rot, interleaved):
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, rest], -1)


def _rotate_plain(s):
    case, dt = s["case"], s["k_pages"].dtype
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if case["norms"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + 1e-6) * s["q_gain"]
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + 1e-6) * s["k_gain"]
    angles = s["table"][s["positions"].long()][:, None]
    cos, sin = angles[..., 0], angles[..., 1]
    q, k = (_turned(x, cos, sin, case["rot"], case["interleaved"]) for x in (q, k))
    slots = s["slots"].long()
    live = slots >= 0
    at, page = slots[live], case["page"]
    s["k_pages"][at // page, :, at % page] = k[live].to(dt)
    s["v_pages"][at // page, :, at % page] = v[live].to(dt)
    return q.to(dt), s["k_pages"], s["v_pages"]


def _attend_plain(s):
    case, n, most, length = s["case"], s["kv_len"].numel(), s["max_rows"], s["max_len"]
    heads, kv, dim, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    i = torch.arange(most, device="cuda")
    count = (s["cu_rows"][1:] - s["cu_rows"][:-1]).long()
    at = torch.where(i < count[:, None], s["cu_rows"][:-1, None].long() + i, 0)            # [n, most]
    q = s["q"][at].float().view(n, most, kv, heads // kv, dim).permute(0, 2, 3, 1, 4).reshape(n * kv, -1, dim)
    ids = s["tables"][:, :-(-length // page)].long().clamp(min=0)

    def pages(pool):
        x = pool[ids].permute(0, 2, 1, 3, 4).reshape(n * kv, -1, dim)[:, :length]
        return x.float()
    z = torch.bmm(q, pages(s["k_pages"]).transpose(1, 2).contiguous()) * s["scale"]
    z = z.view(n, kv, heads // kv, most, length)
    key, p = torch.arange(length, device="cuda"), (s["first"].long()[:, None] + i)[:, :, None]
    seen = key < s["kv_len"].long()[:, None, None]
    if case["causal"]:
        seen = seen & (key <= p)
    if case["window"]:
        seen = seen & (((p - key).abs() < case["window"]) | (key < case["sinks"]))
    z = torch.where(seen[:, None, None], z, float("-inf"))
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(top == float("-inf"), 0.0, top))
    total = e.sum(-1, keepdim=True)
    values = torch.where((key < s["kv_len"][:, None]).repeat_interleave(kv, 0)[:, :, None], pages(s["v_pages"]), 0.0)
    o = torch.bmm(e.view(n * kv, -1, length), values).view(n, kv, heads // kv, most, dim)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(n, most, heads, dim)
    return o[i < count[:, None]].to(s["q"].dtype)


def run(state):
    s, case = state, state["case"]
    if case["kind"] == "tables":
        if own:
            from paper_2511_21759_amd import binding as B
            length, cu, slots, positions, counts = B.odb_page_tables(
                s["held"], s["wanted"], s["tables"], s["free"], s["n_free"], case["page"], s["n_pages"], row_first=s["first"],
                row_count=s["count"], slots=s["slots"], positions=s["positions"])
            return length, s["tables"], s["free"], counts, cu, slots, positions
        return _tables_plain(s)
    if case["kind"] == "angles":
        if own:
            from paper_2511_21759_amd import binding as B
            return B.odb_rope_table(case["positions"], case["rot"], s["base"], scaling=case["scaling"], factor=case["factor"],
                                    original_len=case["original"])
        return _angles_plain(s)
    if case["kind"] == "rotate":
        if own:
            from paper_2511_21759_amd import binding as B
            q = B.odb_qk_norm_rope(s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["positions"], s["slots"],
                                   q_gain=s["q_gain"], k_gain=s["k_gain"], eps=1e-6, interleaved=case["interleaved"])
            return q, s["k_pages"], s["v_pages"]
        return _rotate_plain(s)
    if own:
        from paper_2511_21759_amd import binding as B
        return B.odb_paged_attention(s["q"], s["k_pages"], s["v_pages"], s["tables"], s["kv_len"], causal=case["causal"],
                                     cu_rows=s["cu_rows"], first_pos=s["first"], scale=s["scale"], window=case["window"],
                                     sinks=case["sinks"], max_rows=s["max_rows"], max_len=s["max_len"])
    return _attend_plain(s)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    if case["kind"] == "tables":
        step, page = _step(case), case["page"]
        n, rows = len(step), sum(r for _, _, _, r in step)
        pages = sum(abs(-(-w // page) - -(-h // page)) for h, w, _, _ in step)
        read = sum(-(-r // page) + 1 for _, _, _, r in step if r)          # entries behind the rows' slots
        return {"bytes": 4 * (6 * n + 2 * pages + read + 2 * rows), "flops": 0}
    if case["kind"] == "angles":
        return {"bytes": case["positions"] * case["rot"] * 4, "flops": 0}
    if case["kind"] == "rotate":
        elements = case["rows"] * (case["heads"] + 2 * case["kv_heads"]) * case["dim"]
        table = min(case["rows"], case["positions"]) * case["rot"] * 4
        return {"bytes": elements * (DTYPES[case["given"]].itemsize + 2) + table + case["rows"] * 8, "flops": 8 * elements}
    heads, kv, dim = case["heads"], case["kv_heads"], case["dim"]
    moved = pairs = rows = 0
    for m, length, first in _lengths(case):
        _, lo, _ = _seen(case, first, length)
        _, _, hi = _seen(case, first + m - 1, length)
        keys = max(0, hi - lo) + min(case["sinks"] if case["window"] else 0, lo)
        moved += 2 * keys * kv * dim * 2 + 4 * -(-keys // case["page"])
        pairs += sum(_seen(case, first + i, length)[0] for i in range(m))
        rows += m
    return {"bytes": moved + 2 * rows * heads * dim * 2, "flops": 4.0 * pairs * heads * dim}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------

def _tables_exact(s):
    """One request after the other, on the host."""
    case, page = s["case"], s["case"]["page"]
    tables, free = s["tables"].cpu().numpy().copy(), s["free"].cpu().numpy().copy()
    held, wanted, first, count = (s[x].tolist() for x in ("held", "wanted", "first", "count"))
    slots, positions = s["slots"].cpu().numpy().copy(), s["positions"].cpu().numpy().copy()
    top, given, used, refused, length, cu, stuck = int(s["n_free"][0]), 0, 0, 0, [], [0], False
    up = lambda x: -(-x // page)  # noqa: E731
    for r in range(len(held)):
        for j in range(up(wanted[r]), up(held[r])):
            free[top] = tables[r, j]
            top, given = top + 1, given + 1
    for r in range(len(held)):
        more = max(0, up(wanted[r]) - up(held[r]))
        if more and (stuck or more > top):
            stuck, refused = True, refused + 1
            length.append(held[r])
            continue
        for j in range(more):
            top, used = top - 1, used + 1
            tables[r, up(held[r]) + j] = free[top]
        length.append(wanted[r])
    for r in range(len(held)):
        p = first[r] + np.arange(count[r])
        inside = p < length[r]
        ids = tables[r, np.where(inside, p // page, 0)]
        at = slice(cu[-1], cu[-1] + count[r])
        positions[at] = p
        slots[at] = np.where(inside, ids * page + p % page, -1)
        cu.append(cu[-1] + count[r])
    return tuple(torch.from_numpy(np.asarray(x, np.int32)).cuda() for x in (length, tables, free, [top, used, given, refused], cu, slots, positions))


def _angles_exact(s):
    case, out = s["case"], []
    p = torch.arange(case["positions"], device="cuda", dtype=torch.float64)
    for j in range(case["rot"] // 2):
        share, base, factor, size = 2 * j / case["rot"], s["base"], case["factor"], 1.0
        f = math.exp(-share * math.log(base))
        if case["scaling"] == "linear":
            f /= factor
        elif case["scaling"] == "ntk" and case["rot"] > 2:
            f = math.exp(-share * (math.log(base) + case["rot"] / (case["rot"] - 2) * math.log(factor)))
        elif case["scaling"] == "yarn":
            turns, size = case["original"] * f / (2 * math.pi), 0.1 * math.log(factor) + 1
            keep = min(1.0, max(0.0, (turns - 1) / 31))
            f = (1 - keep) * f / factor + keep * f
        out.append(torch.view_as_real(torch.polar(torch.full_like(p, size), p * f)))
    return torch.stack(out, 1)


def _rotate_exact(s):
    case, page, rot = s["case"], s["case"]["page"], s["case"]["rot"]
    angle = torch.view_as_complex(s["table"].double())[s["positions"].long()]
    out = []
    for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
        x = x.double()
        if case["norms"]:
            x = x / (x.pow(2).sum(-1, keepdim=True) / case["dim"] + 1e-6).sqrt() * gain.double()
        x = x.clone()
        pairs = x[..., :rot].unflatten(-1, (rot // 2, 2) if case["interleaved"] else (2, rot // 2))
        pairs = pairs if case["interleaved"] else pairs.transpose(-1, -2)
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * angle[:, None])
        x[..., :rot] = (pairs if case["interleaved"] else pairs.transpose(-1, -2)).flatten(-2)
        out.append(x)
    k, v = s["k_pages"].double(), s["v_pages"].double()
    rows = torch.nonzero(s["slots"] >= 0).flatten()
    at = s["slots"][rows].long()
    where, inside = torch.div(at, page, rounding_mode="floor"), at.remainder(page)
    k[where, :, inside] = out[1][rows]
    v[where, :, inside] = s["v"][rows].double()
    return out[0], k, v


def _attend_exact(s):
    case, page, dim = s["case"], s["case"]["page"], s["case"]["dim"]
    group = case["heads"] // case["kv_heads"]
    out, cu = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), s["cu_rows"].tolist()
    for r, (m, length, first) in enumerate(_lengths(case)):
        ids = s["tables"][r, :-(-length // page)].long()
        row, key = first + torch.arange(m, device="cuda")[:, None], torch.arange(length, device="cuda")[None, :]
        hidden = torch.zeros(m, length, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden |= key > row
        if case["window"]:
            hidden |= ((row - key >= case["window"]) | (key - row >= case["window"])) & (key >= case["sinks"])
        for h in range(case["kv_heads"]):
            k, v = (x[ids, h].reshape(-1, dim)[:length].double() for x in (s["k_pages"], s["v_pages"]))
            q = s["q"][cu[r]:cu[r + 1], h * group:(h + 1) * group].double().transpose(0, 1).reshape(-1, dim)
            z = (q @ k.t().contiguous()).view(group, m, length) * s["scale"]
            z = torch.softmax(z.masked_fill(hidden, float("-inf")), -1).nan_to_num(0.0)
            out[cu[r]:cu[r + 1], h * group:(h + 1) * group] = (z.view(-1, length) @ v).view(group, m, dim).transpose(0, 1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"tables": _tables_exact, "angles": _angles_exact, "rotate": _rotate_exact, "attend": _attend_exact}[case["kind"]](s)
