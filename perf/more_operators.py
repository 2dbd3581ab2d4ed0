"""The operators of a paged K/V cache in 8 bits that are timed, and what they have to return.

Pages hold codes, INT8 (-127 .. 127) or E4M3 (largest 448); a value is code * scale, with a scale for every `group` consecutive
positions of a K/V head, K and V each their own.  The operators:

  store   norms of queries and keys for each head, the rotation of both, K/V to codes and scales of the groups that the new rows fall
          into (values that stay there are rounded anew where the scale grows), and those groups read back
  read    positions read back in 16 bits or 32, K and V
  attend  attention of one or more new rows of every request over its pages, causal or bidirectional, with a sliding window and a
          few first positions that stay visible

`own` says whether run() calls the framework or computes the plain form.  Sizes are generic, or those of the package's own models
("8b": 32 heads of 128, blocks of 32 rows; "tiny": 4 heads of 64).
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
LARGEST = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -100                       # a group whose largest value is below has codes and scale 0


def listed():
    return [
        # eleven running requests that each get one more token, most of them into groups that are partly filled: latency only
        dict(name="store-11x1", kind="store", use="token", requests=11, rows=1, lo=30, hi=4000, lens=1, heads=32, kv_heads=8, dim=128, rot=128,
             given="bf16", rounded="bf16", codes="e4m3", group=16, page=16, interleaved=False, norms=True),
        # blocks of 32 rows of six requests of the 8b shape, from 32-bit sums of the projection, anywhere in their groups
        dict(name="store-6x32-f32", kind="store", use="block", requests=6, rows=32, lo=100, hi=2500, lens=2, heads=32, kv_heads=32, dim=128, rot=128,
             given="f32", rounded="f16", codes="int8", group=32, page=32, interleaved=True, norms=False),
        # four prompts prefilled at once, half of each head rotated, a scale for each position
        dict(name="store-4-prompts", kind="store", use="prompt", requests=4, rows=1, lo=1900, hi=5000, lens=3, heads=32, kv_heads=8, dim=128, rot=64,
             given="bf16", rounded="bf16", codes="e4m3", group=1, page=16, interleaved=False, norms=True),
        # a few positions of a request that is moved to another place: latency only
        dict(name="read-70", kind="read", rows=70, kv_heads=8, dim=128, rounded="f16", codes="int8", group=16, page=16, missing=0.05),
        # a long prefix read back for pages of 16 bits
        dict(name="read-24001", kind="read", rows=24001, kv_heads=8, dim=128, rounded="bf16", codes="e4m3", group=32, page=64, missing=0.0),
        # the tiny shape, one request, one token
        dict(name="attend-1x1", kind="attend", requests=1, rows_lo=1, rows_hi=1, lo=217, hi=217, lens=4, heads=4, kv_heads=4, dim=64,
             rounded="f16", codes="int8", group=16, page=16, causal=True, window=0, sinks=0),
        # 48 requests decode one token each, lengths from a few positions to 20000
        dict(name="attend-48x1", kind="attend", requests=48, rows_lo=1, rows_hi=1, lo=20, hi=20000, lens=5, heads=32, kv_heads=8, dim=128,
             rounded="bf16", codes="e4m3", group=16, page=16, causal=True, window=0, sinks=0),
        # two requests at a very long context, a scale for each position
        dict(name="attend-2x1-long", kind="attend", requests=2, rows_lo=1, rows_hi=1, lo=150001, hi=200000, lens=6, heads=32, kv_heads=8, dim=128,
             rounded="f16", codes="int8", group=1, page=64, causal=True, window=0, sinks=0),
        # block decoding at the 8b shape: 32 rows of each of ten requests see the whole sequence
        dict(name="attend-10x32", kind="attend", requests=10, rows_lo=32, rows_hi=32, lo=400, hi=3500, lens=7, heads=32, kv_heads=32, dim=128,
             rounded="f16", codes="int8", group=32, page=32, causal=False, window=0, sinks=0),
        # prompts that come in pieces behind what is cached of them
        dict(name="attend-4-pieces", kind="attend", requests=4, rows_lo=600, rows_hi=1500, lo=2500, hi=6000, lens=8, heads=32, kv_heads=8, dim=128,
             rounded="bf16", codes="e4m3", group=64, page=64, causal=True, window=0, sinks=0),
        # wide heads, a sliding window and four first positions that stay visible
        dict(name="attend-3-window-256", kind="attend", requests=3, rows_lo=300, rows_hi=1200, lo=2000, hi=5000, lens=9, heads=16, kv_heads=2, dim=256,
             rounded="bf16", codes="int8", group=1, page=16, causal=True, window=900, sinks=4),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["store", "store", "read", "attend", "attend", "attend", "attend"])
    page = rng.choice([16, 32, 64, 128])
    lens, codes, rounded = rng.randrange(1 << 20), rng.choice(["int8", "e4m3"]), rng.choice(["f16", "bf16"])
    group = rng.choice([g for g in (1, 16, 32, 64) if g <= page])
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (32, 32, 128), (4, 4, 64), (8, 8, 128), (28, 4, 128), (64, 8, 64), (16, 2, 128), (8, 1, 256)])
    common = dict(kind=kind, lens=lens, heads=heads, kv_heads=kv_heads, dim=dim, codes=codes, rounded=rounded, group=group, page=page)
    if kind == "read":
        return dict(kind=kind, rows=_spread(rng, 1, 24000), kv_heads=kv_heads if kv_heads < 32 else 8, dim=dim, rounded=rng.choice(["f16", "bf16", "f32"]),
                    codes=codes, group=group, page=page, missing=rng.choice([0.0, 0.0, 0.1]))
    if kind == "store":
        use = rng.choice(["token", "block", "prompt"])
        more = dict(rot=rng.choice([dim, dim, dim // 2]), given=rng.choice([rounded, rounded, "f32"]), interleaved=rng.random() < 0.4, norms=rng.random() < 0.6)
        if use == "token":
            return dict(common, use=use, requests=_spread(rng, 1, 200), rows=1, lo=4, hi=3000, **more)
        if use == "block":
            return dict(common, use=use, requests=rng.randint(1, 12), rows=rng.choice([5, 16, 32, 32, 48]), lo=64, hi=2500, **more)
        return dict(common, use=use, requests=rng.randint(1, 4), rows=1, lo=50, hi=_spread(rng, 60, 2800), **more)
    window = rng.choice([0, 0, rng.randint(1, 2000)])
    common.update(window=window, sinks=rng.randint(0, 40) if window else 0)
    use = rng.choice(["token", "token", "block", "prefill"])
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


def _lengths(case):
    """(rows, positions, first row's position) of every request."""
    rng, out = random.Random(case["lens"]), []
    for _ in range(case["requests"]):
        length = _between(rng, case["lo"], case["hi"])
        if case["kind"] == "attend":        # the rows are the last positions, those of a block lie anywhere
            rows = min(length, _between(rng, case["rows_lo"], case["rows_hi"]))
            out.append((rows, length, length - rows if case["causal"] else rng.randint(0, length - rows)))
        elif case["use"] == "prompt":
            out.append((length, length, 0))
        else:                               # one more token, or a block whose sequence goes on behind it
            rows = min(length, case["rows"])
            out.append((rows, length, length - rows if case["use"] == "token" else rng.randint(0, length - rows)))
    return out


def _touched(case, m, length, first):
    """First and last (exclusive) position of the groups that a request's rows fall into, as far as it goes."""
    group = case["group"]
    return first // group * group, min(length, -(-(first + m) // group) * group)


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


def _pool(case, n_pages, g, size):
    """Codes and scales of a pool: `size` = largest value of a group over the standard deviation of 1."""
    shape, most = (n_pages, case["kv_heads"], case["page"], case["dim"]), LARGEST[case["codes"]]
    x = (torch.randn(shape, dtype=torch.bfloat16, generator=g, device="cuda") * (most / size)).clamp_(-most, most)
    x = x.round_().to(torch.int8) if case["codes"] == "int8" else x.to(CODES["e4m3"])
    scale = torch.rand(shape[:2] + (case["page"] // case["group"],), generator=g, device="cuda")
    return x, (0.75 + 0.5 * scale) * (size / most)


def _pages(case, g):
    """Two pools and the tables of requests of these lengths; the pages lie anywhere."""
    page, lengths = case["page"], _lengths(case)
    counts = [-(-length // page) for _, length, _ in lengths]
    n_pages, columns = sum(counts) + 3, max(counts) + 2
    tables = torch.full((len(lengths), columns), -1, dtype=torch.int32, device="cuda")
    ids = torch.randperm(n_pages, generator=g, device="cuda").int()
    tables[torch.arange(columns, device="cuda") < torch.tensor(counts, device="cuda")[:, None]] = ids[:sum(counts)]
    (k, ks), (v, vs) = (_pool(case, n_pages, g, 4.0) for _ in range(2))
    cu = [0]
    for m, _, _ in lengths:
        cu.append(cu[-1] + m)
    return dict(case=case, k_pages=k, v_pages=v, k_scale=ks, v_scale=vs, tables=tables, cu_rows=_ints(cu),
                kv_len=_ints([length for _, length, _ in lengths]), first=_ints([f for _, _, f in lengths]),
                max_rows=max(m for m, _, _ in lengths), max_len=max(length for _, length, _ in lengths))


def _slots(tables, page, spans):
    """Slots of positions lo .. hi - 1 of every request, one behind the other."""
    request = torch.cat([torch.full((hi - lo,), r) for r, (lo, hi) in enumerate(spans)]).cuda()
    position = torch.cat([torch.arange(lo, hi) for lo, hi in spans]).cuda()
    return tables[request, position // page] * page + (position % page).int()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["kind"] == "read":
        n_pages = -(-case["rows"] // case["page"]) + 5
        (k, ks), (v, vs) = (_pool(case, n_pages, g, 4.0) for _ in range(2))
        at = torch.arange(case["rows"], device="cuda")
        slots = torch.randperm(n_pages, generator=g, device="cuda")[at // case["page"]] * case["page"] + at % case["page"]
        missing = torch.rand(case["rows"], generator=g, device="cuda") < case["missing"]
        return dict(case=case, k_pages=k, v_pages=v, k_scale=ks, v_scale=vs, slots=torch.where(missing, -1, slots).int())
    s = _pages(case, g)
    rows, heads, kv, dim = int(s["cu_rows"][-1]), case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "attend":
        s["q"] = (1.5 * torch.randn(rows, heads, dim, generator=g, device="cuda")).to(DTYPES[case["rounded"]])
        s["scale"] = 1.0 / math.sqrt(dim)
        return s
    # the projection's output: queries, keys and values of a row beside each other
    qkv = torch.randn(rows, heads + 2 * kv, dim, generator=g, device="cuda").to(DTYPES[case["given"]])
    s.update(q=qkv[:, :heads], k=qkv[:, heads:heads + kv], v=qkv[:, heads + kv:])
    lengths, n_pos = _lengths(case), 8192
    s["positions"] = torch.cat([torch.arange(f, f + m, dtype=torch.int32) for m, _, f in lengths]).cuda()
    s["back"] = _slots(s["tables"], case["page"], [_touched(case, *x) for x in lengths])
    gains = [1 + 0.2 * torch.randn(dim, generator=g, device="cuda") for _ in range(2)] if case["norms"] else [None, None]
    angles = torch.arange(n_pos, device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda").double() / case["rot"])
    s.update(q_gain=gains[0], k_gain=gains[1], table=torch.stack([angles.cos(), angles.sin()], -1).float())
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def _codes(pages, *at):
    """pages[at], by its bytes."""
    return pages.view(torch.int8)[at].view(pages.dtype)


def _values(pages, scale, slots, page, group):
    """Values at slots, 32 bits: [rows, kv_heads, dim]."""
    at, inside = slots // page, slots % page
    return _codes(pages, at, slice(None), inside).float() * scale[at, :, inside // group][..., None]


def _turned(x, cos, sin, rot, interleaved):
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, rest], -1)


def _rounded_codes(x, codes):
    most = LARGEST[codes]
    x = x.clamp(-most, most)
    return x.round().to(torch.int8) if codes == "int8" else x.to(CODES["e4m3"])


def _write(s, x, pages, scale, slots, kept):
    """x [rows, kv_heads, dim] to `slots`; `kept` [n_pages * page]: slots of positions that stay."""
    case = s["case"]
    page, group, most, (n_pages, kv, _, dim) = case["page"], case["group"], LARGEST[case["codes"]], pages.shape
    groups = n_pages * page // group
    in_group = slots // group
    index = in_group[:, None].expand(-1, kv)
    top = torch.zeros(groups, kv, device="cuda").scatter_reduce(0, index, x.abs().amax(-1), "amax")
    new = torch.zeros(groups, dtype=torch.bool, device="cuda")
    new[in_group] = True
    old = scale.permute(0, 2, 1).reshape(groups, kv)
    stays = kept.view(groups, group).any(1)[:, None]
    mine, theirs = torch.where(top < TINY, 0.0, top / most), torch.where(stays, old, 0.0)
    grows = mine > theirs
    now = torch.where(new[:, None], torch.maximum(mine, theirs), old)
    # x / scale, before the scale is rounded: values that lie between two codes stay there
    times, over = torch.where(mine >= theirs, most, 1.0), torch.where(mine >= theirs, top, theirs)
    over = torch.where(now > 0, over, float("inf"))
    # what stays is rounded anew where the scale has grown
    again = torch.nonzero(kept & new.repeat_interleave(group)).flatten()
    at, inside, of = again // page, again % page, again // group
    less = (old[of] * times[of] / over[of])[..., None]
    codes = _rounded_codes(_codes(pages, at, slice(None), inside).float() * less, case["codes"]).view(torch.int8)
    raw = pages.view(torch.int8)
    raw[at, :, inside] = torch.where(grows[of][..., None], codes, raw[at, :, inside])
    codes = _rounded_codes(x * times[in_group][..., None] / over[in_group][..., None], case["codes"])
    raw[slots // page, :, slots % page] = codes.view(torch.int8)
    scale.copy_(now.view(n_pages, page // group, kv).permute(0, 2, 1))


def _store_plain(s):
    case, dt = s["case"], DTYPES[s["case"]["rounded"]]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if case["norms"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + 1e-6) * s["q_gain"]
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + 1e-6) * s["k_gain"]
    angles = s["table"][s["positions"].long()][:, None]
    q, k = (_turned(x, angles[..., 0], angles[..., 1], case["rot"], case["interleaved"]) for x in (q, k))
    page, (n_pages, columns) = case["page"], (s["k_pages"].shape[0], s["tables"].shape[1])
    request = torch.searchsorted(s["cu_rows"][1:].contiguous(), torch.arange(q.shape[0], device="cuda", dtype=torch.int32), right=True)
    at = s["positions"].long()
    slots = s["tables"][request, at // page].long() * page + at % page
    # positions below a request's length, and not among the new rows
    p = torch.arange(columns * page, device="cuda")
    first = s["first"].long()[:, None]
    stays = (p < s["kv_len"][:, None]) & ~((p >= first) & (p < first + (s["cu_rows"][1:] - s["cu_rows"][:-1])[:, None]))
    kept = torch.zeros(n_pages * page + 1, dtype=torch.bool, device="cuda")
    ids = s["tables"].long().repeat_interleave(page, 1)
    kept[torch.where(stays, ids * page + p % page, n_pages * page)] = True
    _write(s, k, s["k_pages"], s["k_scale"], slots, kept[:-1])
    _write(s, v, s["v_pages"], s["v_scale"], slots, kept[:-1])
    back = s["back"].long()
    k, v = (_values(s[x + "_pages"], s[x + "_scale"], back, page, case["group"]).to(dt) for x in "kv")
    return q.to(dt), k, v, s["k_scale"], s["v_scale"]


def _read_plain(s):
    case, dt = s["case"], DTYPES[s["case"]["rounded"]]
    slots = s["slots"].long()
    there = (slots >= 0)[:, None, None]
    return tuple(torch.where(there, _values(s[x + "_pages"], s[x + "_scale"], slots.clamp(min=0), case["page"], case["group"]), 0.0).to(dt) for x in "kv")


def _attend_plain(s):
    case, n, most, length = s["case"], s["kv_len"].numel(), s["max_rows"], s["max_len"]
    heads, kv, dim, page, group = case["heads"], case["kv_heads"], case["dim"], case["page"], case["group"]
    i = torch.arange(most, device="cuda")
    count = (s["cu_rows"][1:] - s["cu_rows"][:-1]).long()
    at = torch.where(i < count[:, None], s["cu_rows"][:-1, None].long() + i, 0)            # [n, most]
    q = s["q"][at].float().view(n, most, kv, heads // kv, dim).permute(0, 2, 3, 1, 4).reshape(n * kv, -1, dim)
    ids = s["tables"][:, :-(-length // page)].long().clamp(min=0)

    def pages(pool, scale):
        x = _codes(pool, ids).float() * scale[ids].repeat_interleave(group, -1)[..., None]
        return x.permute(0, 2, 1, 3, 4).reshape(n * kv, -1, dim)[:, :length]
    z = torch.bmm(q, pages(s["k_pages"], s["k_scale"]).transpose(1, 2).contiguous()) * s["scale"]
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
    values = torch.where((key < s["kv_len"][:, None]).repeat_interleave(kv, 0)[:, :, None], pages(s["v_pages"], s["v_scale"]), 0.0)
    o = torch.bmm(e.view(n * kv, -1, length), values).view(n, kv, heads // kv, most, dim)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(n, most, heads, dim)
    return o[i < count[:, None]].to(s["q"].dtype)


def run(state):
    s, case = state, state["case"]
    if not own:
        return {"store": _store_plain, "read": _read_plain, "attend": _attend_plain}[case["kind"]](s)
    from paper_2511_21759_amd import binding as B
    pools = s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"]
    if case["kind"] == "store":
        q = B.odb_qk_norm_rope_quant(s["q"], s["k"], s["v"], *pools, s["table"], s["positions"], s["tables"], s["kv_len"], cu_rows=s["cu_rows"],
                                     first_pos=s["first"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=1e-6, interleaved=case["interleaved"],
                                     dtype=DTYPES[case["rounded"]])
        k, v = B.odb_paged_read_quant(*pools, s["back"], dtype=DTYPES[case["rounded"]])
        return q, k, v, s["k_scale"], s["v_scale"]
    if case["kind"] == "read":
        return B.odb_paged_read_quant(*pools, s["slots"], dtype=DTYPES[case["rounded"]])
    return B.odb_paged_attention_quant(s["q"], *pools, s["tables"], s["kv_len"], causal=case["causal"], cu_rows=s["cu_rows"], first_pos=s["first"],
                                       scale=s["scale"], window=case["window"], sinks=case["sinks"], max_rows=s["max_rows"], max_len=s["max_len"])


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    kv, dim, group = case["kv_heads"], case["dim"], case["group"]
    if case["kind"] == "read":
        elements = 2 * case["rows"] * kv * dim
        return {"bytes": elements * (1 + DTYPES[case["rounded"]].itemsize) + 8 * kv * -(-case["rows"] // group) + 4 * case["rows"], "flops": elements}
    heads, lengths = case["heads"], _lengths(case)
    rows = sum(m for m, _, _ in lengths)
    if case["kind"] == "store":
        spans = [_touched(case, *x) for x in lengths]
        back = sum(hi - lo for lo, hi in spans)
        groups = sum(-(-(hi - lo) // group) for lo, hi in spans)
        given = rows * (heads + 2 * kv) * dim * DTYPES[case["given"]].itemsize + rows * (case["rot"] * 4 + 4)
        written = rows * heads * dim * 2 + rows * 2 * kv * dim + 8 * kv * groups
        # read back: codes that were there before, values written (those just stored need no second read)
        return {"bytes": given + written + 2 * (back - rows) * kv * dim + back * (2 * kv * dim * 2 + 4), "flops": 10 * rows * (heads + 2 * kv) * dim}
    moved = pairs = 0
    for m, length, first in lengths:
        _, lo, _ = _seen(case, first, length)
        _, _, hi = _seen(case, first + m - 1, length)
        keys = max(0, hi - lo) + min(case["sinks"] if case["window"] else 0, lo)
        moved += 2 * keys * kv * dim + 8 * kv * -(-keys // group) + 4 * -(-keys // case["page"])
        pairs += sum(_seen(case, first + i, length)[0] for i in range(m))
    return {"bytes": moved + 2 * rows * heads * dim * 2, "flops": 4.0 * pairs * heads * dim}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------

def _nearest(x, codes):
    """The value that a code has, nearest to x, ties to the even one."""
    if codes == "int8":
        return x.round().clamp(-127, 127)
    _, e = torch.frexp(x)                                  # |x| in [2^(e-1), 2^e); below 2^-6 the steps stay those of 2^-6
    step = torch.pow(2.0, (e - 1).clamp(min=-6).double() - 3)
    return ((x / step).round() * step).clamp(-448, 448)


def _store_exact(s):
    case, page, group, rot, dim = s["case"], s["case"]["page"], s["case"]["group"], s["case"]["rot"], s["case"]["dim"]
    angle = torch.view_as_complex(s["table"].double())[s["positions"].long()]
    turned = []
    for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
        x = x.double()
        if case["norms"]:
            x = x / (x.pow(2).sum(-1, keepdim=True) / dim + 1e-6).sqrt() * gain.double()
        x = x.clone()
        pairs = x[..., :rot].unflatten(-1, (rot // 2, 2) if case["interleaved"] else (2, rot // 2))
        pairs = pairs if case["interleaved"] else pairs.transpose(-1, -2)
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * angle[:, None])
        x[..., :rot] = (pairs if case["interleaved"] else pairs.transpose(-1, -2)).flatten(-2)
        turned.append(x)
    most, out = LARGEST[case["codes"]], [turned[0]]
    scales, cu = [], s["cu_rows"].tolist()
    for x, pool, scale in ((turned[1], s["k_pages"], s["k_scale"]), (s["v"].double(), s["v_pages"], s["v_scale"])):
        scale, back = scale.double().clone(), []
        for r, (m, length, first) in enumerate(_lengths(case)):
            lo, hi = _touched(case, m, length, first)
            p = torch.arange(lo, hi, device="cuda")
            ids, inside = s["tables"][r, p // page].long(), p % page
            value = _codes(pool, ids, slice(None), inside).double()
            value[first - lo:first - lo + m] = x[cu[r]:cu[r + 1]]
            for a in range(lo, hi, group) if group > 1 else [None]:       # one group after the other; groups of one position need no loop
                if a is None:
                    top = value.abs().amax(-1)                             # all of them hold new rows only
                    top = torch.where(top < TINY, 0.0, top)
                    scale[ids, :, inside] = top / most
                    top = top[..., None]
                    value = torch.where(top > 0, _nearest(value * most / top, case["codes"]) * (top / most), 0.0)
                    continue
                part = slice(a - lo, min(a + group, hi) - lo)
                new = (p[part] >= first) & (p[part] < first + m)
                before, got = scale[ids[part.start], :, (a % page) // group].clone(), value[part]
                top = got[new].abs().amax((0, 2))
                unit = torch.where(top < TINY, 0.0, top / most)
                if bool(new.all()):
                    before = torch.zeros_like(before)
                unit = torch.maximum(unit, before)
                scale[ids[part.start], :, (a % page) // group] = unit
                unit, before, top = unit[None, :, None], before[None, :, None], top[None, :, None]
                fresh = torch.where(unit == top / most, got * most / top, got / unit)
                fresh = torch.where(unit > 0, _nearest(fresh, case["codes"]) * unit, 0.0)
                stay = torch.where(unit > before, _nearest(got * (before / unit), case["codes"]) * unit, got * before)
                value[part] = torch.where(new[:, None, None], fresh, stay)
            back.append(value)
        out.append(torch.cat(back))
        scales.append(scale)
    return (*out, *scales)


def _read_exact(s):
    case, out = s["case"], []
    slots = s["slots"].cpu()
    for pool, scale in ((s["k_pages"], s["k_scale"]), (s["v_pages"], s["v_scale"])):
        x = pool.double() * scale.double()[..., None].expand(-1, -1, -1, case["group"]).flatten(2)[..., None]
        x = x.transpose(1, 2).flatten(0, 1)                # [slots, kv_heads, dim]
        got = torch.zeros(len(slots), *x.shape[1:], dtype=torch.float64, device="cuda")
        there = torch.nonzero(slots >= 0).flatten().cuda()
        got[there] = x[s["slots"][there].long()]
        out.append(got)
    return tuple(out)


def _attend_exact(s):
    case, page, dim = s["case"], s["case"]["page"], s["case"]["dim"]
    per = case["heads"] // case["kv_heads"]
    out, cu = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), s["cu_rows"].tolist()
    for r, (m, length, first) in enumerate(_lengths(case)):
        ids = s["tables"][r, :-(-length // page)].long()
        row, key = first + torch.arange(m, device="cuda")[:, None], torch.arange(length, device="cuda")[None, :]
        hidden = torch.zeros(m, length, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden |= key > row
        if case["window"]:
            hidden |= ((row - key >= case["window"]) | (key - row >= case["window"])) & (key >= case["sinks"])
        at = torch.arange(length, device="cuda") // case["group"]
        for h in range(case["kv_heads"]):
            k, v = (_codes(x, ids, h).reshape(-1, dim)[:length].double() * y[ids, h].reshape(-1)[at].double()[:, None]
                    for x, y in ((s["k_pages"], s["k_scale"]), (s["v_pages"], s["v_scale"])))
            q = s["q"][cu[r]:cu[r + 1], h * per:(h + 1) * per].double().transpose(0, 1).reshape(-1, dim)
            z = (q @ k.t().contiguous()).view(per, m, length) * s["scale"]
            z = torch.softmax(z.masked_fill(hidden, float("-inf")), -1).nan_to_num(0.0)
            out[cu[r]:cu[r + 1], h * per:(h + 1) * per] = (z.view(-1, length) @ v).view(per, m, dim).transpose(0, 1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"store": _store_exact, "read": _read_exact, "attend": _attend_exact}[case["kind"]](s)
