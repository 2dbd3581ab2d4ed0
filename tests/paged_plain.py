"""Plain implementations of the paged K/V operators for the tests: one request after the other, in 64 bits, on the CPU."""
import math

import numpy as np
import torch


def page_tables(held, wanted, tables, free, n_free, page, first, count, cap, slots, positions):
    """Copies in, copies out: (len, tables, free, state, cu_rows, slots, positions) as lists and int arrays."""
    n, columns = tables.shape
    n_pages = len(free)
    tables, free, slots, positions = tables.copy(), free.copy(), slots.copy(), positions.copy()
    up = lambda x: -(-x // page)                                    # noqa: E731
    held = [min(max(h, 0), columns * page) for h in held]
    fits = [0 <= w <= columns * page for w in wanted]
    n_free = min(max(n_free, 0), n_pages)
    stack, given = list(free[:n_free]), 0
    for r in range(n):
        if fits[r]:
            for j in range(up(wanted[r]), up(held[r])):
                stack.append(tables[r, j])
                given += 1
    for i, page_id in enumerate(stack[n_free:]):
        if n_free + i < n_pages:
            free[n_free + i] = page_id
    need_so_far, taken, refused, length, there = 0, 0, 0, [], len(stack)
    for r in range(n):
        more = max(0, up(wanted[r]) - up(held[r])) if fits[r] else 0
        need_so_far += more
        if not fits[r] or (more and need_so_far > there):
            refused += 1
            length.append(held[r])
            continue
        for j in range(more):
            tables[r, up(held[r]) + j] = stack.pop()
        taken += more
        length.append(wanted[r])
    cu = [0]
    for r in range(n):
        p0 = held[r] if first is None else first[r]
        c = (wanted[r] - held[r] if fits[r] else 0) if count is None else count[r]
        c = min(max(c, 0), cap)
        for i in range(min(c, cap - cu[-1])):
            p, slot = p0 + i, -1
            if 0 <= p < length[r]:
                page_id = tables[r, p // page]
                if 0 <= page_id < n_pages:
                    slot = page_id * page + p % page
            positions[cu[-1] + i], slots[cu[-1] + i] = p, slot
        cu.append(min(cap, cu[-1] + c))
    state = [min(len(stack), n_pages), taken, given, refused]
    return length, tables, free, state, cu, slots, positions


def rope_table(n_pos, rot, base, scaling="plain", factor=1.0, original=0, fast=32.0, slow=1.0, magnitude=0.0, positions=None):
    """Rows of the table at `positions` (all by default), in the host's extended precision."""
    ld = np.longdouble
    two_pi = ld("6.28318530717958647692528676655900577")
    p = np.arange(n_pos) if positions is None else np.asarray(positions)
    j = np.arange(rot // 2).astype(ld)
    if scaling == "ntk" and rot > 2:
        base = ld(base) * ld(factor) ** (ld(rot) / (rot - 2))
    f = ld(base) ** (-2 * j / rot)
    if scaling == "linear":
        f = f / ld(factor)
    if scaling == "yarn":
        w = np.clip((original * f / two_pi - ld(slow)) / (ld(fast) - ld(slow)), 0, 1)
        f = f * w + f / ld(factor) * (1 - w)
    size = magnitude if magnitude else (0.1 * math.log(factor) + 1 if scaling == "yarn" else 1.0)
    a = p.astype(ld)[:, None] * f
    a = a - np.rint(a / two_pi) * two_pi
    return np.stack([np.cos(a), np.sin(a)], -1) * size


def rotate(x, gain, eps, angles, rot, interleaved):
    """x [rows, heads, dim] float64, angles [rows, rot / 2, 2] -> (result, sum of the magnitudes that make up each element)."""
    if gain is not None:
        x = x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * gain
    out, size = x.clone(), x.abs()
    c, s = angles[:, None, :, 0], angles[:, None, :, 1]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    u, w = x[..., a], x[..., b]
    out[..., a], out[..., b] = u * c - w * s, w * c + u * s
    size[..., a], size[..., b] = (u * c).abs() + (w * s).abs(), (w * c).abs() + (u * s).abs()
    return out, size


def attention(q, k_pages, v_pages, tables, kv_len, rows, first, scale, causal, window, sinks):
    """q [rows, heads, dim] float64 -> (out, weighted mean of |v|, largest scale * sum |q||k| of a row).  Keys that a row does not
    see are left out, never multiplied by zero; positions whose page lies outside the pool are seen by nobody."""
    n_pages, kv_heads, page, dim = k_pages.shape
    heads = q.shape[1]
    group = heads // kv_heads
    out, size, big = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64)
    row = 0
    for r, m in enumerate(rows):
        length = min(max(kv_len[r], 0), tables.shape[1] * page)
        key = torch.arange(length)
        ids = torch.tensor([int(x) for x in tables[r, :-(-length // page)]], dtype=torch.long)
        ids = ids.repeat_interleave(page)[:length]
        there = (ids >= 0) & (ids < n_pages)
        for i in range(m):
            p = (length - m if first is None else first[r]) + i
            seen = there.clone()
            if causal:
                seen &= key <= p
            if window:
                seen &= ((p - key).abs() < window) | (key < sinks)
            at = key[seen]
            if len(at):
                for h in range(kv_heads):
                    k = k_pages[ids[at], h, at % page].double()
                    v = v_pages[ids[at], h, at % page].double()
                    z = q[row, h * group:(h + 1) * group] @ k.t() * scale
                    w = torch.softmax(z, -1)
                    out[row, h * group:(h + 1) * group] = w @ v
                    size[row, h * group:(h + 1) * group] = w @ v.abs()
                    big[row, h * group:(h + 1) * group] = (q[row, h * group:(h + 1) * group].abs() @ k.abs().t()).amax(-1) * scale
            row += 1
    return out, size, big


def attention_many(q, k_pages, v_pages, tables, kv_len, rows, first, scale, causal, window, sinks):
    """attention() for many rows of requests whose visible positions hold numbers and lie in pages of the pool: all rows of a head at once."""
    page, dim = k_pages.shape[2:]
    group = q.shape[1] // k_pages.shape[1]
    out, size, big = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64)
    row = 0
    for r, m in enumerate(rows):
        length = kv_len[r]
        if m == 0 or length <= 0:                 # (rows that see nothing stay zero)
            row += m
            continue
        p = ((length - m if first is None else first[r]) + torch.arange(m))[:, None]
        key = torch.arange(length)[None, :]
        seen = torch.ones(m, length, dtype=torch.bool)
        if causal:
            seen &= key <= p
        if window:
            seen &= ((p - key).abs() < window) | (key < sinks)
        ids = torch.tensor([int(x) for x in tables[r, :-(-length // page)]], dtype=torch.long)
        for h in range(q.shape[1]):
            k, v = (x[ids, h // group].reshape(-1, dim)[:length].double() for x in (k_pages, v_pages))
            x = q[row:row + m, h]
            z = torch.softmax((x @ k.t() * scale).masked_fill(~seen, float("-inf")), -1).nan_to_num(0.0)
            out[row:row + m, h], size[row:row + m, h] = z @ v, z @ v.abs()
            big[row:row + m, h] = (x.abs() @ k.abs().t()).masked_fill(~seen, 0.0).amax(-1) * scale
        row += m
    return out, size, big
