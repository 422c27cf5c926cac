"""Plain implementations of the paged-cache operators for the tests: attention
in 64 bits from its definition, the page bookkeeping as loops over Python
lists.  Nothing here comes from the library."""
import math

import torch


class Rows:
    """A batch's packed rows: request i has depth[i] + 1 rows from offsets[i]."""

    def __init__(self, depth, K, packed=True):
        self.depth, self.K, self.B = list(depth), K, len(depth)
        self.offsets = [0]
        for n in self.depth:
            self.offsets.append(self.offsets[-1] + (n + 1 if packed else K + 1))
        self.packed = packed
        self.R = self.offsets[-1]


def random_table(B, slots_needed, pages, max_pages, gen, hole=lambda i, t: False):
    """A table that gives every needed slot a page of its own, in random order."""
    perm = torch.randperm(pages, generator=gen).tolist()
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    for i in range(B):
        for t in range(slots_needed[i]):
            if not hole(i, t):
                table[i, t] = perm.pop()
    return table


def visible(P, window, sinks):
    """Positions that a row at position P sees."""
    if P < 0:
        return []
    if window == 0:
        return list(range(P + 1))
    lo = max(0, P - window + 1)
    return list(range(min(sinks, lo))) + list(range(lo, P + 1))


def attend(q, k, v, table, pos, rows, scale, window=0, sinks=0):
    """out, lse and the two sums the error bounds are made of, all fp64 on the CPU:
    sum_t p_t |v_t| and max_t scale * sum_d |q_d k_td|.  Rows of no request are NaN."""
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    table = table.cpu()
    R, Hq, D = q.shape
    ps, Hkv = k.shape[1], k.shape[2]
    G = Hq // Hkv
    out = torch.full((R, Hq, D), float("nan"), dtype=torch.float64)
    lse = torch.full((R, Hq), float("nan"), dtype=torch.float64)
    mass, big = torch.zeros_like(out), torch.zeros_like(lse)
    for i in range(rows.B):
        for j in range(rows.depth[i] + 1):
            r = rows.offsets[i] + j
            t = visible(int(pos[i]) + j, window, sinks)
            if not t:
                out[r], lse[r] = 0.0, float("-inf")
                continue
            t = torch.tensor(t)
            page = table[i][t // ps].long()
            kk = k[page, t % ps].repeat_interleave(G, dim=1)      # [T, Hq, D]
            vv = v[page, t % ps].repeat_interleave(G, dim=1)
            x = torch.einsum("hd,thd->ht", q[r], kk) * scale
            lse[r] = torch.logsumexp(x, 1)
            p = torch.exp(x - lse[r][:, None])
            out[r] = torch.einsum("ht,thd->hd", p, vv)
            mass[r] = torch.einsum("ht,thd->hd", p, vv.abs())
            big[r] = (torch.einsum("hd,thd->ht", q[r].abs(), kk.abs()) * scale).amax(1)
    return out, lse, mass, big


def bounds(out, mass, big, terms, D, bf16):
    """Error bounds of the kernel's out and lse, from its arithmetic.

    A score is a sum of D exact (bf16) or rounded (fp32) products in fp32: off
    by at most (D + 2) 2^-23 big, truncating adders included, and by 2^-23 big
    more for its scaling; a weight 2^x by ln 2 times that and 2^-22 of its own
    rounding; a sum of `terms` weights or products by terms 2^-23.  With bf16
    every weight is rounded to 8 bits (2^-9) before it meets its value, and the
    result is once more."""
    score = (D + 4) * 2.0 ** -23 * big
    weight = 2 * score + 2.0 ** -21 + (terms + 8) * 2.0 ** -23
    tol = mass * weight[..., None] + out.abs() * 2.0 ** -23 + 1e-37
    if bf16:
        tol = tol + mass * 2.0 ** -9 + out.abs() * 2.0 ** -9 * 1.01 + mass * 2.0 ** -17
    return tol, weight + 2.0 ** -22 * 20


# ---------------------------------------------------------------------------
# Pages, as lists
# ---------------------------------------------------------------------------
def fork(table, refs, parent):
    M = len(table[0])
    out = [list(table[p]) if p >= 0 else [-1] * M for p in parent]
    refs = list(refs)
    for row in out:
        for e in row:
            if e >= 0:
                refs[e] += 1
    for row in table:
        for e in row:
            if e >= 0:
                refs[e] -= 1
    return out, refs


def reserve(table, refs, pos, depth, page_size):
    table, start, refs = [list(r) for r in table], list(refs), list(refs)
    free = [p for p, n in enumerate(start) if n == 0]
    src, dst, granted, used, full = [], [], [], 0, False
    wanted = 0
    for i, row in enumerate(table):
        a, b = max(0, pos[i]), pos[i] + depth[i]
        slots = range(a // page_size, b // page_size + 1) if b >= 0 else []
        need = [t for t in slots if row[t] < 0 or start[row[t]] > 1]
        wanted += len(need)
        ok = not need or wanted <= len(free)
        granted.append(1 if ok else 0)
        full |= not ok
        if not ok:
            continue
        for t in need:
            page = free[used]
            used += 1
            if row[t] >= 0:
                src.append(row[t])
                dst.append(page)
                refs[row[t]] -= 1
            refs[page] = 1
            row[t] = page
    return table, refs, src, dst, used, granted, full


def release(table, refs, keep, page_size, window=0, sinks=0):
    table, refs = [list(r) for r in table], list(refs)
    for i, row in enumerate(table):
        for t, e in enumerate(row):
            past = t * page_size >= keep[i]
            hidden = window > 0 and (t + 1) * page_size <= keep[i] - window + 1 and t * page_size >= sinks
            if e >= 0 and (past or hidden):
                row[t] = -1
                refs[e] -= 1
    return table, refs


def compact(table, refs):
    n = sum(1 for c in refs if c > 0)
    src = [p for p, c in enumerate(refs) if c > 0 and p >= n]
    dst = [p for p, c in enumerate(refs) if c <= 0 and p < n]
    where = {p: p for p, c in enumerate(refs) if c > 0 and p < n}
    where.update(zip(src, dst))
    out = [0] * len(refs)
    for p, c in enumerate(refs):
        if c > 0:
            out[where[p]] = c
    table = [[where.get(e, -1) if e >= 0 else -1 for e in row] for row in table]
    return table, out, src, dst, [where.get(p, -1) for p in range(len(refs))], n


def random_pages(B, max_pages, pages, have, gen, share=0.3, extra=0):
    """A table with shared prefixes and its counts; `extra` pages are held by no table entry."""
    order = torch.randperm(pages, generator=gen).tolist()
    table = [[-1] * max_pages for _ in range(B)]
    refs = [0] * pages
    for i in range(B):
        common = int(share * min(have[i], have[i - 1])) if i % 3 and i else 0
        for t in range(have[i]):
            table[i][t] = table[i - 1][t] if t < common else order.pop()
            refs[table[i][t]] += 1
    for _ in range(extra):
        refs[order.pop()] = 1
    return table, refs


def sqrt_scale(D):
    return 1.0 / math.sqrt(D)
