"""What stands around the paged cache's reads and writes in plain form, on the CPU, from the definitions in include/gear.h: rotary positions
in 64 bits, and page tables one entry of a list after the other."""
import math

import torch

D = 128


def frequencies(rot, base=10000.0):
    return torch.tensor([base ** (-2.0 * p / rot) for p in range(rot // 2)], dtype=torch.float64)


def rotate(x, positions, freq, interleaved=False, inverse=False, factor=1.0):
    """(y, bound) in 64 bits: rows [n_seqs, tokens, heads, 128] at positions [n_seqs, tokens], and how far an implementation in the declared
    precisions may be off; |position * freq| below 2^24.

    A cosine or sine is off by 2^-22: the angle, reduced in 64 bits, by 2.5 roundings of at most 2^21.4 turns (2^-30 turns, 2^-27 rad) and by its rounding to fp32, at most
    pi / 4 (2^-25); the series by less than two roundings of numbers up to 1 and one more below 1 (2^-23 + 2^-25); times the factor, a rounding (2^-24).
    Their products with the two channels, in fp32: a rounding of the one, one of the fused sum, and one to the type."""
    dtype, half = x.dtype, freq.numel()
    eps = torch.finfo(dtype).eps / 2
    t = positions.double()[..., None, None] * freq * (-1.0 if inverse else 1.0)
    c, s = factor * torch.cos(t), factor * torch.sin(t)
    y, bound = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    p = torch.arange(half)
    i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + half)
    a, b = x.double()[..., i], x.double()[..., j]
    y[..., i], y[..., j] = a * c - b * s, a * s + b * c
    off = abs(factor) * (a.abs() + b.abs()) * (2.0 ** -22 + 2.0 ** -23)
    for k in (i, j):
        bound[..., k] = off + eps * (y[..., k].abs() + off) + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    return y, bound


class Table:
    """A page table as include/gear.h states it."""

    def __init__(self, n_pages, page, n_rows, width):
        self.page, self.width = page, width
        self.table = [[-1] * width for _ in range(n_rows)]
        self.kv = [0] * n_rows
        self.refs = [0] * n_pages

    def extend(self, rows, counts, most):
        """(slots, copies, refused)"""
        page, refs = self.page, list(self.refs)
        free = [p for p, r in enumerate(self.refs) if r == 0]
        slots, copies, refused = [], [], []
        taken, seen, counted_on = 0, set(), {}   # counted_on: page -> whether the last to give it up was refused
        for row, count in zip(rows, counts):
            out, pair, why = [-1] * most, [-1, -1], 0
            ok = 0 <= row < len(self.kv) and row not in seen
            seen.add(row)
            ok = ok and 0 <= count <= most and self.kv[row] + count <= self.width * page
            if not ok:
                why = 1
            elif count > 0:
                kv = self.kv[row]
                first, last = kv // page, (kv + count - 1) // page
                held = self.table[row][first] if kv % page else -1
                copy = held >= 0 and refs[held] > 1
                fresh = list(range(first if held < 0 or copy else first + 1, last + 1))
                start, taken = taken, taken + len(fresh)
                if fresh and taken > len(free):
                    why = 2
                if held >= 0 and not copy and counted_on.get(held):
                    why = 2
                if copy:
                    refs[held] -= 1
                    counted_on[held] = why == 2
                if not why:
                    if copy:
                        self.refs[held] -= 1
                        pair = [held, free[start]]
                    for k, e in enumerate(fresh):
                        self.table[row][e] = free[start + k]
                        self.refs[free[start + k]] = 1
                    for t in range(count):
                        out[t] = self.table[row][(kv + t) // page] * page + (kv + t) % page
                    self.kv[row] = kv + count
            slots.append(out)
            copies.append(pair)
            refused.append(why)
        return slots, copies, refused

    def truncate(self, rows, lens):
        for row, n in zip(rows, lens):
            if not 0 <= row < len(self.kv) or self.kv[row] <= max(n, 0):
                continue
            for e in range(-(-max(n, 0) // self.page), -(-self.kv[row] // self.page)):
                self.refs[self.table[row][e]] -= 1
                self.table[row][e] = -1
            self.kv[row] = max(n, 0)

    def fork(self, src, dst):
        was, kv, seen = [list(r) for r in self.table], list(self.kv), set()
        for a, b in zip(src, dst):
            if not (0 <= a < len(kv) and 0 <= b < len(kv)) or b in seen:
                continue
            seen.add(b)
            for p in self.table[b]:
                if p >= 0:
                    self.refs[p] -= 1
            self.table[b] = list(was[a])
            self.kv[b] = kv[a]
            for p in self.table[b]:
                if p >= 0:
                    self.refs[p] += 1

    def compact(self, most):
        """(moves, [pages in use, moves])"""
        live = sum(r > 0 for r in self.refs)
        free = [p for p in range(live) if self.refs[p] == 0]
        high = [p for p in range(len(self.refs) - 1, live - 1, -1) if self.refs[p] > 0]
        moves = list(zip(high, free))[:most]
        goes = dict(moves)
        self.table = [[goes.get(p, p) for p in r] for r in self.table]
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        return [list(m) for m in moves] + [[-1, -1]] * (most - len(moves)), [live, len(moves)]

    def consistent(self):
        count = [0] * len(self.refs)
        for r, kv in zip(self.table, self.kv):
            assert all(p >= 0 for p in r[:-(-kv // self.page)]) and all(p == -1 for p in r[-(-kv // self.page):])
            for p in r:
                if p >= 0:
                    count[p] += 1
        return count == self.refs


def shared_table(page, groups, n_pages, gen):
    """(q_start, kv_len, table, group_start, prefix_len, copies): sequences (new tokens, own tokens) of groups (shared tokens, sequences); a group without
    shared tokens is none.  copies: (page, its copy) where sequences part within a page."""
    q_start, kv, start, prefix, spans, copies = [0], [], [], [], [], []
    rows, used = [], 0
    order = torch.randperm(n_pages, generator=gen).tolist()
    for shared, seqs in groups:
        first = len(kv)
        for i, (n, own) in enumerate(seqs):
            total = shared + own
            if i == 0 or not shared:
                row = order[used:used + -(-total // page)]
                used += len(row)
            else:
                whole = shared // page
                fresh = order[used:used + -(-total // page) - whole]
                used += len(fresh)
                row = rows[first][:whole] + fresh
                if shared % page:
                    copies.append((rows[first][whole], fresh[0]))
            rows.append(row)
            kv.append(total)
            q_start.append(q_start[-1] + n)
        spans.append((first, len(kv)))
        prefix.append(shared)
    width = max(1, max(len(r) for r in rows))
    assert used <= n_pages
    table = torch.tensor([r + [-1] * (width - len(r)) for r in rows], dtype=torch.int32)
    return q_start, kv, table, [s for s, _ in spans] + [len(kv)], prefix, copies


def is_close(got, want, bound):
    off = (got.double() - want).abs()
    ratio = torch.where(off == 0, 0.0, off / bound)
    return float(ratio.max()) if ratio.numel() and not math.isnan(float(ratio.max())) else (0.0 if not ratio.numel() else math.inf)
