"""Plain definitions of what a rollout step does between two attention calls: the page table, the slots of new tokens,
queries and keys by norm and rotation, and the rules of its logits.  Float64 and plain loops over items; test
infrastructure that shares no code with the HIP library.
"""
import math

import numpy as np

PAGE_TOKENS = 16


def page_table(seg_len, spare, old_offsets, old_pages, free_pages):
    """(offsets, pages) of the new table; -1 where the free pages end."""
    known = max(len(old_offsets) - 1, 0)
    offsets, pages, taken = [0], [], 0
    old = [min(max(int(x), 0), len(old_pages)) for x in old_offsets]
    for s, n in enumerate(seg_len):
        b = old[s] if s < known else 0
        had = max(old[s + 1] - b, 0) if s < known else 0
        need = max(had, -(-(max(int(n), 0) + spare) // PAGE_TOKENS))
        pages += [int(x) for x in old_pages[b:b + had]]
        for i in range(need - had):
            pages.append(int(free_pages[taken + i]) if taken + i < len(free_pages) else -1)
        taken += need - had
        offsets.append(offsets[-1] + need)
    return np.array(offsets, dtype=np.int64), np.array(pages, dtype=np.int64)


class Graph:
    """The arrays of a device graph; segments and pages outside them are empty, or none."""

    def __init__(self, seg_len, seg_page_offsets, seg_pages, path_offsets, path_segs, num_pages):
        self.seg_len, self.page_offsets, self.pages = seg_len, seg_page_offsets, seg_pages
        self.path_offsets, self.path_segs, self.num_pages = path_offsets, path_segs, num_pages

    def length(self, s):
        return max(int(self.seg_len[s]), 0) if 0 <= s < len(self.seg_len) else 0

    def slot(self, s, t):
        """Slot word of token t of segment s, or -1."""
        if not 0 <= s < len(self.seg_len):
            return -1
        at, end = int(self.page_offsets[s]) + t // PAGE_TOKENS, int(self.page_offsets[s + 1])
        if int(self.page_offsets[s]) < 0 or at >= min(end, len(self.pages)):
            return -1
        page = int(self.pages[at])
        return page * PAGE_TOKENS + t % PAGE_TOKENS if 0 <= page < self.num_pages else -1

    def path(self, b):
        lo, hi = int(self.path_offsets[b]), min(int(self.path_offsets[b + 1]), len(self.path_segs))
        return [int(s) for s in self.path_segs[lo:hi]] if 0 <= lo < hi else []


def slot_map(g: Graph, counts, capacity):
    """(token_offsets, slot_words, positions, branches), the last three [capacity]."""
    B = len(g.path_offsets) - 1
    offsets, rows = [0], []
    for b in range(B):
        n = 1 if counts is None else max(int(counts[b]), 0)
        offsets.append(min(offsets[-1] + n, 2**31 - 1))
        path = g.path(b)
        last = path[-1] if path else -1
        known = 0 <= last < len(g.seg_len)
        before = sum(g.length(s) for s in path[:-1])
        for j in range(min(n, max(0, capacity - len(rows)))):
            t = g.length(last) - n + j
            if known and t >= 0 and before + t < 2**31:
                rows.append((g.slot(last, t), before + t, b))
            else:
                rows.append((-1, -1, -1))
    rows = (rows + [(-1, -1, -1)] * (capacity - len(rows)))[:capacity]
    out = np.array(rows, dtype=np.int64).reshape(capacity, 3)
    return np.array(offsets, dtype=np.int64), out[:, 0], out[:, 1], out[:, 2]


def norm_rotate(x, positions, inv_freq, interleaved, weight, eps, scale):
    """(y, reach) of heads x [n, H, D]: reach is the sum of the magnitudes that a value is made of."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    half = len(inv_freq)
    y, reach = x.copy(), np.abs(x)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = np.asarray(positions, dtype=np.float64) * float(inv_freq[i])
        c, s = np.cos(angle)[:, None] * scale, np.sin(angle)[:, None] * scale
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        reach[..., a] = reach[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * abs(scale)
    return y, reach


def context(g: Graph, b, position, token_ids, prompt_segments):
    """[(token, of the prompt)] of branch b's tokens up to and with `position` (None: all); tokens without a page or
    with a negative id are left out."""
    out, at = [], 0
    for i, s in enumerate(g.path(b)):
        n = g.length(s)
        if position is not None:
            n = min(n, max(0, position + 1 - at))
        for t in range(n):
            w = g.slot(s, t)
            if w >= 0:
                out.append((int(token_ids[w]), i < prompt_segments))
        at += g.length(s)
    return out


def logits_row(x, seen, rep=None, freq=None, pres=None, temp=None, bias=(), allowed=None):
    """(z, reach) of one row: x [V] float64, seen as context() gives it, bias [(token, value)], allowed bool [V]."""
    V = len(x)
    z, size = np.array(x, dtype=np.float64), np.abs(np.asarray(x, dtype=np.float64))
    for v, value in bias:
        if 0 <= v < V:
            z[v] += value
            size[v] += abs(value)
    count, was = np.zeros(V), np.zeros(V, dtype=bool)
    for v, prompt in seen:
        if 0 <= v < V:
            was[v] = True
            count[v] += not prompt
    r = 1.0 if rep is None else float(rep)
    z = np.where(was, np.where(z > 0, z / r, z * r), z)
    size = np.where(was, size * max(r, 1 / r), size)
    take = (0.0 if freq is None else float(freq)) * count + (0.0 if pres is None else float(pres)) * (count > 0)
    taken = (0.0 if freq is None else abs(float(freq))) * count + (0.0 if pres is None else abs(float(pres))) * (count > 0)
    z, size = np.where(count > 0, z - take, z), size + taken
    t = 1.0 if temp is None else float(temp)
    z, size = z / t, size / t
    if allowed is not None:
        z = np.where(allowed, z, -math.inf)
    return z, size
