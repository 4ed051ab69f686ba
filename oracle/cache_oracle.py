"""Plain float64 definitions of the compressed cache: MXFP4 pages, the attention mass of cached tokens
and the choice of the tokens that stay.  Test infrastructure: it shares no code with the HIP library.

MXFP4: a block of 32 channels of one token's K or V is 2^e times one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (or a
negative) per channel.  Rounding searches the eight magnitudes; positions of codes and scales in a page
are written down index by index.
"""
import math

import numpy as np

from .graphattn_oracle import PAGE_TOKENS, query_context_length

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = 32
NAN_SCALE = 255


def block_exponent(x) -> int:
    """Exponent of a block's shared power of two, or None where it holds a NaN or an infinity."""
    x = np.asarray(x, dtype=np.float64)
    if not np.isfinite(x).all():
        return None
    top = float(np.abs(x).max())
    if top == 0.0:
        return -125
    e = math.frexp(top)[1] - 1 - 2                 # floor(log2 top) - 2
    if top >= 7.0 * 2.0 ** e:
        e += 1
    return min(max(e, -125), 125)


def nearest_code(y: float) -> int:
    """Code of the magnitude nearest to |y| (ties to the even code), bit 3 the sign."""
    a = abs(y)
    best = min(range(8), key=lambda c: (abs(MAGNITUDES[c] - a), c & 1))
    return best + (8 if math.copysign(1.0, y) < 0 else 0)


def quantise_block(x):
    """(32 codes, scale byte) of a block."""
    e = block_exponent(x)
    if e is None:
        return [0] * BLOCK, NAN_SCALE
    return [nearest_code(float(v) * 2.0 ** -e) for v in x], e + 127


def code_value(code: int, byte: int) -> float:
    if byte == NAN_SCALE:
        return math.nan
    v = MAGNITUDES[code & 7] * 2.0 ** (byte - 127)
    return -v if code & 8 else v


def code_place(t: int, c: int, D: int, value: bool):
    """(byte of a page's head block, half of the byte) of channel c of token t of K (or V)."""
    if not value:
        return t * (D // 2) + c // 2, c % 2
    w = D // 16
    return 8 * D + ((t // 4 * 16 + c // w) * 4 + t % 4) * (w // 2) + (c % w) // 2, c % 2


def scale_place(t: int, c: int, D: int, value: bool) -> int:
    if not value:
        return 16 * D + t * (D // BLOCK) + c // BLOCK
    return 16 * D + D // 2 + (t // 4 * (D // BLOCK) + c // BLOCK) * 4 + t % 4


def append(pool: np.ndarray, k, v, slot_words) -> np.ndarray:
    """The pool (uint8 [P, Hkv, 17 D]) with tokens k / v [n, Hkv, D] (float64) stored; words outside
    the pool are skipped."""
    out = pool.copy()
    P, H, blk = pool.shape
    D = blk // 17
    for j, w in enumerate(int(x) for x in slot_words):
        if not 0 <= w < P * PAGE_TOKENS:
            continue
        page, t = divmod(w, PAGE_TOKENS)
        for h in range(H):
            for value, x in ((False, k), (True, v)):
                for b in range(0, D, BLOCK):
                    codes, byte = quantise_block(x[j, h, b:b + BLOCK])
                    out[page, h, scale_place(t, b, D, value)] = byte
                    for i, code in enumerate(codes):
                        at, half = code_place(t, b + i, D, value)
                        old = int(out[page, h, at])
                        out[page, h, at] = (old & 0xF0) | code if half == 0 else (old & 0x0F) | code << 4
    return out


_PLACES = {}


def _places(D: int):
    if D not in _PLACES:
        code = np.zeros((2, PAGE_TOKENS, D), dtype=np.int64)
        half = np.zeros_like(code)
        scale = np.zeros_like(code)
        for value in (0, 1):
            for t in range(PAGE_TOKENS):
                for c in range(D):
                    code[value, t, c], half[value, t, c] = code_place(t, c, D, bool(value))
                    scale[value, t, c] = scale_place(t, c, D, bool(value))
        _PLACES[D] = code, half, scale
    return _PLACES[D]


def pool_values(pool: np.ndarray) -> np.ndarray:
    """float64 [P, Hkv, 2, 16, D] values of a pool uint8 [P, Hkv, 17 D]."""
    D = pool.shape[2] // 17
    code, half, scale = _places(D)
    byte = pool[:, :, code].astype(np.int64)
    nib = np.where(half == 1, byte >> 4, byte & 15)
    mag = np.array(MAGNITUDES + tuple(-m for m in MAGNITUDES))
    s = pool[:, :, scale].astype(np.int64)
    val = mag[nib] * np.exp2((s - 127).astype(np.float64))
    return np.where(s == NAN_SCALE, np.nan, val)


def attend_rows(q, values, graph, Hq: int, Hkv: int, counts=None, scale=None, rows=None):
    """Textbook attention of every query row (or the listed ones) over its branch's context, from
    values [P, Hkv, 2, 16, D].  counts: queries per branch (None: one each).  Yields (row, slot words
    seen, scores [Hq, L], probabilities [Hq, L], K [L, Hkv, D], V [L, Hkv, D])."""
    D = values.shape[-1]
    scale = 1.0 / math.sqrt(D) if not scale else scale
    group = Hq // Hkv
    wanted = None if rows is None else set(int(r) for r in rows)
    r = 0
    for b in range(graph.num_branches):
        n = 1 if counts is None else int(counts[b])
        if wanted is not None and not wanted & set(range(r, r + n)):
            r += n
            continue
        words = []
        for s in graph.path(b):
            for t in range(int(graph.seg_len[s])):
                page = int(graph.seg_pages[graph.seg_page_offsets[s] + t // PAGE_TOKENS])
                words.append(page * PAGE_TOKENS + t % PAGE_TOKENS)
        words = np.array(words)
        kv = values[words // PAGE_TOKENS, :, :, words % PAGE_TOKENS]       # [L, Hkv, 2, D]
        for i in range(n):
            if wanted is None or r in wanted:
                L = query_context_length(len(words), n, i)
                K, V = kv[:L, :, 0], kv[:L, :, 1]
                s = np.stack([scale * (K[:, h // group] @ q[r, h]) for h in range(Hq)])
                p = np.exp(s - s.max(1, keepdims=True))
                yield r, words[:L], s, p / p.sum(1, keepdims=True), K, V
            r += 1


def attention(q, values, graph, Hq, Hkv, counts=None, scale=None, rows=None):
    """(out [n, Hq, D], lse [n, Hq], spread [n, Hq, D], reach): the result, the probability-weighted
    sum of |V| per output, and the largest sum of |scale q k| of any score (both bound rounding)."""
    group = Hq // Hkv
    D = values.shape[-1]
    sc = 1.0 / math.sqrt(D) if not scale else scale
    outs, lses, spread, reach = [], [], [], 0.0
    for r, _, s, p, K, V in attend_rows(q, values, graph, Hq, Hkv, counts, scale, rows):
        m = s.max(1)
        lses.append(m + np.log(np.exp(s - m[:, None]).sum(1)))
        outs.append(np.stack([p[h] @ V[:, h // group] for h in range(Hq)]))
        spread.append(np.stack([p[h] @ np.abs(V[:, h // group]) for h in range(Hq)]))
        reach = max(reach, max(float((sc * np.abs(K[:, h // group]) @ np.abs(q[r, h])).max())
                               for h in range(Hq)))
    return np.stack(outs), np.stack(lses), np.stack(spread), reach


def mass(q, values, graph, lse, Hq, Hkv, mass_in, decay, counts=None, scale=None):
    """decay x mass_in plus the weights exp(score - lse) of every slot that some row sees (other
    slots: NaN)."""
    new = np.zeros_like(np.asarray(mass_in, dtype=np.float64))
    hit = np.zeros(len(new), dtype=bool)
    # Slots of segments on a path count even where no row of a multi-query call sees them.
    for s in sorted(set(int(x) for x in graph.path_segs)):
        for t in range(int(graph.seg_len[s])):
            page = int(graph.seg_pages[graph.seg_page_offsets[s] + t // PAGE_TOKENS])
            hit[page * PAGE_TOKENS + t % PAGE_TOKENS] = True
    for r, words, s, _, _, _ in attend_rows(q, values, graph, Hq, Hkv, counts, scale):
        live = np.isfinite(lse[r])
        new[words] += np.exp(s[live] - lse[r][live, None]).sum(0)
    return np.where(hit, decay * np.asarray(mass_in, dtype=np.float64) + new, np.nan)


def keep_tokens(weights, keep: int, first: int, recent: int):
    """Positions that stay of one segment with these weights, ascending."""
    n = len(weights)

    def rank(t):
        if t < first or t >= n - recent:
            return (0, 0.0, t)
        if math.isnan(weights[t]):
            return (1, 0.0, t)
        return (2, -float(weights[t]), t)

    return sorted(sorted(range(n), key=rank)[:keep])


def evict_select(mass_, seg_len, seg_page_offsets, seg_pages, keep, first: int, recent: int):
    """(positions, slot words) of the tokens that stay, segments one behind the other."""
    pos, words = [], []
    for s, n in enumerate(int(x) for x in seg_len):
        at = [int(seg_pages[seg_page_offsets[s] + t // PAGE_TOKENS]) * PAGE_TOKENS + t % PAGE_TOKENS
              for t in range(n)]
        stay = keep_tokens([float(mass_[w]) for w in at], int(keep[s]), first, recent)
        pos += stay
        words += [at[t] for t in stay]
    return np.array(pos, dtype=np.int64), np.array(words, dtype=np.int64)
