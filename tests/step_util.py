"""Cases of the calls between two attention calls, drawn and built by hand, their oracle values and tolerances.

A case is a dict of numpy arrays and numbers; tests run it on the CPU model of the device and on the GPU alike.
"""
import numpy as np

from oracle import step_oracle as S

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def to_bf16(x):
    """float64 / float32 values as bf16 bits (uint16), to nearest even."""
    w = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    nan = np.isnan(np.asarray(x, dtype=np.float32))
    return np.where(nan, 0x7FC0, (w + 0x7FFF + ((w >> 16) & 1)) >> 16).astype(np.uint16)


def values(a, dtype):
    """float64 values of bf16 bits or float32."""
    if dtype == "f32":
        return a.astype(np.float64)
    return (a.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def stored(x, dtype):
    return np.asarray(x, dtype=np.float32) if dtype == "f32" else to_bf16(x)


# Graphs ---------------------------------------------------------------------------------------------------

def graph(lens, paths, rng, spare_pages=0, offsets=None):
    """A graph with a random placement of its pages (and spare_pages per segment more than its tokens need)."""
    need = [(max(n, 0) + 15) // 16 + spare_pages for n in lens]
    off = np.concatenate([[0], np.cumsum(need)]).astype(np.int64)
    num_pages = int(off[-1]) + 2
    pages = rng.permutation(num_pages)[:off[-1]].astype(np.int32)
    po = np.concatenate([[0], np.cumsum([len(p) for p in paths])]).astype(np.int64)
    ps = np.array([s for p in paths for s in p], dtype=np.int32)
    return {"seg_len": np.array(lens, dtype=np.int32), "off": off, "pages": pages, "po": po, "ps": ps,
            "num_pages": num_pages}


def random_graph(rng, most_branches=40, most_len=70, bad=False):
    n_seg = int(rng.integers(1, 30))
    lens = rng.integers(0 if bad else 1, most_len, n_seg)
    paths = [list(rng.permutation(n_seg)[:rng.integers(0 if bad else 1, min(n_seg, 6) + 1)])
             for _ in range(rng.integers(1, most_branches))]
    g = graph(lens, paths, rng, int(rng.integers(0, 2)))
    if bad:
        # Indices outside their arrays, here and there: empty segments and no pages, never a fault.
        for name, extremes in (("seg_len", [-5, -2**31]), ("pages", [-1, 2**31 - 1, g["num_pages"]]),
                               ("ps", [-1, n_seg, 2**31 - 1]), ("off", [-3, 2**62, -2**62, 2**63 - 1]),
                               ("po", [-1, 2**40, 2**63 - 1])):
            a = g[name]
            for i in rng.integers(0, max(len(a), 1), 1 + len(a) // 20):
                if len(a):
                    a[i] = rng.choice(np.array(extremes, dtype=a.dtype))
    return g


def oracle_graph(g):
    return S.Graph(g["seg_len"], g["off"], g["pages"], g["po"], g["ps"], g["num_pages"])


# Page tables ----------------------------------------------------------------------------------------------

def page_case(rng, n_seg=None, bad=False):
    n = int(rng.integers(0, 60)) if n_seg is None else n_seg
    lens = rng.integers(0, 90, n).astype(np.int32)
    known = int(rng.integers(0, n + 1))
    old = np.concatenate([[0], np.cumsum(rng.integers(0, 7, known))]).astype(np.int64)
    total = int(old[-1])
    spare = int(rng.choice([0, 1, 16, 33]))
    need = int(((np.maximum(lens, 0) + spare + 15) // 16).sum())
    ids = rng.permutation(total + need + 5).astype(np.int32)
    free = ids[total:total + int(rng.integers(0, need + 5))]
    if bad and known:
        for i in rng.integers(0, known + 1, 2):
            old[i] = rng.choice(np.array([-7, 2**40, -2**62, 2**63 - 1]))
        lens[rng.integers(0, n)] = -9
    capacity = max(0, total + need + int(rng.integers(-6, 9)))
    return {"op": 0, "lens": lens, "spare": spare, "old": old if known else np.zeros(0, np.int64),
            "old_pages": ids[:total] if known else ids[:0], "free": free, "capacity": capacity}


def check_page(c, off, pages):
    want, list_ = S.page_table(c["lens"], c["spare"], c["old"], c["old_pages"], c["free"])
    np.testing.assert_array_equal(off, want)
    n = min(c["capacity"], len(list_))
    np.testing.assert_array_equal(pages[:n], list_[:n])
    assert (pages[n:] == -77).all()                       # left as they were


# Slot maps ------------------------------------------------------------------------------------------------

def slot_case(rng, bad=False, g=None, counts="drawn"):
    g = random_graph(rng, bad=bad) if g is None else g
    B = len(g["po"]) - 1
    if isinstance(counts, str):
        counts = None if rng.random() < 0.2 else rng.integers(-1 if bad else 0, 9, B).astype(np.int32)
        if counts is not None and bad and B:
            counts[rng.integers(0, B)] = rng.choice([2**31 - 1, -2**31, 500])
    total = B if counts is None else int(np.maximum(counts.astype(np.int64), 0).sum())
    capacity = max(0, min(total, 4000) + int(rng.integers(-4, 40)))
    return {"op": 1, "graph": g, "counts": counts, "capacity": capacity}


def check_slots(c, offsets, words, positions, branches):
    want = S.slot_map(oracle_graph(c["graph"]), c["counts"], c["capacity"])
    for name, got, ref in zip(("offsets", "words", "positions", "branches"), (offsets, words, positions, branches), want):
        np.testing.assert_array_equal(got, ref, err_msg=name)


# Norm, rotation, append -----------------------------------------------------------------------------------

def qkv_case(rng, n, Hq, Hkv, D, dtype, rotary, interleaved=False, norm=(True, True), scale=1.0, far=5000, pad=0,
             in_place=False, eps=1e-6, x=None):
    """Rows as parts of one projection's with `pad` values behind each; words and positions with padding among them."""
    H = Hq + 2 * Hkv
    row = "f32" if dtype == "f32" else "bf16"
    rows = rng.standard_normal((n, H * D + pad)) * np.exp(rng.uniform(-3, 3, (n, 1)))
    if x is not None:
        rows[:, :] = x
    rows = stored(rows, row)
    num_pages = n // 10 + 2
    words = rng.permutation(16 * num_pages)[:n].astype(np.int32)
    positions = rng.integers(0, far, n).astype(np.int32)
    if n > 3:
        words[rng.integers(0, n)] = -1
        words[rng.integers(0, n)] = 16 * num_pages
        positions[rng.integers(0, n)] = -1
        positions[rng.integers(0, n)] = 0
    half = rotary // 2
    return {"op": 2, "rows": rows, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "dtype": dtype, "row": row, "words": words,
            "positions": positions, "num_pages": num_pages, "inv_freq": 10000.0 ** (-np.arange(half) / max(half, 1)),
            "interleaved": interleaved, "eps": eps, "scale": scale, "in_place": in_place,
            "weights": tuple((1 + 0.3 * rng.standard_normal(D)).astype(np.float32) if on else None for on in norm)}


def qkv_parts(c):
    """q, k, v [n, heads, D] as parts (views) of the rows."""
    Hq, Hkv, D, n = c["Hq"], c["Hkv"], c["D"], c["n"]
    body = c["rows"][:, :(Hq + 2 * Hkv) * D].reshape(n, -1, D) if n else np.zeros((0, Hq + 2 * Hkv, D), c["rows"].dtype)
    return body[:, :Hq], body[:, Hq:Hq + Hkv], body[:, Hq + Hkv:]


def qkv_bound(y, reach, dtype):
    """Sine and cosine are within 2^-22 (their argument in half turns is rounded to float32, the functions are within two
    steps), the weight folded in, two products and their sum add five half steps of float32, the norm (a sum of at
    most 128 squares in a tree of eleven additions, halved by the root, the root's step, two products) 2^-21: under
    2^-20 of the magnitudes together.  Then the rounding to the output's type."""
    tol = 2.0 ** -20 * reach
    return tol + (HALF["bf16"] * (np.abs(y) + tol) if dtype == "bf16" else 0.0)


def check_rows(got, x, c, weight, mask):
    """Rows got [n, H, D] (bits) of tokens `mask` against the oracle; returns the largest share of the bound."""
    y, reach = S.norm_rotate(values(x, c["row"]), c["positions"], c["inv_freq"], c["interleaved"], weight,
                             np.float32(c["eps"]), float(np.float32(c["scale"])))
    off = np.abs(values(got, c["row"]) - y)[mask]
    bound = qkv_bound(y, reach, c["row"])[mask]
    assert np.isfinite(off).all()
    worst = float((off / np.maximum(bound, 1e-300)).max()) if off.size else 0.0
    assert worst <= 1.0, worst
    return worst


def check_qkv(c, q_out, pool, fill):
    """q_out [n, Hq, D], pool [num_pages, Hkv, 2, 16, D] (bits) of a float32 or bf16 pool, both `fill` before."""
    q, k, v = qkv_parts(c)
    real = c["positions"] >= 0
    there = real & (c["words"] >= 0) & (c["words"] < 16 * c["num_pages"])
    check_rows(q_out, q, c, c["weights"][0], real)
    left = q[~real] if c["in_place"] else np.full_like(q[~real], fill)
    np.testing.assert_array_equal(q_out[~real], left)
    j = np.nonzero(there)[0]
    page, slot = c["words"][j] // 16, c["words"][j] % 16
    got = np.zeros_like(k)
    got[j] = pool[page, :, 0, slot]
    check_rows(got, k, c, c["weights"][1], there)
    np.testing.assert_array_equal(pool[page, :, 1, slot], v[j])
    rest = np.ones((c["num_pages"], 16), dtype=bool)
    rest[page, slot] = False
    assert (pool.transpose(0, 3, 1, 2, 4)[rest] == fill).all()


# Logit rules ----------------------------------------------------------------------------------------------

def logits_case(rng, g, rows, vocab, dtype="bf16", out_f32=False, rules="rfptbm", prompt=1, drafts=True, pad=0,
                in_place=False, bad=False, masks=3, biases=6):
    """`rules`: repetition, frequency, presence, temperature, biases, masks."""
    B = len(g["po"]) - 1
    c = {"op": 3, "graph": g, "vocab": vocab, "dtype": dtype, "out_f32": out_f32, "prompt": prompt, "in_place": in_place,
         "pad": pad}
    c["logits"] = stored(4 * rng.standard_normal((rows, vocab + pad)), dtype)
    c["ids"] = rng.integers(-1, min(vocab + 2, 30), 16 * g["num_pages"]).astype(np.int32)
    far = rng.integers(0, vocab, c["ids"].shape)
    c["ids"] = np.where(rng.random(c["ids"].shape) < 0.5, far, c["ids"]).astype(np.int32)
    c["branches"] = c["positions"] = None
    if drafts:
        c["branches"] = rng.integers(-1 if bad else 0, B + (2 if bad else 0), rows).astype(np.int32)
        c["positions"] = rng.integers(-1 if bad else 0, 150, rows).astype(np.int32)
    u = lambda lo, hi: rng.uniform(lo, hi, rows).astype(np.float32)  # noqa: E731
    c["rep"] = u(0.8, 2.0) if "r" in rules else None
    c["freq"] = u(-0.5, 1.0) if "f" in rules else None
    c["pres"] = u(-0.5, 1.0) if "p" in rules else None
    c["temp"] = u(0.3, 2.0) if "t" in rules else None
    c["bias"] = None
    if "b" in rules:
        n = rng.integers(0, biases + 1, rows)
        off = np.concatenate([[0], np.cumsum(n)]).astype(np.int64)
        tokens = [np.sort(rng.integers(-1, vocab + 1, k)) for k in n]       # (some twice, some outside)
        c["bias"] = (off, np.concatenate(tokens + [[]]).astype(np.int32),
                     rng.normal(0, 4, int(off[-1])).astype(np.float32))
    c["masks"] = None
    if "m" in rules:
        words = (vocab + 31) // 32 + int(rng.integers(0, 3))
        m = rng.integers(0, 2**32, (masks, words), dtype=np.uint32)
        m[0] = 0                                                             # forbids everything
        c["masks"] = (m, rng.integers(-1, masks + 1, rows).astype(np.int32))
    return c


def check_logits(c, out, before):
    """out [rows, vocab + pad] (bits) against the oracle; `before`: what it held."""
    g, V = oracle_graph(c["graph"]), c["vocab"]
    B = len(g.path_offsets) - 1
    wide = "f32" if c["out_f32"] or c["dtype"] == "f32" else "bf16"
    x = values(c["logits"], c["dtype"])
    np.testing.assert_array_equal(out[:, V:], before[:, V:])
    worst = 0.0
    for r in range(len(x)):
        b = r if c["branches"] is None else int(c["branches"][r])
        p = None if c["positions"] is None else int(c["positions"][r])
        if not 0 <= b < B or (p is not None and p < 0):
            np.testing.assert_array_equal(out[r], before[r])
            continue
        at = lambda a: None if a is None else a[r]  # noqa: E731
        bias = []
        if c["bias"] is not None:
            off, tokens, vals = c["bias"]
            bias = list(zip(tokens[off[r]:off[r + 1]].tolist(), vals[off[r]:off[r + 1]].tolist()))
        allowed = None
        if c["masks"] is not None and 0 <= c["masks"][1][r] < len(c["masks"][0]):
            m = c["masks"][0][c["masks"][1][r]]
            v = np.arange(V)
            allowed = (m[v // 32] >> (v % 32)) & 1 == 1
        counted = not (c["rep"] is None and c["freq"] is None and c["pres"] is None)
        seen = S.context(g, b, p, c["ids"], c["prompt"]) if counted else []
        z, size = S.logits_row(x[r, :V], seen, at(c["rep"]), at(c["freq"]), at(c["pres"]), at(c["temp"]), bias, allowed)
        got = values(out[r, :V], wide)
        inf = np.isinf(z)
        np.testing.assert_array_equal(np.isinf(got), inf)
        assert (got[inf] == z[inf]).all()
        # At most eight roundings of float32, each of at most the magnitudes together; then the output's.
        tol = 2.0 ** -21 * size[~inf]
        if wide == "bf16":
            tol = tol + HALF["bf16"] * (np.abs(z[~inf]) + tol)
        off = np.abs(got[~inf] - z[~inf])
        worst = max(worst, float((off / np.maximum(tol, 1e-300)).max()) if off.size else 0.0)
        assert worst <= 1.0, (r, worst)
    return worst
