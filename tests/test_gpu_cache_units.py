"""MXFP4 attention and attention mass in units as large as real steps have them: chunks of 24 to 128 pages, whose
loops come round many times (small graphs are cut into chunks of 4), against the float64 oracle on sampled rows
and slots.

Attention: many segments that list the same few pages are much work in little memory.  Mass: pages of their own,
small ones (one kv-head of 64 channels), and an lse that is given, so that a slot's mass needs only the rows that
see its segment.  Each test asserts the size that it is about.
"""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as C
from paper_2606_18954_amd import graphattn as G
from paper_2606_18954_amd import workloads as W

from cache_util import bits_of, check_attention, draw_q, random_pool
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu

SHARED = 300                                              # full pages that every segment lists


def _trunks(rng, trunks, step, Hkv, D):
    """Trunks (pages, branches, tokens on the last page) with a segment of `step` tokens a branch; the raw pool."""
    pages, off, lens, paths = [], [0], [], []
    last = SHARED

    def segment(n, tail):
        nonlocal last
        pages.extend(rng.integers(0, SHARED, n - 1))
        pages.append(last)
        last += 1
        off.append(len(pages))
        lens.append(16 * (n - 1) + tail)
        return len(lens) - 1
    for n, branches, tail in trunks:
        t = segment(n, tail)
        paths += [[t, segment((step + 15) // 16, (step - 1) % 16 + 1)] for _ in range(branches)]
    raw = random_pool(rng, last, Hkv, D, -2, 1)
    for s, n in enumerate(lens):                          # (behind a segment's end: NaN)
        page = int(pages[off[s + 1] - 1])
        for t in range((n - 1) % 16 + 1, 16):
            for value in (False, True):
                for c in range(0, D, 32):
                    raw[page, :, C.scale_place(t, c, D, value)] = 255
    g = W.RolloutGraph(np.array(lens, dtype=np.int32), np.array(off, dtype=np.int64), np.array(pages, dtype=np.int32),
                       np.cumsum([0] + [len(p) for p in paths]).astype(np.int64),
                       np.concatenate(paths).astype(np.int32), last)
    return g, raw


def _attend(tag, trunks, step, Hq, Hkv, D, chunk, queries, wgs):
    require_gpu()
    say(f"[case] {tag} {Hq}/{Hkv}/{D}")
    rng = np.random.default_rng(len(tag) + Hq + D)
    g, raw = _trunks(rng, trunks, step, Hkv, D)
    counts = [queries] * g.num_branches if queries else None
    rows = g.num_branches * (queries or 1)
    q = draw_q(rng, rows, Hq, D)
    pool, qd = torch.from_numpy(raw).cuda(), q.cuda()
    p = G.make_params(Hq, Hkv, D, g.num_pages, "mxfp4")
    with G.Plan(G.HostGraph.from_graph(g), p, query_counts=counts) as pl:
        info = pl.info()
        assert info.chunk_pages == chunk and info.workgroups_per_cu == wgs, (info.chunk_pages, info.workgroups_per_cu)
        got = []
        for _ in range(2):                                # (the second from re-armed work streams)
            out = torch.full((rows + 1, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
            lse = torch.full((rows + 1, Hq), 7.0, device="cuda")
            pl.run(qd, pool, out, lse)
            torch.cuda.synchronize()
            assert (out[-1] == 7).all() and (lse[-1] == 7).all()
            got.append((out, lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    # The first and last row of the first and the last branch.
    n = queries or 1
    sample = sorted({b * n + i for b in (0, g.num_branches - 1) for i in (0, n - 1)})
    check_attention(tag, out, lse, q, C.pool_values(raw), g, Hq, Hkv, counts, sample)


# Per case: trunks, heads, the chunk, workgroups per CU (a row tile a wave: one more than two a wave).
DECODE = {
    "one branch a trunk, longest chunks": ([(4200, 1, 5)] * 12, 28, 4, 128, 128, 3),
    "one branch a trunk, odd chunks": ([(1183, 1, 16)] * 12, 28, 4, 128, 37, 3),
    "two row tiles, two groups of waves": ([(1500, 2, 1)] * 8, 40, 4, 128, 32, 3),
    "some trunks of three and five row tiles": ([(1500, 1, 9)] * 10 + [(1400, 6, 3), (1111, 10, 16)], 28, 4, 128, 46, 3),
    "two row tiles a wave, one group": ([(1500, 2, 15)] * 8 + [(1500, 4, 15)], 64, 4, 128, 36, 2),
    "two row tiles a wave, two groups": ([(1500, 8, 2)] * 8, 28, 4, 128, 32, 2),
    "two row tiles a wave, four groups": ([(1500, 12, 2)] * 8, 28, 4, 128, 32, 2),
    "two row blocks": ([(1500, 19, 8)] * 8, 28, 4, 128, 32, 2),
    "64 channels": ([(1500, 1, 7)] * 12, 16, 4, 64, 47, 4),
    "64 channels, three row tiles and eight": ([(1500, 10, 7), (1499, 30, 16)] * 6, 16, 4, 64, 48, 3),
}


@pytest.mark.parametrize("name", DECODE)
def test_decode_in_large_units(name):
    trunks, Hq, Hkv, D, chunk, wgs = DECODE[name]
    _attend(name, trunks, 9, Hq, Hkv, D, chunk, 0, wgs)


# With queries: few rows a page on the decode kernel's causal form, many on the multi-query kernel.
EXTEND = {
    "two queries": ([(1500, 1, 5)] * 12, 28, 4, 128, 36, 2, 3),
    "nine queries a branch, two branches": ([(2500, 2, 5)] * 12, 14, 2, 64, 30, 9, 3),
    "many rows": ([(1150, 3, 5)] * 4, 28, 4, 128, 64, 37, 2),
    "many rows, an odd number of pairs": ([(1230, 2, 16)] * 4, 28, 4, 128, 49, 40, 2),
    "many rows, 64 channels": ([(1001, 9, 5)] * 4, 16, 4, 64, 95, 40, 2),
    "many rows, longest chunks": ([(900, 6, 5)] * 4, 28, 4, 128, 128, 60, 2),
}


@pytest.mark.parametrize("name", EXTEND)
def test_extend_in_large_units(name):
    trunks, Hq, Hkv, D, chunk, queries, wgs = EXTEND[name]
    _attend(name, trunks, queries + 3, Hq, Hkv, D, chunk, queries, wgs)


def _parts(pages, rows, cost):
    pairs = np.minimum((rows + 31) // 32, cost)
    return np.minimum((pages * pairs + cost - 1) // cost, (pages + 3) // 4)


def _cost(pages, rows):
    """What a workgroup takes, as the plan chooses it: pages times pairs of row tiles."""
    cost = 128
    while cost > 4 and _parts(pages, rows, cost).sum() < 12 * 256:
        cost //= 2
    return cost


# Chains (pages, branches), heads, type, what a workgroup takes, pages of the largest part.
MASS = {
    "few rows, parts of 128 pages": ([(32900, 1, 9)] * 12, 4, 1, 64, "mxfp4", 128, 128),
    "few rows, parts of 8 pages": ([(2200, 1, 9)] * 12, 4, 1, 64, "mxfp4", 8, 8),
    "four kv-heads, parts of 128 pages": ([(33100, 1, 3)] * 12, 8, 4, 64, "mxfp4", 128, 128),
    "three pairs of row tiles, parts of 43 pages": ([(11200, 5, 16)] * 12, 16, 1, 64, "mxfp4", 128, 43),
    "many rows, parts of 26 pages": ([(7000, 10, 16)] * 12, 16, 1, 64, "mxfp4", 128, 26),
    "many rows of two kv-heads, 128 channels": ([(7000, 10, 2)] * 12, 32, 2, 128, "mxfp4", 128, 26),
    "bf16": ([(16500, 2, 9)] * 12, 24, 1, 64, "bf16", 128, 64),
    "f32": ([(11200, 5, 16)] * 6 + [(2800, 20, 1)] * 6, 16, 1, 64, "f32", 64, 22),
}


@pytest.mark.parametrize("name", MASS)
def test_mass_in_large_parts(name):
    chains, Hq, Hkv, D, dtype, cost, most = MASS[name]
    require_gpu()
    say(f"[case] {name} {Hq}/{Hkv}/{D} {dtype}")
    rng = np.random.default_rng(len(name))
    pages = np.array([n for n, _, _ in chains])
    rows = np.array([b * Hq // Hkv for _, b, _ in chains])
    # (a branch's own segment: one page, its rows the group's)
    own = int(sum(b for _, b, _ in chains))
    all_pages = np.concatenate([np.where(np.array([b for _, b, _ in chains]) == 1, pages + 1, pages),
                                np.ones(int(sum(b for _, b, _ in chains if b > 1)), dtype=int)])
    all_rows = np.concatenate([rows, np.full(len(all_pages) - len(rows), Hq // Hkv)])
    assert _cost(all_pages, all_rows) == cost
    parts = _parts(all_pages, all_rows, cost)
    assert int(((all_pages + parts - 1) // parts).max()) == most
    lens, paths = [], []
    for n, branches, tail in chains:
        lens.append(16 * (n - 1) + tail)
        t = len(lens) - 1
        for _ in range(branches):
            paths.append([t, len(lens)])
            lens.append(int(rng.integers(1, 17)))
    g = W.assemble_graph(lens, paths, 5, slack_pages=3)
    B, P = len(paths), g.num_pages
    assert B == own
    gen = torch.Generator(device="cuda").manual_seed(7)
    if dtype == "mxfp4":
        pool = torch.randint(0, 256, (P, Hkv, 17 * D), generator=gen, device="cuda", dtype=torch.uint8)
        pool[:, :, 16 * D:] = torch.randint(125, 127, (P, Hkv, D), generator=gen, device="cuda", dtype=torch.uint8)
    else:
        pool = torch.randn(P, Hkv, 2, 16, D, generator=gen, device="cuda")
        pool = pool.bfloat16() if dtype == "bf16" else pool
    q = draw_q(rng, B, Hq, D, "f32" if dtype == "f32" else "bf16")
    lse = rng.uniform(3, 6, (B, Hq)).astype(np.float32)
    mass_in = torch.rand(16 * P, generator=gen, device="cuda")
    out = torch.full((16 * P,), -5.0, device="cuda")
    p = G.make_params(Hq, Hkv, D, P, dtype)
    with G.Plan(G.HostGraph.from_graph(g), p) as pl:
        pl.run_mass(q.cuda(), pool, torch.from_numpy(lse).cuda(), out, mass_in, 0.5)
        torch.cuda.synchronize()
    used = torch.zeros(16 * P, dtype=torch.bool, device="cuda")
    q64, l64, got, before = bits_of(q), lse.astype(float), bits_of(out), bits_of(mass_in)
    for s, n in enumerate(lens):
        pg = torch.from_numpy(g.seg_pages[g.seg_page_offsets[s]:g.seg_page_offsets[s + 1]].astype(np.int64)).cuda()
        slots = (pg[:, None] * 16 + torch.arange(16, device="cuda")).flatten()[:n]
        used[slots] = True
        # The first, middle and last slots of some segments, in float64.
        if n > 16 and s not in (0, chains[0][1] + 1, max(i for i, m in enumerate(lens) if m > 16)):
            continue
        if n <= 16 and s > 40:
            continue
        see = [b for b, path in enumerate(paths) if s in path]
        slot = slots.cpu().numpy()
        for a in sorted({0, max(0, n // 2 - 4096), max(0, n - 8192)}):
            w = slot[a:a + 8192]
            first, where = np.unique(w // 16, return_inverse=True)
            kv = pool[torch.from_numpy(first).cuda()].cpu()
            vals = C.pool_values(kv.numpy()) if dtype == "mxfp4" else bits_of(kv)
            k = vals[where, :, 0, w % 16]                 # [n, Hkv, D]
            ref, bound = 0.5 * before[w], 2.0 ** -22 * before[w]
            for b in see:
                for h in range(Hq):
                    kh = k[:, h // (Hq // Hkv)]
                    e = np.exp(kh @ q64[b, h] / np.sqrt(D) - l64[b, h])
                    reach = np.abs(kh) @ np.abs(q64[b, h]) / np.sqrt(D)
                    # (a score's float32 sum of D terms; a few steps of score and lse in the log2 domain; sums)
                    rel = (D + 8) * 2.0 ** -24 * reach + 2.0 ** -22 * (1 + reach + abs(l64[b, h])) + 2.0 ** -16
                    ref, bound = ref + e, bound + rel * e
            off = np.abs(got[w] - ref) / (bound + 2.0 ** -22 * np.abs(ref))
            assert off.max() <= 1.0, (s, a, float(off.max()))
    assert bool((out[~used] == -5).all())
