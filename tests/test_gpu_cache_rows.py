"""Rows of the attention mass whose lse is no number, on the GPU."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as C
from paper_2606_18954_amd import graphattn as G
from paper_2606_18954_amd import workloads as W

from cache_util import bits_of, draw_q, mass_bound, poison_unused, random_pool
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [20, 33, 200, 1100])
@pytest.mark.parametrize("D", [64, 128])
def test_a_row_without_an_lse_says_nothing_of_later_tokens(n, D):
    """A prompt's prefill (few rows, many, more than 4096 a kv-head): a row whose lse is NaN makes the tokens
    that it sees NaN, and leaves those behind it alone."""
    require_gpu()
    say(f"[case] NaN in a prefill of {n} tokens, {D} channels")
    Hq, Hkv, at = 4, 1, n // 2 + 3
    rng = np.random.default_rng(n + D)
    g = W.assemble_graph([n], [[0]], 4, slack_pages=1)
    raw = poison_unused(random_pool(rng, g.num_pages, Hkv, D, -2, 1), g)
    vals, q = C.pool_values(raw), draw_q(rng, n, Hq, D)
    lse = C.attention(bits_of(q), vals, g, Hq, Hkv, [n])[1].astype(np.float32)
    lse[1, 2] = math.inf
    p = G.make_params(Hq, Hkv, D, g.num_pages, "mxfp4")
    mass_in = rng.uniform(0, 3, 16 * g.num_pages).astype(np.float32)
    given = lse.copy()
    given[at, 1] = math.nan
    out = torch.full((16 * g.num_pages,), -5.0, device="cuda")
    with G.Plan(G.HostGraph.from_graph(g), p, query_counts=[n]) as pl:
        pl.run_mass(q.cuda(), torch.from_numpy(raw).cuda(), torch.from_numpy(given).cuda(), out,
                    torch.from_numpy(mass_in).cuda(), 0.75)
        torch.cuda.synchronize()
    # (without that row and head: an infinite lse counts for nothing)
    lse[at, 1] = math.inf
    ref = C.mass(bits_of(q), vals, g, lse.astype(float), Hq, Hkv, mass_in, 0.75, [n])
    bound = mass_bound(q, vals, g, lse, Hq, Hkv, ref, 0.75, mass_in, [n])
    got, t = bits_of(out), np.arange(n)
    slots = g.seg_pages[t // 16].astype(np.int64) * 16 + t % 16
    assert np.isnan(got[slots[:at + 1]]).all()
    later = slots[at + 1:]
    assert (np.abs(got[later] - ref[later]) <= bound[later]).all()
    rest = np.setdiff1d(np.arange(16 * g.num_pages), slots)
    assert (got[rest] == -5).all()


@pytest.mark.parametrize("counts", [None, [1, 40, 3]])
def test_a_grown_plan_has_a_fresh_plans_bits(counts):
    """Mass of a plan that was given new lengths and of one created with them: small graphs, taken in the same
    parts, have the same bits."""
    require_gpu()
    say(f"[case] mass of a grown and a fresh plan {counts}")
    rng = np.random.default_rng(59)
    Hq, Hkv, D = 8, 2, 64
    lens, paths = [700, 90, 130], [[0, 1], [0, 2], [0]]
    if counts:
        lens, paths = W.with_new_steps(lens, paths, counts)
    g = W.assemble_graph(lens, paths, 6, slack_pages=2)
    rows = sum(counts) if counts else 3
    raw = poison_unused(random_pool(rng, g.num_pages, Hkv, D, -2, 1), g)
    vals, q = C.pool_values(raw), draw_q(rng, rows, Hq, D)
    lse = torch.from_numpy(C.attention(bits_of(q), vals, g, Hq, Hkv, counts)[1].astype(np.float32)).cuda()
    p = G.make_params(Hq, Hkv, D, g.num_pages, "mxfp4")
    short = [max(1, n // 3) for n in lens[:3]] + lens[3:]
    got = []
    for start in (lens, short):
        out = torch.full((16 * g.num_pages,), -5.0, device="cuda")
        with G.Plan(G.HostGraph(start, g.seg_page_offsets, g.seg_pages, g.path_offsets, g.path_segs), p,
                    query_counts=counts) as pl:
            if start is short:
                pl.schedule()
                pl.run_mass(q.cuda(), torch.from_numpy(raw).cuda(), lse, torch.zeros_like(out))
                pl.set_lengths(lens)
            pl.run_mass(q.cuda(), torch.from_numpy(raw).cuda(), lse, out)
            torch.cuda.synchronize()
        got.append(out)
    assert torch.equal(got[0], got[1])


@pytest.mark.parametrize("step", [3, 40, 300])
@pytest.mark.parametrize("D", [64, 128])
def test_keys_behind_a_query_may_be_anything(step, D):
    """NaN in the keys of each branch's last token: attention and mass of the rows before it are as without,
    with few rows a page and many."""
    require_gpu()
    say(f"[case] NaN keys behind {step} queries, {D} channels")
    rng = np.random.default_rng(step + D)
    Hq, Hkv = 12, 2
    counts = [step, step - 1, max(1, step // 2)]
    lens, paths = W.with_new_steps([150, 33], [[0], [0, 1], [0]], [step, step, step])
    g = W.assemble_graph(lens, paths, 6, slack_pages=1)
    raw = poison_unused(random_pool(rng, g.num_pages, Hkv, D, -2, 1), g)
    vals, q = C.pool_values(raw), draw_q(rng, sum(counts), Hq, D)
    bad = raw.copy()
    for s in range(2, 5):
        t = lens[s] - 1
        page = int(g.seg_pages[g.seg_page_offsets[s] + t // 16])
        for c in range(0, D, 32):
            bad[page, :, C.scale_place(t % 16, c, D, False)] = 255
    last = np.cumsum(counts) - 1                           # the rows that see those tokens
    rest = np.setdiff1d(np.arange(sum(counts)), last)
    oo, ol, _, _ = C.attention(bits_of(q), vals, g, Hq, Hkv, counts)
    given = ol.astype(np.float32)
    given[last] = math.inf                                 # (count for nothing)
    p = G.make_params(Hq, Hkv, D, g.num_pages, "mxfp4")
    got = []
    for pool in (raw, bad):
        out = torch.zeros(sum(counts), Hq, D, dtype=torch.bfloat16, device="cuda")
        lse = torch.zeros(sum(counts), Hq, device="cuda")
        mass = torch.full((16 * g.num_pages,), -5.0, device="cuda")
        with G.Plan(G.HostGraph.from_graph(g), p, query_counts=counts) as pl:
            pl.run(q.cuda(), torch.from_numpy(pool).cuda(), out, lse)
            pl.run_mass(q.cuda(), torch.from_numpy(pool).cuda(), torch.from_numpy(given).cuda(), mass)
            torch.cuda.synchronize()
        got.append((bits_of(out)[rest], bits_of(lse)[rest], bits_of(mass)))
    assert np.isfinite(got[0][0]).all()
    assert np.array_equal(got[0][0], got[1][0]) and np.array_equal(got[0][1], got[1][1])
    seen = np.array([int(g.seg_pages[g.seg_page_offsets[s] + (lens[s] - 1) // 16]) * 16 + (lens[s] - 1) % 16
                     for s in range(2, 5)])
    others = np.setdiff1d(np.arange(16 * g.num_pages), seen)
    assert np.array_equal(got[0][2][others], got[1][2][others])
    assert np.isnan(got[1][2][seen]).all()
