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
