"""Rounds of a long rollout in one pool, as the header describes them: append, attend, gather mass, choose, move
the tokens that stay with their mass, append again into pages that others gave up."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as C
from paper_2606_18954_amd import graphattn as G
from paper_2606_18954_amd import workloads as W

from cache_util import bits_of, check_attention, draw_q, mass_bound
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu

PATHS = [[0, 1], [0, 2], [0, 1, 3]]
DECAY = 0.9


def _slots(graph):
    """Slot words of every segment's tokens."""
    return [graph.seg_pages[graph.seg_page_offsets[s] + np.arange(n) // 16].astype(np.int64) * 16 + np.arange(n) % 16
            for s, n in enumerate(int(x) for x in graph.seg_len)]


def _place(rng, lens, free, P):
    """A graph of segments of these lengths on pages drawn from the free ones."""
    need = [-(-n // 16) for n in lens]
    pages = rng.permutation(free)[:sum(need)].astype(np.int32)
    off = np.concatenate([[0], np.cumsum(need)]).astype(np.int64)
    g = W.assemble_graph(lens, PATHS, 1)
    return W.RolloutGraph(np.array(lens, dtype=np.int32), off, pages, g.path_offsets, g.path_segs, P)


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("mxfp4", 28, 4, 128), ("mxfp4", 8, 2, 64), ("f32", 6, 3, 64)])
def test_masses_over_several_evictions(dtype, Hq, Hkv, D):
    require_gpu()
    say(f"[case] cycles {dtype} {Hq}/{Hkv}/{D}")
    rng = np.random.default_rng(41)
    lens = [90, 33, 64, 17]
    P = 3 * sum(-(-n // 16) for n in lens)
    p = G.make_params(Hq, Hkv, D, P, dtype)
    pool = G.empty_pool(p)
    pool.zero_()
    row = torch.float32 if dtype == "f32" else torch.bfloat16
    # (what a slot held before is no token's: pages are taken up again and again)
    mass = torch.full((16 * P,), 99.0, device="cuda")
    gathered, ids = {}, [[] for _ in lens]               # mass by token, tokens by segment

    def words_of(parts):
        return torch.from_numpy(np.concatenate(parts)).int().cuda()

    def append(parts):
        words = words_of(parts)
        kv = draw_q(rng, 2 * words.numel(), Hkv, D, "f32").to(row).cuda()
        G.kv_append(pool, kv[:words.numel()].contiguous(), kv[words.numel():].contiguous(), words, p)
        mass[words.long()] = 0

    g = _place(rng, lens, np.arange(P), P)
    append(_slots(g))
    for s, n in enumerate(lens):
        ids[s] = [(0, s, t) for t in range(n)]
        gathered.update({i: 0.0 for i in ids[s]})
    for turn in range(4):
        at = _slots(g)
        torch.cuda.synchronize()
        vals = C.pool_values(pool.cpu().numpy()) if dtype == "mxfp4" else bits_of(pool)
        q = draw_q(rng, 3, Hq, D, "f32" if dtype == "f32" else "bf16")
        out, lse = torch.empty((3, Hq, D), dtype=row, device="cuda"), torch.empty((3, Hq), device="cuda")
        with G.Plan(G.HostGraph.from_graph(g), p) as pl:
            pl.run(q.cuda(), pool, out, lse)
            pl.run_mass(q.cuda(), pool, lse, mass, mass, DECAY)
            torch.cuda.synchronize()
        check_attention(f"turn {turn}", out, lse, q, vals, g, Hq, Hkv)
        before = np.zeros(16 * P)
        for s, words in enumerate(at):
            before[words] = [gathered[i] for i in ids[s]]
        l64 = bits_of(lse)
        ref = C.mass(bits_of(q), vals, g, l64, Hq, Hkv, before, DECAY)
        bound = mass_bound(q, vals, g, l64, Hq, Hkv, ref, DECAY, before)
        got = bits_of(mass)
        for s, words in enumerate(at):
            assert (np.abs(got[words] - ref[words]) <= bound[words]).all(), (turn, s)
            gathered.update(zip(ids[s], got[words]))     # (the next turn starts from what was gathered)
        # A third of every segment goes; the others move to pages that are free.
        keep = [max(1, 2 * n // 3) for n in lens]
        with G.Evict(G.HostGraph.from_graph(g), keep, 1, 2, P) as ev:
            pos, src = ev.select(mass)
            torch.cuda.synchronize()
        rp, rw = C.evict_select(got, g.seg_len, g.seg_page_offsets, g.seg_pages, keep, 1, 2)
        assert np.array_equal(pos.cpu().numpy(), rp) and np.array_equal(src.cpu().numpy(), rw)
        grown = [k + int(rng.integers(0, 30)) for k in keep]
        new = _place(rng, grown, np.setdiff1d(np.arange(P), g.seg_pages), P)
        to = _slots(new)
        dst = words_of([w[:k] for w, k in zip(to, keep)])
        G.kv_copy(pool, src, dst, p)
        mass[dst.long()] = mass[src.long()]
        start = np.concatenate([[0], np.cumsum(keep)])
        ids = [[ids[s][t] for t in rp[start[s]:start[s + 1]]] for s in range(len(lens))]
        append([w[k:] for w, k in zip(to, keep)])
        for s, (k, n) in enumerate(zip(keep, grown)):
            ids[s] += [(turn + 1, s, t) for t in range(k, n)]
            gathered.update({i: 0.0 for i in ids[s][k:]})
        lens, g = grown, new
