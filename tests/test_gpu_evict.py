"""Attention mass and eviction on the GPU against the float64 oracle, alone and in a run of the whole
cycle: append, attend, gather mass, choose, move, attend again."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as C
from paper_2606_18954_amd import graphattn as G
from paper_2606_18954_amd import workloads as W

from cache_util import (bits_of, check_attention, draw_q, mass_bound, poison_unused, random_pool)
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


def _pool(rng, graph, Hkv, D, dtype):
    """(device pool, float64 values), NaN in every slot without a token."""
    if dtype == "mxfp4":
        raw = poison_unused(random_pool(rng, graph.num_pages, Hkv, D, -2, 1), graph)
        return torch.from_numpy(raw).cuda(), C.pool_values(raw)
    x = rng.standard_normal((graph.num_pages, Hkv, 2, 16, D)).astype(np.float32)
    used = np.zeros(16 * graph.num_pages, dtype=bool)
    for s in range(graph.num_segments):
        for t in range(int(graph.seg_len[s])):
            used[16 * int(graph.seg_pages[graph.seg_page_offsets[s] + t // 16]) + t % 16] = True
    for w in np.nonzero(~used)[0]:
        x[w // 16, :, :, w % 16] = np.nan
    t = torch.from_numpy(x)
    t = t.bfloat16() if dtype == "bf16" else t
    return t.cuda(), bits_of(t)


def _check_mass(rng, graph, Hq, Hkv, D, dtype, counts=None, decay=0.75, alias=False, plan=None):
    rows = graph.num_branches if counts is None else int(sum(counts))
    pool, vals = _pool(rng, graph, Hkv, D, dtype)
    q = draw_q(rng, rows, Hq, D, "f32" if dtype == "f32" else "bf16")
    lse = C.attention(bits_of(q), vals, graph, Hq, Hkv, counts)[1].astype(np.float32)
    mass_in = rng.uniform(0, 3, 16 * graph.num_pages).astype(np.float32)
    p = G.make_params(Hq, Hkv, D, graph.num_pages, dtype)
    min_ = torch.from_numpy(mass_in).cuda()
    out = min_ if alias else torch.full_like(min_, -5.0)
    with G.Plan(G.HostGraph.from_graph(graph), p, query_counts=counts) as pl:
        pl.run_mass(q.cuda(), pool, torch.from_numpy(lse).cuda(), out, min_, decay)
        torch.cuda.synchronize()
    ref = C.mass(bits_of(q), vals, graph, lse.astype(float), Hq, Hkv, mass_in, decay, counts)
    got = bits_of(out)
    bound = mass_bound(q, vals, graph, lse, Hq, Hkv, ref, decay, mass_in, counts)
    live = np.isfinite(ref)
    off = np.abs(got - ref)[live] / bound[live]
    say(f"[parity] mass {Hq}/{Hkv}/{D} {dtype}: {off.max():.3f} of its bound")
    assert off.max() <= 1.0
    assert np.array_equal(got[~live], mass_in[~live] if alias else np.full((~live).sum(), -5.0))


HEADS = [(28, 4, 128), (8, 2, 64), (5, 1, 128), (6, 6, 64), (24, 3, 128), (40, 8, 64)]


@pytest.mark.parametrize("dtype", ["mxfp4", "bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_mass_of_a_decode_step(Hq, Hkv, D, dtype):
    require_gpu()
    say(f"[case] mass {Hq}/{Hkv}/{D} {dtype}")
    rng = np.random.default_rng(Hq + D)
    g = W.random_graph(rng, 8, 17, 150, 4, slack_pages=3, seed=2)
    _check_mass(rng, g, Hq, Hkv, D, dtype, alias=Hq == 8)


@pytest.mark.parametrize("dtype", ["mxfp4", "bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS[:3])
def test_mass_of_multi_query_steps(Hq, Hkv, D, dtype):
    require_gpu()
    rng = np.random.default_rng(Hq + D)
    step = [int(n) for n in rng.integers(1, 90, 5)]
    lens, paths = W.with_new_steps([130, 40], [[0], [0, 1], [1], [0], [0, 1]], step)
    counts = [int(rng.integers(1, n + 1)) for n in step]
    say(f"[case] mass of {counts} queries {Hq}/{Hkv}/{D} {dtype}")
    g = W.assemble_graph(lens, paths, 6, slack_pages=2)
    _check_mass(rng, g, Hq, Hkv, D, dtype, counts)


@pytest.mark.parametrize("lens", [[1], [16], [17], [64], [65], [130]])
@pytest.mark.parametrize("dtype", ["mxfp4", "f32"])
def test_mass_of_a_prefill(lens, dtype):
    require_gpu()
    say(f"[case] mass of a prefill {lens} {dtype}")
    rng = np.random.default_rng(lens[0])
    g = W.assemble_graph(lens, [[i] for i in range(len(lens))], 4, slack_pages=1)
    _check_mass(rng, g, 7, 1, 128, dtype, lens)


def test_mass_of_many_rows():
    """90 branches of 7 rows a kv-head on one segment: five row blocks."""
    require_gpu()
    say("[case] mass of 90 branches")
    rng = np.random.default_rng(3)
    g = W.assemble_graph([100] + [3] * 90, [[0, 1 + b] for b in range(90)], 5)
    _check_mass(rng, g, 14, 2, 64, "bf16")


@pytest.mark.parametrize("Hq,Hkv,D,dtype", [(16, 2, 64, "mxfp4"), (7, 1, 128, "bf16"), (24, 3, 64, "f32"),
                                             (28, 4, 128, "mxfp4"), (8, 1, 128, "f32")])
def test_mass_of_a_great_many_rows(Hq, Hkv, D, dtype):
    """One plan with a chain of more than 4096 rows a kv-head (a prompt's prefill: workgroups of sixteen waves),
    one of a few hundred (a shared prefix of several branches) and one of few."""
    require_gpu()
    say(f"[case] mass of a great many rows {Hq}/{Hkv}/{D} {dtype}")
    rng = np.random.default_rng(Hq)
    n = 4100 * Hkv // Hq + 7
    lens, paths = [n, 75, 40, 40, 90], [[0], [1, 2], [1, 3], [4]]
    counts = [n, 40, 33, 2]
    g = W.assemble_graph(lens, paths, 6, slack_pages=2)
    assert n * Hq // Hkv > 4096 and 73 * Hq // Hkv > 128 and 2 * Hq // Hkv < 128
    _check_mass(rng, g, Hq, Hkv, D, dtype, counts)


def test_rows_without_weight_count_for_nothing_and_no_mass_in():
    require_gpu()
    say("[case] infinite lse")
    rng = np.random.default_rng(6)
    g = W.assemble_graph([40, 9], [[0, 1], [0]], 5, slack_pages=1)
    pool, vals = _pool(rng, g, 2, 64, "bf16")
    q = draw_q(rng, 2, 4, 64)
    lse = C.attention(bits_of(q), vals, g, 4, 2)[1].astype(np.float32)
    lse[0, 1], lse[1, 3] = math.inf, -math.inf
    p = G.make_params(4, 2, 64, g.num_pages, "bf16")
    out = torch.full((16 * g.num_pages,), -5.0, device="cuda")
    with G.Plan(G.HostGraph.from_graph(g), p) as pl:
        pl.run_mass(q.cuda(), pool, torch.from_numpy(lse).cuda(), out, None, math.pi)
        torch.cuda.synchronize()
    zero = np.zeros(16 * g.num_pages, dtype=np.float32)
    ref = C.mass(bits_of(q), vals, g, lse.astype(float), 4, 2, zero, 1.0)
    live = np.isfinite(ref)
    off = np.abs(bits_of(out) - ref) / mass_bound(q, vals, g, lse, 4, 2, ref, 0.0, zero)
    assert off[live].max() <= 1.0 and (bits_of(out)[~live] == -5).all()


def test_mass_refusals():
    require_gpu()
    lib = G.load_library()
    p = G.make_params(4, 2, 64, 4, "bf16")
    shared = G.HostGraph([20, 20], [0, 2, 4], [0, 1, 1, 2], [0, 1, 2], [0, 1])
    buf = torch.zeros(1 << 16, device="cuda")
    ptr = ctypes.c_void_p(buf.data_ptr())
    with G.Plan(shared, p) as pl:
        assert lib.graphattn_run_mass(pl.handle, ptr, ptr, ptr, None, 1.0, ptr, None) == G.GA_EINVAL
        assert "same page" in G.last_error()
    # A page that comes twice only in a segment on no path is harmless.
    with G.Plan(G.HostGraph([20, 20], [0, 2, 4], [0, 1, 1, 2], [0, 1], [0]), p) as pl:
        def call(*a):
            return lib.graphattn_run_mass(pl.handle, *a)
        odd, mis = ctypes.c_void_p(buf.data_ptr() + 8), ctypes.c_void_p(buf.data_ptr() + 2)
        for a in ((None, ptr, ptr, None, 1.0, ptr, None), (ptr, None, ptr, None, 1.0, ptr, None),
                  (ptr, ptr, None, None, 1.0, ptr, None), (ptr, ptr, ptr, None, 1.0, None, None),
                  (odd, ptr, ptr, None, 1.0, ptr, None), (ptr, odd, ptr, None, 1.0, ptr, None),
                  (ptr, ptr, mis, None, 1.0, ptr, None), (ptr, ptr, ptr, mis, 1.0, ptr, None),
                  (ptr, ptr, ptr, None, math.nan, ptr, None),
                  (ptr, ptr, ptr, None, math.inf, ptr, None)):
            assert call(*a) == G.GA_EINVAL and G.last_error()
        with pytest.raises(ValueError):
            pl.run_mass(buf, buf, buf, torch.zeros(63, device="cuda"))
        # (1 row of 4 heads x 64, 4 pages)
        for q, lse, out, into in ((buf[:255], buf, buf[:64], None), (buf, buf[:3], buf[:64], None),
                                  (buf, buf.double(), buf[:64], None), (buf, buf, buf[:64].double(), None),
                                  (buf, buf, buf[:64], buf[:64].half())):
            with pytest.raises(ValueError):
                pl.run_mass(q, buf, lse, out, into)


# ----------------------------------------------------------------------------------------------
# Eviction
# ----------------------------------------------------------------------------------------------

def _select(mass, graph, keep, first, recent):
    with G.Evict(G.HostGraph.from_graph(graph), keep, first, recent, graph.num_pages) as ev:
        pos, words = ev.select(torch.from_numpy(mass).cuda())
        torch.cuda.synchronize()
        assert list(ev.offsets) == [0] + list(np.cumsum(keep))
        return pos.cpu().numpy(), words.cpu().numpy()


def _check_select(mass, graph, keep, first, recent):
    pos, words = _select(mass, graph, keep, first, recent)
    rp, rw = C.evict_select(mass, graph.seg_len, graph.seg_page_offsets, graph.seg_pages, keep,
                            first, recent)
    assert np.array_equal(pos, rp) and np.array_equal(words, rw)


def _masses(rng, kind, n):
    if kind == "spread":
        return np.exp(3 * rng.standard_normal(n)).astype(np.float32)
    if kind == "ties":
        return rng.integers(0, 3, n).astype(np.float32)
    if kind == "equal":
        return np.full(n, 0.25, dtype=np.float32)
    if kind == "mostly zero":
        return np.where(rng.random(n) < 0.97, 0.0, rng.random(n)).astype(np.float32)
    if kind == "uneven":                                 # a dense run of keys, far from a few others
        x = (1 + 2.0 ** -23 * rng.integers(0, 5000, n)).astype(np.float32)
        x[rng.random(n) < 0.02] = 1e-40
        x[rng.random(n) < 0.02] = 1e38
        return x
    x = rng.standard_normal(n).astype(np.float32)        # signs, zeros of both signs, NaN, infinities
    x[rng.random(n) < 0.2] = 0.0
    x[rng.random(n) < 0.2] = -0.0
    x[rng.random(n) < 0.1] = np.nan
    x[rng.random(n) < 0.05] = np.inf
    x[rng.random(n) < 0.05] = -np.inf
    x[rng.random(n) < 0.02] = -np.nan
    return x


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "special", "mostly zero", "uneven"])
@pytest.mark.parametrize("lens", [[1], [2, 16, 17, 64, 65, 1023, 1024], [1025, 2048, 5],
                                  [16383, 16384, 1000], [16385, 40, 40000, 1500]])
def test_select(lens, kind):
    require_gpu()
    say(f"[case] select {lens} {kind}")
    rng = np.random.default_rng(len(lens) + len(kind))
    g = W.assemble_graph(lens, [list(range(len(lens)))], 4, slack_pages=2)
    mass = _masses(rng, kind, 16 * g.num_pages)
    n = np.array(lens)
    for first, recent, keep in ((0, 0, (n * 0.5).astype(int)), (4, 9, np.minimum(n, n // 3 + 13)),
                                (0, 0, n), (0, 0, 0 * n), (0, 0, np.minimum(n, 1)), (0, 0, n - 1),
                                (3, 0, np.minimum(n, 3)), (0, 7, np.minimum(n, 7))):
        _check_select(mass, g, keep, first, recent)


def test_two_selections_at_once():
    """One handle, two streams and two masses: nothing is shared but the tables."""
    require_gpu()
    say("[case] two selections at once")
    rng = np.random.default_rng(5)
    lens = [700, 3000, 64, 20000, 1024]
    g = W.assemble_graph(lens, [list(range(5))], 4)
    mass = [_masses(rng, kind, 16 * g.num_pages) for kind in ("spread", "special")]
    keep = [n // 2 for n in lens]
    dev = [torch.from_numpy(m).cuda() for m in mass]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    with G.Evict(G.HostGraph.from_graph(g), keep, 2, 3, g.num_pages) as ev:
        out = [[torch.zeros(ev.total, dtype=torch.int32, device="cuda") for _ in range(2)] for _ in dev]
        torch.cuda.synchronize()
        for _ in range(3):
            for m, o, st in zip(dev, out, streams):
                ev.select(m, *o, stream=st)
        torch.cuda.synchronize()
    for m, (p, w) in zip(mass, out):
        rp, rw = C.evict_select(m, g.seg_len, g.seg_page_offsets, g.seg_pages, keep, 2, 3)
        assert np.array_equal(p.cpu().numpy(), rp) and np.array_equal(w.cpu().numpy(), rw)


def test_select_writes_only_its_outputs():
    require_gpu()
    say("[case] select: outputs one by one, guard values")
    rng = np.random.default_rng(2)
    g = W.assemble_graph([50, 1200, 3], [[0, 1, 2]], 4)
    mass = torch.from_numpy(_masses(rng, "spread", 16 * g.num_pages)).cuda()
    keep = [20, 700, 0]
    lib = G.load_library()
    with G.Evict(G.HostGraph.from_graph(g), keep, 0, 0, g.num_pages) as ev:
        ref_p, ref_w = ev.select(mass)
        both = torch.full((2, 730), -9, dtype=torch.int32, device="cuda")
        st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        for p, w in ((both[0], None), (None, both[1])):
            assert lib.graphattn_evict_select(
                ev.handle, ctypes.c_void_p(mass.data_ptr()),
                ctypes.c_void_p(p.data_ptr()) if p is not None else None,
                ctypes.c_void_p(w.data_ptr()) if w is not None else None, st) == G.GA_OK
        assert lib.graphattn_evict_select(ev.handle, ctypes.c_void_p(mass.data_ptr()), None, None,
                                          st) == G.GA_EINVAL
        assert lib.graphattn_evict_select(ev.handle, None, ctypes.c_void_p(both.data_ptr()), None,
                                          st) == G.GA_EINVAL
        with pytest.raises(ValueError):
            ev.select(mass[:-1].contiguous())
        with pytest.raises(ValueError):
            ev.select(mass.double())
        with pytest.raises(ValueError):
            ev.select(mass, torch.empty(720, dtype=torch.int64, device="cuda"))
        with pytest.raises(ValueError):
            ev.select(mass, torch.empty(719, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
    assert torch.equal(both[0, :720], ref_p) and torch.equal(both[1, :720], ref_w)
    assert (both[:, 720:] == -9).all()


# ----------------------------------------------------------------------------------------------
# The whole cycle
# ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("mxfp4", 28, 4, 128), ("mxfp4", 8, 2, 64),
                                            ("bf16", 8, 2, 128)])
def test_cycle(dtype, Hq, Hkv, D):
    """Append a graph's tokens, attend for three steps gathering mass, evict half of every segment,
    move the rest to new pages and attend over them: each stage against the oracle."""
    require_gpu()
    say(f"[case] cycle {dtype} {Hq}/{Hkv}/{D}")
    rng = np.random.default_rng(21)
    lens, paths = [90, 33, 64, 17], [[0, 1], [0, 2], [0, 1, 3]]
    old = W.assemble_graph(lens, paths, 6)
    keep = [(n + 1) // 2 for n in lens]
    new = W.assemble_graph(keep, paths, 7)
    P = old.num_pages + new.num_pages
    p = G.make_params(Hq, Hkv, D, P, dtype)
    n = sum(lens)
    k, v = draw_q(rng, n, Hkv, D), draw_q(rng, n, Hkv, D)
    words = np.concatenate([old.seg_pages[old.seg_page_offsets[s] + np.arange(m) // 16].astype(int)
                            * 16 + np.arange(m) % 16 for s, m in enumerate(lens)])
    pool = G.empty_pool(p)
    pool.zero_()
    G.kv_append(pool, k.cuda(), v.cuda(), torch.from_numpy(words).int().cuda(), p)

    def values():
        torch.cuda.synchronize()
        return C.pool_values(pool.cpu().numpy()) if dtype == "mxfp4" else bits_of(pool)

    old.num_pages = P
    vals = values()
    mass = torch.zeros(16 * P, device="cuda")
    ref = np.zeros(16 * P)
    with G.Plan(G.HostGraph.from_graph(old), p) as pl:
        for step in range(3):
            q = draw_q(rng, 3, Hq, D)
            out = torch.empty((3, Hq, D), dtype=torch.bfloat16, device="cuda")
            lse = torch.empty((3, Hq), device="cuda")
            pl.run(q.cuda(), pool, out, lse)
            pl.run_mass(q.cuda(), pool, lse, mass, mass, 0.9)
            torch.cuda.synchronize()
            check_attention(f"step {step}", out, lse, q, vals, old, Hq, Hkv)
            before = ref
            ref = C.mass(bits_of(q), vals, old, bits_of(lse), Hq, Hkv, before, 0.9)
            bound = mass_bound(q, vals, old, bits_of(lse), Hq, Hkv, ref, 0.9, before)
            live = np.isfinite(ref)
            got = bits_of(mass)
            assert (np.abs(got - ref)[live] <= (step + 1) * bound[live]).all()
            ref = np.where(live, ref, 0.0)
            ref[live] = got[live]
    with G.Evict(G.HostGraph.from_graph(old), keep, 2, 6, P) as ev:
        pos, src = ev.select(mass)
    rp, rw = C.evict_select(bits_of(mass), old.seg_len, old.seg_page_offsets, old.seg_pages, keep,
                            2, 6)
    assert np.array_equal(pos.cpu().numpy(), rp) and np.array_equal(src.cpu().numpy(), rw)
    moved = W.RolloutGraph(new.seg_len, new.seg_page_offsets,
                           (new.seg_pages + old_pages(old)).astype(np.int32), new.path_offsets,
                           new.path_segs, P)
    dst = np.concatenate([moved.seg_pages[moved.seg_page_offsets[s] + np.arange(m) // 16].astype(int)
                          * 16 + np.arange(m) % 16 for s, m in enumerate(keep)])
    kept_k, kept_v = G.kv_read(pool, src, p)
    G.kv_copy(pool, src, torch.from_numpy(dst).int().cuda(), p)
    there_k, there_v = G.kv_read(pool, torch.from_numpy(dst).int().cuda(), p)
    torch.cuda.synchronize()
    assert torch.equal(kept_k, there_k) and torch.equal(kept_v, there_v)
    vals = values()
    q = draw_q(rng, 3, Hq, D)
    out, lse = G.decode(q.cuda(), pool, G.HostGraph.from_graph(moved), p)
    torch.cuda.synchronize()
    check_attention("after eviction", out, lse, q, vals, moved, Hq, Hkv)


def old_pages(graph):
    return int(graph.seg_pages.max()) + 1


def test_captured_cycle_replays():
    """attend, mass, select and copy captured into a graph: every replay equals the eager calls on the
    same inputs, with eager work of other plans between the replays."""
    require_gpu()
    say("[case] captured cycle")
    rng = np.random.default_rng(31)
    Hq, Hkv, D = 12, 4, 128
    lens, paths = [200, 33, 64, 1100], [[0, 1], [0, 2], [0, 1, 3]]
    g = W.assemble_graph(lens, paths, 6, slack_pages=60)
    free = np.setdiff1d(np.arange(g.num_pages), g.seg_pages)
    raw = random_pool(rng, g.num_pages, Hkv, D, -2, 1)
    p = G.make_params(Hq, Hkv, D, g.num_pages, "mxfp4")
    keep = [n // 2 for n in lens]
    total = sum(keep)
    dst = torch.from_numpy((free[np.arange(total) // 16] * 16 + np.arange(total) % 16)
                           .astype(np.int32)).cuda()
    start = torch.from_numpy(raw).cuda()

    class Set:
        def __init__(self):
            self.q = torch.zeros(3, Hq, D, dtype=torch.bfloat16, device="cuda")
            self.pool = start.clone()
            self.out = torch.zeros_like(self.q)
            self.lse = torch.zeros(3, Hq, device="cuda")
            self.mass = torch.zeros(16 * g.num_pages, device="cuda")
            self.pos = torch.zeros(total, dtype=torch.int32, device="cuda")
            self.words = torch.zeros(total, dtype=torch.int32, device="cuda")
            self.plan = G.Plan(G.HostGraph.from_graph(g), p)
            self.plan.schedule()
            self.ev = G.Evict(G.HostGraph.from_graph(g), keep, 0, 4, g.num_pages)

        def run(self):
            self.plan.run(self.q, self.pool, self.out, self.lse)
            self.plan.run_mass(self.q, self.pool, self.lse, self.mass, self.mass, 0.5)
            self.ev.select(self.mass, self.pos, self.words)
            G.kv_copy(self.pool, self.words, dst, p)

    a, b = Set(), Set()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.run()
    torch.cuda.synchronize()
    for i in range(5):
        q = draw_q(rng, 3, Hq, D).cuda()
        a.q.copy_(q)
        b.q.copy_(q)
        torch.cuda.synchronize()
        graph.replay()
        b.run()
        torch.cuda.synchronize()
        for name in ("pool", "mass", "pos", "words", "lse"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (i, name)
        assert torch.equal(a.out.view(torch.int16), b.out.view(torch.int16)), i
    for s in (a, b):
        s.plan.close()
        s.ev.close()


def test_pages_beyond_four_gigabytes():
    """Every call on pages at the end of a pool of 4.1 GiB: byte offsets that pass 32 bits."""
    require_gpu()
    say("[case] pages beyond 4 GiB")
    rng = np.random.default_rng(17)
    Hq, Hkv, D = 16, 8, 128
    lens, paths = W.with_new_steps([150, 37], [[0], [0, 1], [0]], [20, 33, 16])
    g = W.assemble_graph(lens, paths, 6, slack_pages=4)
    n = g.num_pages
    P = 2 ** 32 // (Hkv * 17 * D) + 3 * n
    assert (P - n) * Hkv * 17 * D > 2 ** 32
    far = G.HostGraph(g.seg_len, g.seg_page_offsets, g.seg_pages + (P - n), g.path_offsets, g.path_segs)
    p = G.make_params(Hq, Hkv, D, P, "mxfp4")
    pool = torch.zeros(P, Hkv, 17 * D, dtype=torch.uint8, device="cuda")
    raw = poison_unused(random_pool(rng, n, Hkv, D, -2, 1), g)
    pool[-n:] = torch.from_numpy(raw).cuda()
    # append and read: the last segment's tokens again
    s = len(lens) - 1
    words = np.array([int(g.seg_pages[g.seg_page_offsets[s] + t // 16]) * 16 + t % 16 for t in range(lens[s])])
    kv = draw_q(rng, 2 * lens[s], Hkv, D)
    k, v = kv[:lens[s]].contiguous(), kv[lens[s]:].contiguous()
    dev_words = torch.from_numpy(words + 16 * (P - n)).int().cuda()
    G.kv_append(pool, k.cuda(), v.cuda(), dev_words, p)
    raw = C.append(raw, bits_of(k), bits_of(v), words)
    assert np.array_equal(pool[-n:].cpu().numpy(), raw)
    vals = C.pool_values(raw)
    rk, rv = G.kv_read(pool, dev_words, p)
    torch.cuda.synchronize()
    assert np.array_equal(bits_of(rk), vals[words // 16, :, 0, words % 16])
    assert np.array_equal(bits_of(rv), vals[words // 16, :, 1, words % 16])
    for counts in (None, [20, 33, 16], [1, 2, 1]):
        rows = 3 if counts is None else sum(counts)
        q = draw_q(rng, rows, Hq, D)
        out = torch.zeros(rows, Hq, D, dtype=torch.bfloat16, device="cuda")
        lse = torch.zeros(rows, Hq, device="cuda")
        mass = torch.full((16 * P,), -3.0, device="cuda")
        with G.Plan(far, p, query_counts=counts) as pl:
            pl.run(q.cuda(), pool, out, lse)
            check_attention(f"far pages {counts}", out, lse, q, vals, g, Hq, Hkv, counts)
            pl.run_mass(q.cuda(), pool, lse, mass)
            torch.cuda.synchronize()
        zero = np.zeros(16 * n, dtype=np.float32)
        l64 = bits_of(lse).astype(float)
        ref = C.mass(bits_of(q), vals, g, l64, Hq, Hkv, zero, 1.0, counts)
        live = np.isfinite(ref)
        off = np.abs(bits_of(mass[-16 * n:]) - ref)[live] / mass_bound(q, vals, g, l64, Hq, Hkv, ref, 0.0, zero,
                                                                       counts)[live]
        assert off.max() <= 1.0, counts
        assert (mass[:-16 * n] == -3).all() and (bits_of(mass[-16 * n:])[~live] == -3).all()
    # copy: to the first page (its codes and scales are the source's)
    G.kv_copy(pool, dev_words[:16].contiguous(), torch.arange(16, dtype=torch.int32, device="cuda"), p)
    ck, cv = G.kv_read(pool, torch.arange(16, dtype=torch.int32, device="cuda"), p)
    torch.cuda.synchronize()
    assert torch.equal(ck, rk[:16]) and torch.equal(cv, rv[:16])


def test_select_on_the_highest_pages():
    """Slot words up to 2^31 - 1, whose masses lie 8 GiB into their array."""
    require_gpu()
    say("[case] select on the highest pages")
    rng = np.random.default_rng(23)
    lens = [900, 3000, 17000, 64]
    g = W.assemble_graph(lens, [[0, 1, 2, 3]], 4)
    n, P = g.num_pages, 2 ** 27
    mass = _masses(rng, "spread", 16 * n)
    dev = torch.zeros(16 * P, device="cuda")
    dev[-16 * n:] = torch.from_numpy(mass).cuda()
    keep = [m // 3 for m in lens]
    far = G.HostGraph(g.seg_len, g.seg_page_offsets, g.seg_pages + (P - n), g.path_offsets, g.path_segs)
    with G.Evict(far, keep, 2, 5, P) as ev:
        pos, words = ev.select(dev)
        torch.cuda.synchronize()
    rp, rw = C.evict_select(mass, g.seg_len, g.seg_page_offsets, g.seg_pages, keep, 2, 5)
    assert np.array_equal(pos.cpu().numpy(), rp)
    assert np.array_equal(words.cpu().numpy(), rw + 16 * (P - n))


def test_mass_after_new_lengths():
    """A plan that grew gives a fresh plan's mass, bit for bit where the parts are the same and within the
    bound otherwise; slots past the shorter lengths are left as they were."""
    require_gpu()
    say("[case] mass after new lengths")
    rng = np.random.default_rng(29)
    Hq, Hkv, D = 8, 2, 64
    final = W.assemble_graph([700, 90, 130], [[0, 1], [0, 2], [0]], 6, slack_pages=2)
    pool, vals = _pool(rng, final, Hkv, D, "mxfp4")
    p = G.make_params(Hq, Hkv, D, final.num_pages, "mxfp4")
    q = draw_q(rng, 3, Hq, D)
    with G.Plan(G.HostGraph([5, 1, 17], final.seg_page_offsets, final.seg_pages, final.path_offsets,
                            final.path_segs), p) as pl:
        for lens in ([5, 1, 17], [300, 33, 130], [700, 90, 130]):
            pl.set_lengths(lens)
            g = W.RolloutGraph(np.array(lens, dtype=np.int32), final.seg_page_offsets, final.seg_pages,
                               final.path_offsets, final.path_segs, final.num_pages)
            lse = C.attention(bits_of(q), vals, g, Hq, Hkv)[1].astype(np.float32)
            out = torch.full((16 * g.num_pages,), -5.0, device="cuda")
            pl.run_mass(q.cuda(), pool, torch.from_numpy(lse).cuda(), out)
            torch.cuda.synchronize()
            zero = np.zeros(16 * g.num_pages, dtype=np.float32)
            ref = C.mass(bits_of(q), vals, g, lse.astype(float), Hq, Hkv, zero, 1.0)
            live = np.isfinite(ref)
            off = np.abs(bits_of(out) - ref)[live] / mass_bound(q, vals, g, lse, Hq, Hkv, ref, 0.0, zero)[live]
            assert off.max() <= 1.0, lens
            assert (bits_of(out)[~live] == -5).all(), lens


def test_captured_extend_replays():
    """append, attention of many query rows and mass, captured: every replay equals the eager calls."""
    require_gpu()
    say("[case] captured extend")
    rng = np.random.default_rng(37)
    Hq, Hkv, D = 28, 4, 128
    counts = [40, 25, 33]
    lens, paths = W.with_new_steps([300, 20], [[0], [0, 1], [0]], counts)
    g = W.assemble_graph(lens, paths, 6, slack_pages=1)
    start = torch.from_numpy(random_pool(rng, g.num_pages, Hkv, D, -2, 1)).cuda()
    p = G.make_params(Hq, Hkv, D, g.num_pages, "mxfp4")
    rows = sum(counts)
    words = torch.from_numpy(np.concatenate([
        g.seg_pages[g.seg_page_offsets[s] + np.arange(lens[s]) // 16].astype(np.int32) * 16 +
        np.arange(lens[s], dtype=np.int32) % 16 for s in range(2, 5)])).cuda()

    class Set:
        def __init__(self):
            self.q = torch.zeros(rows, Hq, D, dtype=torch.bfloat16, device="cuda")
            self.kv = torch.zeros(2, len(words), Hkv, D, dtype=torch.bfloat16, device="cuda")
            self.pool, self.out = start.clone(), torch.zeros_like(self.q)
            self.lse = torch.zeros(rows, Hq, device="cuda")
            self.mass = torch.zeros(16 * g.num_pages, device="cuda")
            self.plan = G.Plan(G.HostGraph.from_graph(g), p, query_counts=counts)
            self.plan.schedule()

        def run(self):
            G.kv_append(self.pool, self.kv[0], self.kv[1], words, p)
            self.plan.run(self.q, self.pool, self.out, self.lse)
            self.plan.run_mass(self.q, self.pool, self.lse, self.mass, self.mass, 0.5)

    a, b = Set(), Set()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.run()
    torch.cuda.synchronize()
    for i in range(4):
        q, kv = draw_q(rng, rows, Hq, D).cuda(), draw_q(rng, 2 * len(words), Hkv, D).cuda().view_as(a.kv)
        for x in (a, b):
            x.q.copy_(q)
            x.kv.copy_(kv)
        torch.cuda.synchronize()
        graph.replay()
        b.run()
        torch.cuda.synchronize()
        for name in ("pool", "mass", "lse"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (i, name)
        assert torch.equal(a.out.view(torch.int16), b.out.view(torch.int16)), i
    for x in (a, b):
        x.plan.close()
