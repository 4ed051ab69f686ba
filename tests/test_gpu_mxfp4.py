"""MXFP4 pools on the GPU against the float64 oracle: rounding and layout byte for byte, copies and
reads, decode and multi-query attention within bounds derived from the rounding of its steps."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as C
from paper_2606_18954_amd import graphattn as G
from paper_2606_18954_amd import workloads as W

from cache_util import (bits_of, check_attention, draw_q, poison_unused, random_pool)
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------------------------
# Append, copy, read
# ----------------------------------------------------------------------------------------------

def _append(pool, k, v, words, Hkv, D):
    p = G.make_params(Hkv, Hkv, D, pool.shape[0], "mxfp4")
    dev = torch.from_numpy(pool).cuda()
    G.kv_append(dev, k.cuda(), v.cuda(), torch.as_tensor(words, dtype=torch.int32).cuda(), p)
    torch.cuda.synchronize()
    return dev, p


@pytest.mark.parametrize("Hkv,D,n", [(1, 64, 1), (4, 128, 1), (2, 64, 7), (3, 128, 33), (8, 64, 16)])
def test_append_matches_the_oracle_byte_for_byte(Hkv, D, n):
    require_gpu()
    say(f"[case] append {Hkv} x {D}, {n} tokens")
    rng = np.random.default_rng(100 * Hkv + D + n)
    P = n // 8 + 3
    pool = rng.integers(0, 256, (P, Hkv, 17 * D)).astype(np.uint8)
    scale = 10.0 ** rng.uniform(-4, 4, (n, Hkv, 1))
    k = torch.from_numpy((rng.standard_normal((n, Hkv, D)) * scale).astype(np.float32)).bfloat16()
    v = torch.from_numpy(rng.standard_normal((n, Hkv, D)).astype(np.float32)).bfloat16()
    words = rng.permutation(16 * P)[:n].astype(np.int64)
    if n > 5:
        words[2], words[4], words[5] = -1, 16 * P, -(2 ** 31)     # skipped
    dev, _ = _append(pool, k, v, words, Hkv, D)
    ref = C.append(pool, bits_of(k), bits_of(v), words)
    assert np.array_equal(dev.cpu().numpy(), ref)


def test_append_rounds_every_bf16_value():
    """Every finite bf16 magnitude in a block under each of the tops 2^i x {1, 1.5, 1.75}: the value the
    pool stands for is the definition's, by way of the bytes."""
    require_gpu()
    D, Hkv = 128, 4
    allv = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = allv[torch.isfinite(allv.float())]
    x = x[torch.argsort(x.float().abs(), stable=True)]           # neighbours share a block
    pad = -x.numel() % (Hkv * D)
    x = torch.cat([x, torch.zeros(pad, dtype=torch.bfloat16)])
    k = x.view(-1, Hkv, D)
    v = k.flip(0).contiguous()
    # Blocks that mix magnitudes: every 32nd value far larger.
    tops = torch.tensor([2.0 ** e * m for e in range(-120, 120, 16) for m in (1.0, 1.5, 1.75)])
    r = torch.arange(k.shape[0]) % len(tops)
    v = v.clone()
    v.view(-1, Hkv, D // 32, 32)[..., 5] = tops[r].bfloat16()[:, None, None]
    n = k.shape[0]
    P = (n + 15) // 16
    pool = np.zeros((P, Hkv, 17 * D), dtype=np.uint8)
    say(f"[case] append of every bf16 value, {n} tokens")
    dev, p = _append(pool, k, v, np.arange(n), Hkv, D)
    assert np.array_equal(dev.cpu().numpy(), C.append(pool, bits_of(k), bits_of(v), np.arange(n)))


def test_blocks_with_nan_or_infinity_read_as_nan():
    require_gpu()
    say("[case] append of NaN and infinities")
    x = torch.ones(3, 2, 64)
    x[0, 0, 3], x[1, 1, 40], x[2, 0, 0] = float("nan"), float("inf"), -float("inf")
    x = x.bfloat16()
    dev, p = _append(np.zeros((1, 2, 17 * 64), dtype=np.uint8), x, x, [0, 1, 2], 2, 64)
    k, v = G.kv_read(dev, torch.arange(3, dtype=torch.int32).cuda(), p)
    nan = torch.isnan(k.cpu())
    assert torch.equal(nan, torch.isnan(v.cpu()))
    want = torch.zeros(3, 2, 64, dtype=torch.bool)
    want[0, 0, :32] = want[1, 1, 32:] = want[2, 0, :32] = True
    assert torch.equal(nan, want)
    assert (k.cpu()[~want] == 1).all()


@pytest.mark.parametrize("dtype", ["mxfp4", "bf16", "f32"])
@pytest.mark.parametrize("Hkv,D", [(2, 64), (5, 128)])
def test_read_gives_the_values_of_the_slots(dtype, Hkv, D):
    require_gpu()
    say(f"[case] read {dtype} {Hkv} x {D}")
    rng = np.random.default_rng(7)
    P, n = 4, 37
    words = rng.integers(0, 16 * P, n)                            # some twice
    words[3], words[30] = -5, 16 * P
    p = G.make_params(Hkv, Hkv, D, P, dtype)
    if dtype == "mxfp4":
        raw = random_pool(rng, P, Hkv, D, -100, 100)
        pool = torch.from_numpy(raw).cuda()
        vals = C.pool_values(raw)
    else:
        pool = torch.randn(P, Hkv, 2, 16, D, dtype=torch.float32)
        pool = (pool.bfloat16() if dtype == "bf16" else pool).cuda()
        vals = bits_of(pool)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    k = torch.full((n, Hkv, D), 99.0, dtype=dt, device="cuda")
    v = torch.full((n, Hkv, D), 98.0, dtype=dt, device="cuda")
    before = pool.clone()
    G.kv_read(pool, torch.from_numpy(words).int().cuda(), p, k, v)
    torch.cuda.synchronize()
    assert torch.equal(before, pool)
    for j, w in enumerate(words):
        if 0 <= w < 16 * P:
            assert np.array_equal(bits_of(k[j]), vals[w // 16, :, 0, w % 16]), j
            assert np.array_equal(bits_of(v[j]), vals[w // 16, :, 1, w % 16]), j
        else:
            assert (k[j] == 99).all() and (v[j] == 98).all()


@pytest.mark.parametrize("Hkv,D", [(1, 128), (4, 64)])
def test_copy_moves_codes_and_scales(Hkv, D):
    require_gpu()
    say(f"[case] copy {Hkv} x {D}")
    rng = np.random.default_rng(11)
    P = 6
    raw = rng.integers(0, 256, (P, Hkv, 17 * D)).astype(np.uint8)
    src = np.concatenate([rng.permutation(48)[:20], [-1, 16 * P, 50]])
    dst = np.concatenate([48 + rng.permutation(48)[:20], [90, 91, -7]])
    p = G.make_params(Hkv, Hkv, D, P, "mxfp4")
    pool = torch.from_numpy(raw).cuda()
    G.kv_copy(pool, torch.from_numpy(src).int().cuda(), torch.from_numpy(dst).int().cuda(), p)
    torch.cuda.synchronize()
    ref = raw.copy()
    for s, d in zip(src[:20], dst[:20]):
        for value in (False, True):
            for c in range(0, D, 2):
                a, b = C.code_place(s % 16, c, D, value)[0], C.code_place(d % 16, c, D, value)[0]
                ref[d // 16, :, b] = raw[s // 16, :, a]
            for c in range(0, D, 32):
                ref[d // 16, :, C.scale_place(d % 16, c, D, value)] = \
                    raw[s // 16, :, C.scale_place(s % 16, c, D, value)]
    assert np.array_equal(pool.cpu().numpy(), ref)


# ----------------------------------------------------------------------------------------------
# Attention
# ----------------------------------------------------------------------------------------------

HEADS = [(28, 4, 128), (8, 2, 64), (5, 1, 128), (6, 6, 64), (24, 3, 128), (40, 8, 64)]


def _case(rng, graph, Hq, Hkv, D, rows, lo=-2, hi=1):
    raw = poison_unused(random_pool(rng, graph.num_pages, Hkv, D, lo, hi), graph)
    return raw, C.pool_values(raw), draw_q(rng, rows, Hq, D)


def _run(graph, raw, q, Hq, Hkv, D, counts=None, scale=0.0, out_f32=False, plan=True):
    p = G.make_params(Hq, Hkv, D, graph.num_pages, "mxfp4", scale, out_f32)
    hg = G.HostGraph.from_graph(graph)
    pool, q = torch.from_numpy(raw).cuda(), q.cuda()
    if not plan:
        r = G.decode(q, pool, hg, p) if counts is None else G.extend(q, pool, hg, counts, p)
        torch.cuda.synchronize()
        return r
    # (a row behind the last one, which stays as it is)
    out = torch.full((q.shape[0] + 1, Hq, D), 7.0, dtype=torch.float32 if out_f32 else torch.bfloat16,
                     device="cuda")
    lse = torch.full((q.shape[0] + 1, Hq), 7.0, device="cuda")
    with G.Plan(hg, p, query_counts=counts) as pl:
        pl.run(q, pool, out, lse)
        torch.cuda.synchronize()
    assert (out[-1] == 7).all() and (lse[-1] == 7).all()
    return out[:-1], lse[:-1]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("out_f32", [False, True])
def test_decode_on_random_graphs(Hq, Hkv, D, out_f32):
    require_gpu()
    rng = np.random.default_rng(Hq * 1000 + D)
    g = W.random_graph(rng, 9, 21, 150, 5, slack_pages=3, seed=2)
    say(f"[case] decode {Hq}/{Hkv}/{D} f32={out_f32}")
    raw, vals, q = _case(rng, g, Hq, Hkv, D, g.num_branches)
    out, lse = _run(g, raw, q, Hq, Hkv, D, out_f32=out_f32)
    check_attention(f"decode {Hq}/{Hkv}/{D}", out, lse, q, vals, g, Hq, Hkv, out_f32=out_f32)


@pytest.mark.parametrize("lens", [[1], [2], [15], [16], [17], [31], [32], [33], [1, 1], [1, 16, 17],
                                  [47, 1, 48], [129]])
def test_decode_at_page_ends(lens):
    """One branch (one partial: rows written without a merge), and two that share the first segment."""
    require_gpu()
    rng = np.random.default_rng(sum(lens))
    for paths in ([list(range(len(lens)))], [[0]] * 2 if len(lens) == 1 else [[0, 1], [0]]):
        g = W.assemble_graph(lens, paths, 3, slack_pages=1)
        say(f"[case] lens {lens} paths {paths}")
        for Hq, Hkv, D in ((7, 1, 128), (4, 2, 64)):
            raw, vals, q = _case(rng, g, Hq, Hkv, D, len(paths))
            out, lse = _run(g, raw, q, Hq, Hkv, D)
            check_attention(f"lens {lens}", out, lse, q, vals, g, Hq, Hkv)


@pytest.mark.parametrize("branches", [2, 3, 5, 9, 10, 14, 18, 19, 37, 40])
def test_decode_over_row_counts(branches):
    """7 rows a branch: one to eight row tiles in a block, and several blocks."""
    require_gpu()
    rng = np.random.default_rng(branches)
    g = W.assemble_graph([300] + [11] * branches, [[0, 1 + b] for b in range(branches)], 5)
    say(f"[case] {branches} branches")
    raw, vals, q = _case(rng, g, 14, 2, 128, branches)
    out, lse = _run(g, raw, q, 14, 2, 128)
    check_attention(f"{branches} branches", out, lse, q, vals, g, 14, 2)


def test_decode_of_a_long_context_in_many_chunks():
    require_gpu()
    say("[case] 20000 tokens, 3 branches")
    rng = np.random.default_rng(1)
    g = W.assemble_graph([20000, 5, 70], [[0, 1], [0, 2], [0]], 5, slack_pages=2)
    raw, vals, q = _case(rng, g, 4, 1, 64, 3)
    out, lse = _run(g, raw, q, 4, 1, 64)
    check_attention("long", out, lse, q, vals, g, 4, 1)


def test_scales_far_apart():
    """Blocks of scales 2^-60 .. 2^60 in V (bf16's range, not fp16's), and scores of every size through
    a softmax scale."""
    require_gpu()
    say("[case] scales far apart")
    rng = np.random.default_rng(8)
    g = W.assemble_graph([70, 40], [[0, 1], [0]], 5)
    for lo, hi, scale in ((-60, -50, 2.0 ** 50), (40, 60, 2.0 ** -60), (-1, 1, 3.0)):
        raw, vals, q = _case(rng, g, 8, 2, 128, 2, lo, hi)
        out, lse = _run(g, raw, q, 8, 2, 128, scale=scale, out_f32=True)
        check_attention(f"scales 2^{lo}..2^{hi}", out, lse, q, vals, g, 8, 2, scale=scale,
                        out_f32=True)


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_extend_on_trees(Hq, Hkv, D):
    require_gpu()
    rng = np.random.default_rng(Hq + D)
    lens = [int(rng.integers(1, 200)) for _ in range(3)]
    step = [int(n) for n in rng.integers(1, 60, 6)]
    lens, paths = W.with_new_steps(lens, [[0], [0, 1], [0, 2], [1], [2, 1], [0]], step)
    counts = [int(rng.integers(1, n + 1)) for n in step]
    g = W.assemble_graph(lens, paths, 6, slack_pages=2)
    say(f"[case] extend {Hq}/{Hkv}/{D} counts {counts}")
    raw, vals, q = _case(rng, g, Hq, Hkv, D, sum(counts))
    out, lse = _run(g, raw, q, Hq, Hkv, D, counts)
    check_attention(f"extend {Hq}/{Hkv}/{D}", out, lse, q, vals, g, Hq, Hkv, counts)


@pytest.mark.parametrize("lens", [[1], [16], [17, 40], [130], [33, 1, 64]])
def test_prefill(lens):
    """Every token a query: rows that see one token, units whose later pages no row sees."""
    require_gpu()
    rng = np.random.default_rng(len(lens))
    g = W.assemble_graph(lens, [[i] for i in range(len(lens))], 4, slack_pages=1)
    for Hq, Hkv, D in ((7, 1, 128), (4, 2, 64)):
        say(f"[case] prefill {lens} {Hq}/{Hkv}/{D}")
        raw, vals, q = _case(rng, g, Hq, Hkv, D, sum(lens))
        out, lse = _run(g, raw, q, Hq, Hkv, D, lens)
        check_attention(f"prefill {lens}", out, lse, q, vals, g, Hq, Hkv, lens)


def test_prefill_of_many_rows():
    require_gpu()
    say("[case] prefill of 700 tokens, 28/4 heads, sampled rows")
    rng = np.random.default_rng(2)
    lens = [700, 333]
    g = W.assemble_graph(lens, [[0], [1]], 4)
    raw, vals, q = _case(rng, g, 28, 4, 128, sum(lens))
    out, lse = _run(g, raw, q, 28, 4, 128, lens)
    rows = list(range(0, sum(lens), 41)) + [699, 700, 1032]
    check_attention("prefill of many rows", out, lse, q, vals, g, 28, 4, lens, sorted(rows))


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("prefix,step", [(1, 33), (259, 40), (900, 17)])
def test_many_query_rows_a_page(Hq, Hkv, D, prefix, step):
    """Branches of up to `step` queries over a shared prefix: row blocks of 128 rows and less, pages that end
    inside a tile with NaN scales behind, one partial row (prefix 1) and several."""
    require_gpu()
    rng = np.random.default_rng(Hq * prefix + step)
    own = [int(n) for n in rng.integers(1, step + 1, 9)]
    own[0], own[1] = step, 1
    lens, paths = W.with_new_steps([prefix, 18], [[0]] * 8 + [[0, 1]], own)
    g = W.assemble_graph(lens, paths, 6, slack_pages=2)
    say(f"[case] extend {Hq}/{Hkv}/{D} prefix {prefix} counts {own}")
    raw, vals, q = _case(rng, g, Hq, Hkv, D, sum(own))
    out, lse = _run(g, raw, q, Hq, Hkv, D, own)
    check_attention(f"many rows {Hq}/{Hkv}/{D}", out, lse, q, vals, g, Hq, Hkv, own)


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_few_query_rows_a_page(Hq, Hkv, D):
    """One to three queries a branch, mostly over pages of their own."""
    require_gpu()
    rng = np.random.default_rng(Hq)
    own = [1, 2, 3, 2, 1]
    lens, paths = W.with_new_steps([5, 300, 130, 77, 16, 201], [[0, 1], [0, 2], [3], [4], [5]], own)
    g = W.assemble_graph(lens, paths, 6, slack_pages=2)
    say(f"[case] extend {Hq}/{Hkv}/{D} counts {own}")
    raw, vals, q = _case(rng, g, Hq, Hkv, D, sum(own))
    out, lse = _run(g, raw, q, Hq, Hkv, D, own)
    check_attention(f"few rows {Hq}/{Hkv}/{D}", out, lse, q, vals, g, Hq, Hkv, own)


def test_entry_points_agree_bit_for_bit():
    """decode, decode_static, a plan, a plan with one query each and a later run of it: the same bits."""
    require_gpu()
    say("[case] entry points")
    rng = np.random.default_rng(4)
    lens, paths = W.with_new_steps([90, 40, 17], [[0], [0, 1], [0, 2], [1]], [5, 16, 1, 33])
    g = W.assemble_graph(lens, paths, 6, slack_pages=2)
    raw, vals, q = _case(rng, g, 12, 4, 128, 4)
    p = G.make_params(12, 4, 128, g.num_pages, "mxfp4")
    hg = G.HostGraph.from_graph(g)
    pool, qd = torch.from_numpy(raw).cuda(), q.cuda()
    ref_o, ref_l = G.decode(qd, pool, hg, p)
    check_attention("decode", ref_o, ref_l, q, vals, g, 12, 4)
    got = [G.decode_static(qd, pool, hg, p, torch.zeros_like(ref_o), torch.zeros_like(ref_l)),
           G.extend(qd, pool, hg, [1] * 4, p)]
    for counts in (None, [1] * 4):
        with G.Plan(hg, p, query_counts=counts) as pl:
            for _ in range(3):
                o, l = torch.zeros_like(ref_o), torch.zeros_like(ref_l)
                pl.run(qd, pool, o, l)
                got.append((o, l))
            torch.cuda.synchronize()
    for o, l in got:
        assert torch.equal(o.view(torch.int16), ref_o.view(torch.int16)) and torch.equal(l, ref_l)


def test_growing_plan_and_append():
    """The decode loop on an MXFP4 pool: append a token per branch, grow, schedule, attend."""
    require_gpu()
    say("[case] decode loop")
    rng = np.random.default_rng(12)
    Hq, Hkv, D = 8, 2, 128
    lens, paths = [40, 15, 30], [[0, 1], [0, 2]]
    final = W.assemble_graph([40, 15 + 4, 30 + 4], paths, 6, slack_pages=1)
    raw = poison_unused(random_pool(rng, final.num_pages, Hkv, D), final)
    pool = torch.from_numpy(raw).cuda()
    p = G.make_params(Hq, Hkv, D, final.num_pages, "mxfp4")
    start = G.HostGraph(lens, final.seg_page_offsets, final.seg_pages, final.path_offsets,
                        final.path_segs)
    with G.Plan(start, p) as pl:
        for step in range(4):
            new = [15 + step, 30 + step]
            words = [int(final.seg_pages[final.seg_page_offsets[s] + t // 16]) * 16 + t % 16
                     for s, t in zip((1, 2), new)]
            kv = draw_q(rng, 4, Hkv, D)
            G.kv_append(pool, kv[:2].contiguous().cuda(), kv[2:].contiguous().cuda(),
                        torch.tensor(words, dtype=torch.int32).cuda(), p)
            pl.set_lengths([40, new[0] + 1, new[1] + 1])
            q = draw_q(rng, 2, Hq, D)
            out = torch.empty((2, Hq, D), dtype=torch.bfloat16, device="cuda")
            lse = torch.empty((2, Hq), device="cuda")
            pl.run(q.cuda(), pool, out, lse)
            torch.cuda.synchronize()
            raw = C.append(raw, bits_of(kv[:2]), bits_of(kv[2:]), words)
            assert np.array_equal(pool.cpu().numpy(), raw)
            g = W.RolloutGraph(np.array([40, new[0] + 1, new[1] + 1], dtype=np.int32),
                               final.seg_page_offsets, final.seg_pages, final.path_offsets,
                               final.path_segs, final.num_pages)
            check_attention(f"step {step}", out, lse, q, C.pool_values(raw), g, Hq, Hkv)


def test_same_bits_every_time_on_any_stream():
    require_gpu()
    say("[case] determinism")
    rng = np.random.default_rng(14)
    g = W.random_graph(rng, 30, 60, 400, 6, seed=3)
    raw, _, q = _case(rng, g, 28, 4, 128, 60)
    p = G.make_params(28, 4, 128, g.num_pages, "mxfp4")
    pool, qd = torch.from_numpy(raw).cuda(), q.cuda()
    ref = None
    with G.Plan(G.HostGraph.from_graph(g), p) as pl:
        streams = [torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()]
        for i in range(9):
            s = streams[i % 3]
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                o = torch.empty((60, 28, 128), dtype=torch.bfloat16, device="cuda")
                l = torch.empty((60, 28), device="cuda")
                pl.run(qd, pool, o, l)
            torch.cuda.synchronize()
            if ref is None:
                ref = o, l
            assert torch.equal(o.view(torch.int16), ref[0].view(torch.int16))
            assert torch.equal(l, ref[1])
