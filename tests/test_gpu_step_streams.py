"""Streams and captured graphs of the calls between two attention calls, all four of them."""
import numpy as np
import pytest
import torch

import step_util as U
from gpu_util import require_gpu
from oracle import step_oracle as S
from paper_2606_18954_amd import graphattn as G
from test_gpu_step import Logits, Qkv, dev, device_graph, full, host

pytestmark = pytest.mark.gpu


def test_outputs_that_calls_make_on_another_stream():
    """Each call on a stream of its own, without outputs, while the current stream is busy: what the call makes is not
    filled behind it (rows of padding are zero, the table -1 behind its total)."""
    require_gpu()
    rng = np.random.default_rng(60)
    a = Qkv(U.qkv_case(rng, 70, 8, 2, 64, "bf16", 64))
    b = Logits(U.logits_case(rng, U.random_graph(rng, 12), 9, 3000, "f32"))
    b.branches[4] = -1
    c = U.page_case(rng, 200)
    lens, free, old, old_pages = (dev(c[k]) for k in ("lens", "free", "old", "old_pages"))
    graph = device_graph(U.random_graph(rng, 20))
    words = a.words.clamp(min=0)

    def all_of_them(**s):
        return (G.qkv_append(a.pool, a.q, a.k, a.v, a.positions, a.words, a.transform, a.params, **s),
                G.process_logits(b.logits, b.rules, b.graph, b.ids, b.branches, b.positions, **s),
                *G.page_table(lens, free, c["spare"], old, old_pages, **s), *G.slot_map(graph, **s),
                *G.kv_read(a.pool, words, a.params, **s))
    want = [t.clone() for t in all_of_them()]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    got = all_of_them(stream=stream)
    stream.synchronize()
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16 else x,
                           y.view(torch.int16) if y.dtype == torch.bfloat16 else y)
    assert (got[0][host(a.positions) < 0] == 0).all() and not got[1][4].any() and not want[1][4].any()


def growing(rng, S=300):
    """A table as it was, lengths that have grown since, and free pages in the order in which they go."""
    before = rng.integers(1, 90, S).astype(np.int32)
    off, pages = fresh_table(before, rng.permutation(6 * S).astype(np.int32))
    lens = (before + rng.integers(0, 60, S)).astype(np.int32)
    free = np.setdiff1d(np.arange(16 * S), pages).astype(np.int32)
    return lens, off, pages, rng.permutation(free).astype(np.int32)


def fresh_table(lens, free):
    off, pages = S.page_table(lens, 3, [], [], free)
    return off, pages.astype(np.int32)


def test_tables_and_slots_behind_work_on_another_stream():
    """Page table and slot map on a stream of their own, behind work that is still filling their inputs there."""
    require_gpu()
    rng = np.random.default_rng(61)
    lens, off, pages, free = growing(rng)
    c = U.slot_case(rng, g=U.random_graph(rng, 40), counts="drawn")
    g, stream = device_graph(c["graph"]), torch.cuda.Stream()
    d_lens, d_off, d_pages, d_free = dev(lens), dev(off), dev(pages), dev(free)
    keep, graph_lens = d_lens.clone(), g.tensors[0].clone()
    d_lens.zero_(), g.tensors[0].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(2_000_000)
        d_lens.copy_(keep)
        g.tensors[0].copy_(graph_lens)
    made = G.page_table(d_lens, d_free, 2, d_off, d_pages, stream=stream)
    outs = [full((c["capacity"],), -77, torch.int32) for _ in range(3)]
    torch.cuda.synchronize()                                # (the fills of outs are the current stream's)
    slots = G.slot_map(g, dev(c["counts"]), None, *outs, stream=stream)
    stream.synchronize()
    want = S.page_table(lens, 2, off, pages, free)
    np.testing.assert_array_equal(host(made[0]), want[0])
    np.testing.assert_array_equal(host(made[1])[:want[0][-1]], want[1])
    U.check_slots(c, *(host(t) for t in slots))


def test_captured_tables_and_slots_replay():
    """Page table and the slots from it in one captured graph: every replay follows what lengths, old table and free
    list hold by then, and takes from the front of the list again."""
    require_gpu()
    rng = np.random.default_rng(62)
    lens, off, pages, free = growing(rng, 200)
    n, spare = 200, 2
    po = np.arange(0, 2 * n + 1, 2).astype(np.int64)
    ps = np.stack([np.zeros(n), np.arange(n)], 1).astype(np.int32).ravel()
    d_lens, d_off, d_old, d_free = dev(lens), dev(off), dev(pages), dev(free)
    counts, capacity = dev(rng.integers(0, 4, n).astype(np.int32)), 4 * n
    new_off, new_pages = torch.zeros(n + 1, dtype=torch.int64, device="cuda"), full((9000,), -77, torch.int32)
    outs = [full((capacity,), -77, torch.int32) for _ in range(3)]
    token_off = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    graph = G.DeviceGraph(d_lens, new_off, new_pages, dev(po), dev(ps), 16 * n)

    def step():
        G.page_table(d_lens, d_free, spare, d_off, d_old, new_off, new_pages)
        G.slot_map(graph, counts, token_off, *outs)

    step()
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured):
        step()
    for i in range(4):
        d_lens.add_(dev(rng.integers(0, 9, n).astype(np.int32)))
        d_free.copy_(dev(rng.permutation(free).astype(np.int32)))
        counts.copy_(dev(rng.integers(0, 4, n).astype(np.int32)))
        if i == 2:
            new_off.zero_(), new_pages.fill_(-1)              # (the program's own work between replays)
        torch.cuda.synchronize()
        captured.replay()
        torch.cuda.synchronize()
        got = [host(t).copy() for t in (new_off, new_pages, token_off, *outs)]
        step()
        for a, b in zip(got, (new_off, new_pages, token_off, *outs)):
            np.testing.assert_array_equal(a, host(b), err_msg=str(i))
        want = S.page_table(host(d_lens), spare, off, pages, host(d_free))
        np.testing.assert_array_equal(got[0], want[0])
        np.testing.assert_array_equal(got[1][:want[0][-1]], want[1])
        slots = S.slot_map(S.Graph(host(d_lens), want[0], want[1], po, ps, 16 * n), host(counts), capacity)
        for a, b in zip(got[2:], slots):
            np.testing.assert_array_equal(a, b)


def test_calls_of_one_graph_on_two_streams_at_once():
    """Slot maps, tables and rules that read the same arrays at the same time, from two streams, into outputs of their own:
    called, and as two captured graphs."""
    require_gpu()
    rng = np.random.default_rng(63)
    lens, off, pages, free = growing(rng)
    table = [dev(x) for x in (lens, free)] + [3, dev(off), dev(pages)]
    c = U.slot_case(rng, g=U.random_graph(rng, 40), counts="drawn")
    g, counts = device_graph(c["graph"]), dev(c["counts"])
    rows = Logits(U.logits_case(rng, c["graph"], 40, 9001, "f32", rules="rfptb"))
    streams = [torch.cuda.Stream() for _ in range(2)]

    class Side:
        def __init__(self):
            self.off, self.pages = torch.zeros(len(lens) + 1, dtype=torch.int64, device="cuda"), full((9000,), -77, torch.int32)
            self.words = [full((c["capacity"],), -77, torch.int32) for _ in range(3)]
            self.token_off = torch.zeros(g.num_branches + 1, dtype=torch.int32, device="cuda")
            self.out = torch.full((40, 9001), 9.0, device="cuda")

        def call(self, stream=None):
            G.page_table(*table, self.off, self.pages, stream=stream)
            G.slot_map(g, counts, self.token_off, *self.words, stream=stream)
            G.process_logits(rows.logits, rows.rules, rows.graph, rows.ids, rows.branches, rows.positions, self.out, stream=stream)

        def check(self):
            want = S.page_table(lens, 3, off, pages, free)
            np.testing.assert_array_equal(host(self.off), want[0])
            np.testing.assert_array_equal(host(self.pages)[:want[0][-1]], want[1])
            assert (host(self.pages)[want[0][-1]:] == -77).all()
            U.check_slots(c, host(self.token_off), *(host(t) for t in self.words))
            U.check_logits(rows.c, host(self.out), np.full((40, 9001), 9, np.float32))
    sides = [Side(), Side()]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, x in zip(streams, sides):
            x.call(s)
    torch.cuda.synchronize()
    for x in sides:
        x.check()
    graphs = []
    for x in sides:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            x.call()
        x.off.zero_(), x.pages.fill_(-77), x.token_off.zero_(), x.out.fill_(9.0)
        for t in x.words:
            t.fill_(-77)
    torch.cuda.synchronize()
    for _ in range(3):
        for s, r in zip(streams, graphs):
            with torch.cuda.stream(s):
                r.replay()
    torch.cuda.synchronize()
    for x in sides:
        x.check()
