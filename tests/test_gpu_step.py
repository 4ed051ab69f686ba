"""The calls between two attention calls on the GPU, against the oracle: page table, slot map, queries and keys with
their append, logit rules; alone, captured and replayed, on other streams, and together as a decode loop runs them."""
import numpy as np
import pytest
import torch

import step_util as U
from gpu_util import compare, require_gpu, say
from oracle import graphattn_oracle as O
from oracle import step_oracle as S
from paper_2606_18954_amd import graphattn as G

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(a, dtype=None):
    """A numpy array on the GPU (uint16: bf16 bits); None stays None."""
    if a is None:
        return None
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).cuda().view(torch.bfloat16)
    if a.dtype == np.uint32:
        return torch.from_numpy(a.view(np.int32)).cuda()
    return torch.from_numpy(a).cuda()


def host(t):
    """A device tensor as numpy (bf16: its bits)."""
    if t.dtype == torch.bfloat16:
        return t.view(torch.int16).cpu().numpy().view(np.uint16)
    return t.cpu().numpy()


def full(shape, value, dtype):
    """A device tensor of that value's bits (bf16) or value."""
    if dtype == torch.bfloat16:
        return torch.full(shape, value, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    return torch.full(shape, value, dtype=dtype, device="cuda")


def device_graph(g):
    return G.DeviceGraph(dev(g["seg_len"]), dev(g["off"]), dev(g["pages"]), dev(g["po"]), dev(g["ps"]), g["num_pages"])


def run_page(c, stream=None):
    known = len(c["old"]) > 0
    pages = full((c["capacity"],), -77, torch.int32)
    off, pages = G.page_table(dev(c["lens"]), dev(c["free"]), c["spare"], dev(c["old"]) if known else None,
                              dev(c["old_pages"]) if known else None, None, pages, stream)
    return host(off), host(pages)


def run_slots(c):
    outs = [full((c["capacity"],), -77, torch.int32) for _ in range(3)]
    got = G.slot_map(device_graph(c["graph"]), dev(c["counts"]), None, *outs)
    return [host(t) for t in got]


class Qkv:
    """A case's tensors on the device; call() makes the call."""

    def __init__(self, c, dtype=None):
        self.c, dtype = c, dtype or c["dtype"]
        n, Hq, Hkv, D = c["n"], c["Hq"], c["Hkv"], c["D"]
        row = TORCH[c["row"]]
        rows = dev(c["rows"])
        body = rows[:, :(Hq + 2 * Hkv) * D].view(n, Hq + 2 * Hkv, D)
        self.q, self.k, self.v = body.split([Hq, Hkv, Hkv], 1)
        if c["in_place"]:
            self.q = self.q.contiguous()
        self.out = self.q if c["in_place"] else full((n, Hq, D), 9, row)
        self.params = G.make_params(Hq, Hkv, D, c["num_pages"], dtype)
        self.pool = G.empty_pool(self.params)
        if dtype == "bf16":
            self.pool.view(torch.int16).fill_(9)
        else:
            self.pool.fill_(9)
        self.words, self.positions = dev(c["words"]), dev(c["positions"])
        self.transform = G.QKTransform(D, dev(c["inv_freq"]), c["interleaved"], *(dev(w) for w in c["weights"]),
                                       c["eps"], float(c["scale"]))

    def call(self, stream=None):
        return G.qkv_append(self.pool, self.q, self.k, self.v, self.positions, self.words, self.transform, self.params,
                            self.out, stream)


class Logits:
    def __init__(self, c):
        self.c, V = c, c["vocab"]
        self.buffer = dev(c["logits"])
        self.logits = self.buffer[:, :V]
        wide = torch.float32 if c["out_f32"] or c["dtype"] == "f32" else torch.bfloat16
        self.out_buffer = self.buffer if c["in_place"] else full(tuple(self.buffer.shape), 9, wide)
        self.out = self.out_buffer[:, :V]
        self.before = host(self.out_buffer).copy()
        bias, masks = c["bias"] or (None,) * 3, c["masks"] or (None, None)
        self.rules = G.LogitRules(dev(c["rep"]), dev(c["freq"]), dev(c["pres"]), dev(c["temp"]), c["prompt"],
                                  *(dev(x) for x in bias), *(dev(x) for x in masks))
        self.graph, self.ids = device_graph(c["graph"]), dev(c["ids"])
        self.branches, self.positions = dev(c["branches"]), dev(c["positions"])

    def call(self, stream=None):
        G.process_logits(self.logits, self.rules, self.graph, self.ids, self.branches, self.positions, self.out,
                         stream=stream)
        return self.out_buffer


@pytest.mark.parametrize("seed", range(3))
def test_page_tables(seed):
    require_gpu()
    rng = np.random.default_rng(100 + seed)
    cases = [U.page_case(rng, bad=i % 4 == 3) for i in range(12)] + [U.page_case(rng, n) for n in (0, 1, 513, 5000)]
    for c in cases:
        U.check_page(c, *run_page(c))


def test_page_table_of_many_segments():
    """More segments than workgroups of the most segments each."""
    require_gpu()
    c = U.page_case(np.random.default_rng(3), 530_000)
    U.check_page(c, *run_page(c))


def test_page_table_grows_in_place_of_a_rollout():
    """Tables of a growing rollout, each from the one before: pages stay, new ones follow, children come."""
    require_gpu()
    rng = np.random.default_rng(8)
    lens, off, pages = np.array([40, 3], np.int32), None, None
    order = rng.permutation(4000).astype(np.int32)
    for step in range(6):
        taken = 0 if off is None else int(off[-1])
        free = dev(order[taken:])
        new_off, new_pages = G.page_table(dev(lens), free, 5, None if off is None else dev(off),
                                          None if off is None else dev(pages))
        o, p = host(new_off), host(new_pages)
        want = S.page_table(lens, 5, np.zeros(0) if off is None else off, np.zeros(0) if off is None else pages,
                            order[taken:])
        np.testing.assert_array_equal(o, want[0])
        np.testing.assert_array_equal(p[:o[-1]], want[1])
        assert (p[o[-1]:] == -1).all() and len(set(p[:o[-1]])) == o[-1]
        off, pages = o, p[:o[-1]]
        lens = np.concatenate([lens + rng.integers(0, 30, len(lens)), rng.integers(0, 50, 3)]).astype(np.int32)


@pytest.mark.parametrize("seed", range(3))
def test_slot_maps(seed):
    require_gpu()
    rng = np.random.default_rng(200 + seed)
    cases = [U.slot_case(rng, bad=i % 3 == 2) for i in range(12)]
    cases.append(U.slot_case(rng, g=U.graph([70000], [[0]], rng), counts=np.array([70000], np.int32)))
    cases.append(U.slot_case(rng, g=U.graph(list(rng.integers(1, 5, 700)), [[i] for i in range(700)], rng)))
    cases.append(U.slot_case(rng, g=U.graph([5], [], rng), counts=None))
    for c in cases:
        U.check_slots(c, *run_slots(c))


def test_slot_map_of_some_outputs():
    require_gpu()
    rng = np.random.default_rng(1)
    g = U.graph([20, 33, 7], [[0, 1], [0, 2]], rng)
    counts = np.array([33, 2], np.int32)
    want = S.slot_map(U.oracle_graph(g), counts, 40)
    for pick in ((0,), (1,), (2,), (0, 2)):
        outs = [full((40,), -77, torch.int32) if i in pick else None for i in range(3)]
        got = G.slot_map(device_graph(g), dev(counts), None, *outs)
        np.testing.assert_array_equal(host(got[0]), want[0])
        for i in range(3):
            assert (got[1 + i] is None) == (i not in pick)
            if i in pick:
                np.testing.assert_array_equal(host(got[1 + i]), want[1 + i])
    _, words, positions, branches = G.slot_map(device_graph(g))
    np.testing.assert_array_equal(host(positions), [52, 26])
    np.testing.assert_array_equal(host(branches), [0, 1])


SHAPES = [(28, 4, 128), (16, 2, 64), (5, 5, 64), (3, 1, 128), (40, 8, 128)]
TURNS = [(1.0, False), (1.0, True), (0.5, False), (0.25, True), (0.0, False)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", SHAPES)
def test_qkv(dtype, Hq, Hkv, D):
    require_gpu()
    rng = np.random.default_rng(D + Hq)
    worst = 0.0
    for i, (share, inter) in enumerate(TURNS):
        for n in (1, 2, 77, 1500 if i == 0 else 5):
            c = U.qkv_case(rng, n, Hq, Hkv, D, dtype, int(share * D), inter, (n % 2 == 1, n != 77),
                           float(rng.choice([1.0, 1.25])), int(rng.choice([3, 4096, 2**31 - 1])),
                           int(rng.choice([0, 8, 64])), in_place=n == 2)
            s = Qkv(c)
            out = s.call()
            U.check_qkv(c, host(out), host(s.pool), 9)
    say(f"[qkv] {dtype} {Hq}/{Hkv} x {D}: within bounds")


@pytest.mark.parametrize("Hq,Hkv,D", SHAPES)
def test_qkv_into_mxfp4_is_append_of_its_bf16_rows(Hq, Hkv, D):
    require_gpu()
    rng = np.random.default_rng(D + Hq)
    for n in (1, 13, 900):
        c = U.qkv_case(rng, n, Hq, Hkv, D, "bf16", D, bool(n % 2))
        if n > 1:
            c["rows"][2, (Hq + Hkv) * D + 7] = 0x7F80
            c["rows"][1, Hq * D + 3] = 0x7FC0
        a, b = Qkv(c), Qkv(c, "mxfp4")
        qa, qb = a.call(), b.call()
        assert torch.equal(qa.view(torch.int16), qb.view(torch.int16))
        there = (c["positions"] >= 0) & (c["words"] >= 0) & (c["words"] < 16 * c["num_pages"])
        words = dev(c["words"][there])
        k, v = G.kv_read(a.pool, words, a.params)
        want = torch.full_like(b.pool, 9)
        G.kv_append(want, k, v, words, b.params)
        assert torch.equal(b.pool, want)


@pytest.mark.parametrize("what", ["zero", "inf", "nan", "huge", "tiny"])
def test_qkv_of_extreme_rows(what):
    """One head's extreme values stay its own; a row of zeros is zero, and large and tiny ones have their norm."""
    require_gpu()
    rng = np.random.default_rng(4)
    c = U.qkv_case(rng, 6, 4, 2, 128, "f32", 128)
    c["positions"][:] = [0, 5, 9, 100, 7, 3]
    value = {"zero": 0.0, "inf": np.inf, "nan": np.nan, "huge": 1e18, "tiny": 1e-25}[what]
    c["rows"][2, :128] = value * (1 if what in ("zero", "inf", "nan") else rng.standard_normal(128))
    s = Qkv(c)
    out = host(s.call())
    if what in ("inf", "nan"):
        assert np.isnan(out[2, 0]).any()
        out[2, 0] = 0
        c["rows"][2, :128] = 0
    elif what == "zero":
        assert (out[2, 0] == 0).all()
    U.check_rows(out, U.qkv_parts(c)[0], c, c["weights"][0], c["positions"] >= 0)


def test_channels_that_do_not_turn_take_nothing_from_others():
    require_gpu()
    rng = np.random.default_rng(6)
    c = U.qkv_case(rng, 3, 2, 1, 128, "bf16", 32, norm=(False, False))
    c["rows"][:, 5] = 0x7F80
    out = host(Qkv(c).call())
    np.testing.assert_array_equal(out[:, 0, 32:], U.qkv_parts(c)[0][:, 0, 32:])


@pytest.mark.parametrize("seed", range(3))
@pytest.mark.parametrize("dtype,wide", [("f32", False), ("bf16", False), ("bf16", True)])
def test_logits(dtype, wide, seed):
    require_gpu()
    rng = np.random.default_rng(300 + seed)
    worst = 0.0
    for i in range(14):
        bad = i % 4 == 3
        g = U.random_graph(rng, 12, bad=bad)
        rows = int(rng.integers(1, 30)) if i else 0
        rules = "".join(x for x in "rfptbm" if rng.random() < 0.7) if i > 1 else "rfptbm"
        drafts = bad or rng.random() < 0.6
        if not drafts:
            rows = min(rows, len(g["po"]) - 1)
        c = U.logits_case(rng, g, rows, int(rng.choice([1, 7, 31, 33, 500, 2049, 5000, 40001])), dtype, wide, rules,
                          int(rng.integers(0, 3)), drafts, int(rng.choice([0, 1, 5])),
                          in_place=not wide and rng.random() < 0.4, bad=bad, biases=int(rng.choice([1, 6, 300])))
        s = Logits(c)
        worst = max(worst, U.check_logits(c, host(s.call()), s.before))
    say(f"[logits] {dtype} wide={wide} seed={seed}: {worst:.3f} of the bound")


def test_logits_of_long_contexts_and_paths():
    require_gpu()
    rng = np.random.default_rng(5)
    long = U.graph([100, 20000, 5], [[0, 1], [0, 2]], rng)
    paths = U.graph(list(rng.integers(0, 4, 150)), [list(range(150)), list(range(149, 19, -1)), [3]], rng)
    for g, vocab, rows in ((long, 41000, 2), (long, 333, 2), (paths, 700, 3)):
        c = U.logits_case(rng, g, rows, vocab, "f32", drafts=False)
        if g is long:
            c["ids"][:] = np.where(rng.random(len(c["ids"])) < 0.95, 300, c["ids"])
        s = Logits(c)
        U.check_logits(c, host(s.call()), s.before)
    c = U.logits_case(rng, long, 3, 333, "f32", rules="fp")
    c["branches"][:], c["positions"][:] = 0, [16482, 16483, 99]
    c["ids"][:] = 7
    s = Logits(c)
    U.check_logits(c, host(s.call()), s.before)


def test_logits_of_extreme_values():
    """Infinities and NaN where they are, and never where the mask forbids; rows that a mask empties."""
    require_gpu()
    rng = np.random.default_rng(9)
    g = U.graph([30, 10], [[0, 1], [0]], rng)
    c = U.logits_case(rng, g, 2, 300, "f32", rules="rfptm", drafts=False)
    c["logits"][:, ::7], c["logits"][:, 1::7], c["logits"][:, 2::7] = np.inf, -np.inf, np.nan
    c["masks"][0][1] = 0xAAAAAAAA
    c["masks"][1][:] = [1, 0]
    out = host(Logits(c).call())
    v = np.arange(300)
    assert (out[0, v % 2 == 0] == -np.inf).all() and (out[1] == -np.inf).all()
    odd = v % 2 == 1
    assert np.isnan(out[0, odd & (v % 7 == 2)]).all()
    assert (out[0, odd & (v % 7 == 0)] == np.inf).all() and (out[0, odd & (v % 7 == 1)] == -np.inf).all()
    assert np.isfinite(out[0, odd & (v % 7 > 2)]).all()


def test_rows_without_penalties_need_no_graph():
    require_gpu()
    rng = np.random.default_rng(2)
    x = dev(U.stored(rng.standard_normal((3, 77)), "f32"))
    out = G.process_logits(x, G.LogitRules(temperature=dev(np.array([0.5, 1, 2], np.float32))))
    np.testing.assert_allclose(host(out), host(x) / np.array([[0.5], [1], [2]]), rtol=2.0 ** -23)
    assert torch.equal(G.process_logits(x, G.LogitRules()), x)
    rows = dev(np.array([0, -1, 5], np.int32))
    out = G.process_logits(x, G.LogitRules(), row_branches=rows)
    assert torch.equal(out[0], x[0]) and (out[1] == 0).all() and torch.equal(out[2], x[2])


def test_calls_on_another_stream():
    """Each call on a stream of its own, behind work that is still filling its inputs there."""
    require_gpu()
    rng = np.random.default_rng(12)
    c, d = U.qkv_case(rng, 300, 28, 4, 128, "bf16", 128), None
    g = U.random_graph(rng, 12)
    d = U.logits_case(rng, g, 6, 5000, "f32")
    a, b = Qkv(c), Logits(d)
    keep = a.positions.clone(), b.logits.clone()
    a.positions.fill_(-1)
    b.logits.zero_()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(2_000_000)
        a.positions.copy_(keep[0])
        b.logits.copy_(keep[1])
        a.call()
        b.call(stream)
    stream.synchronize()
    U.check_qkv(c, host(a.out), host(a.pool), 9)
    U.check_logits(d, host(b.out_buffer), b.before)


def test_captured_steps_replay():
    """Slot map, append and rules in one captured graph: replays follow what the arrays hold by then."""
    require_gpu()
    rng = np.random.default_rng(21)
    Hq, Hkv, D, B, V = 8, 2, 64, 6, 3001
    lens = rng.integers(20, 40, 7).astype(np.int32)
    g = U.graph(lens, [[0, 1 + b] for b in range(B)], rng, spare_pages=2)
    graph = device_graph(g)
    seg_len, new = graph.tensors[0], dev(np.arange(1, 7))
    params = G.make_params(Hq, Hkv, D, g["num_pages"], "bf16")
    pool = torch.zeros_like(G.empty_pool(params))
    rows = torch.randn(B, Hq + 2 * Hkv, D, device="cuda").bfloat16()
    q, k, v = rows.split([Hq, Hkv, Hkv], 1)
    transform = G.QKTransform(D, dev(10000.0 ** (-np.arange(32) / 32)), q_norm=torch.ones(D, device="cuda"))
    ids = dev(rng.integers(0, V, 16 * g["num_pages"]).astype(np.int32))
    logits = torch.randn(B, V, device="cuda")
    rules = G.LogitRules(frequency=torch.rand(B, device="cuda"), repetition=torch.rand(B, device="cuda") + 0.8)
    off = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    words, positions, branches = (torch.zeros(B + 2, dtype=torch.int32, device="cuda") for _ in range(3))
    q_out, out = torch.zeros(B, Hq, D, device="cuda").bfloat16(), torch.zeros(B, V, device="cuda")

    def step():
        G.slot_map(graph, None, off, words, positions, branches)
        G.qkv_append(pool, q, k, v, positions[:B], words[:B], transform, params, q_out)
        G.process_logits(logits, rules, graph, ids, branches[:B], positions[:B], out)

    step()                                                # (loads the kernels)
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured):
        step()
    for i in range(4):
        seg_len[new] += 1
        rows.copy_(torch.randn(rows.shape, device="cuda"))
        logits.copy_(torch.randn(logits.shape, device="cuda"))
        pool.zero_(), q_out.zero_(), out.zero_()
        captured.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (off, words, positions, branches, q_out, pool, out)]
        pool.zero_(), q_out.zero_(), out.zero_()
        step()
        for a, b in zip(got, (off, words, positions, branches, q_out, pool, out)):
            assert torch.equal(a, b), i
        g["seg_len"] = host(seg_len)
        want = S.slot_map(U.oracle_graph(g), None, B + 2)
        np.testing.assert_array_equal(host(words), want[1])
        np.testing.assert_array_equal(host(positions), want[2])


@pytest.mark.parametrize("dtype", ["bf16", "f32", "mxfp4"])
def test_a_rollout_by_these_calls(dtype):
    """A prompt's prefill, its children's steps and their penalties: pages and slots from the device's lengths, queries
    and keys by qkv_append, attention by a plan over the same table, all against the oracle."""
    require_gpu()
    rng = np.random.default_rng(31)
    Hq, Hkv, D, V, eps = 8, 2, 64, 1000, 1e-5
    row = "f32" if dtype == "f32" else "bf16"
    lens = np.array([37, 1, 1, 1], np.int32)              # the prompt, then three children's first tokens
    paths = [[0, 1], [0, 2], [0, 3]]
    num_pages = 20
    free = dev(rng.permutation(num_pages).astype(np.int32))
    off, table = G.page_table(dev(lens), free, 20)
    params = G.make_params(Hq, Hkv, D, num_pages, dtype)
    pool = torch.zeros_like(G.empty_pool(params))
    inv_freq = 10000.0 ** (-np.arange(D // 2) / (D // 2))
    wq, wk = (dev((1 + 0.1 * rng.standard_normal(D)).astype(np.float32)) for _ in range(2))
    transform = G.QKTransform(D, dev(inv_freq), False, wq, wk, eps)
    ids = torch.full((16 * num_pages,), -1, dtype=torch.int32, device="cuda")
    keys = {s: [] for s in range(4)}                      # per segment: (k, v) of its tokens, float64, as stored
    said = {s: [] for s in range(4)}
    seg_len = dev(lens)
    po = dev(np.array([0, 2, 4, 6]))
    ps = dev(np.array(paths, dtype=np.int32).ravel())
    graph = G.DeviceGraph(seg_len, off, table, po, ps, num_pages)
    first = G.DeviceGraph(seg_len, off, table, dev(np.array([0, 1])), dev(np.array([0], np.int32)), num_pages)

    def append(g, counts, total, segs):
        """One step's tokens; their queries by the oracle's norm and rotation."""
        _, words, positions, branches = G.slot_map(g, counts, capacity=total + 3)
        x = U.stored(rng.standard_normal((total + 3, Hq + 2 * Hkv, D)), row)
        t = dev(x)
        q = G.qkv_append(pool, *t.split([Hq, Hkv, Hkv], 1), positions, words, transform, params)
        tokens = dev(rng.integers(0, V, total).astype(np.int32))
        ids[words[:total].long()] = tokens
        p = host(positions)[:total]
        k, v = G.kv_read(pool, words[:total].contiguous(), params)
        made = [(slice(0, Hq), wq, q[:total])] + ([(slice(Hq, Hq + Hkv), wk, k)] if dtype != "mxfp4" else [])
        for heads, w, got in made:
            y, reach = S.norm_rotate(U.values(x[:total, heads], row), p, inv_freq, False, host(w), np.float32(eps), 1.0)
            assert (np.abs(U.values(host(got), row) - y) <= U.qkv_bound(y, reach, row)).all()
        for j, s in enumerate(segs):
            keys[s].append((k[j].double().cpu().numpy(), v[j].double().cpu().numpy()))
            said[s].append(int(tokens[j]))
        return q[:total].contiguous(), positions[:total].contiguous(), branches[:total].contiguous()

    append(first, dev(np.array([37], np.int32)), 37, [0] * 37)
    h_off, h_pages = host(off), host(table)[:int(off[-1])]
    for step in range(5):
        if step:
            seg_len[1:] += 1
        q, positions, branches = append(graph, None, 3, [1, 2, 3])
        now = host(seg_len)
        plan = G.Plan(G.HostGraph(now, h_off, h_pages, [0, 2, 4, 6], np.array(paths).ravel()), params)
        out, lse = torch.empty_like(q), torch.empty(3, Hq, device="cuda")
        plan.run(q, pool, out, lse)
        plan.close()
        logits = torch.randn(3, V, device="cuda")
        f, r = torch.rand(3, device="cuda"), 1 + torch.rand(3, device="cuda")
        z = G.process_logits(logits, G.LogitRules(repetition=r, frequency=f, prompt_segments=1), graph, ids, branches,
                             positions)
        for b in range(3):
            chain = keys[0] + keys[1 + b]
            K, Vv = np.stack([c[0] for c in chain]), np.stack([c[1] for c in chain])
            qq = q[b].double().cpu().numpy()
            o, l = O.attend(qq, K, Vv, D ** -0.5)
            compare(f"step {step} branch {b}", out[b].double().cpu().numpy(), lse[b].double().cpu().numpy(), o, l)
            seen = [(t, True) for t in said[0]] + [(t, False) for t in said[1 + b]]
            want, size = S.logits_row(logits[b].double().cpu().numpy(), seen, float(r[b]), float(f[b]))
            assert (np.abs(z[b].double().cpu().numpy() - want) <= 2.0 ** -21 * size).all()


def test_many_rows_of_drafts():
    """More rows than the device takes at once: several positions a branch, in order and not, with padding between them."""
    require_gpu()
    rng = np.random.default_rng(44)
    g = U.random_graph(rng, 12)
    c = U.logits_case(rng, g, 1300, 1201, "bf16", rules="rfptbm", biases=2)
    c["branches"][:] = np.repeat(rng.integers(-1, len(g["po"]) - 1, 260), 5)
    c["positions"][:] = (rng.integers(0, 60, 260)[:, None] + np.cumsum(rng.choice([0, 1, 2, 40, -3], (260, 5)), 1)).reshape(-1)
    s = Logits(c)
    U.check_logits(c, host(s.call()), s.before)


def test_offsets_beyond_32_bits():
    """Rows of logits, tokens of a projection and pages behind 4 GiB."""
    require_gpu()
    rng = np.random.default_rng(45)
    g = U.graph([40, 3], [[0], [0, 1]], rng)
    rows, V = 9000, 152064
    x = torch.zeros(rows, V, device="cuda")                # 5.5 GB
    last = torch.randn(2, V, device="cuda")
    x[-2:] = last
    branches = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    branches[-2:] = dev(np.array([0, 1], np.int32))
    c = U.logits_case(rng, g, 2, V, "f32", rules="rfptm", drafts=False)
    c["logits"] = host(last)

    def long(a):
        """A rule's values in the last two rows of many."""
        t = torch.zeros(rows, dtype=torch.float32 if a.dtype == np.float32 else torch.int32, device="cuda")
        t[-2:] = dev(a)
        return t
    rules = G.LogitRules(long(c["rep"]), long(c["freq"]), long(c["pres"]), long(c["temp"]), c["prompt"], masks=dev(c["masks"][0]),
                         row_mask=long(c["masks"][1]))
    out = G.process_logits(x, rules, device_graph(g), dev(c["ids"]), branches, None, x)
    U.check_logits(c, host(out[-2:]), c["logits"])
    assert not out[:-2].any()
    del x, out
    # A pool of 5 GB, its last pages; rows 2 MB apart, the last beyond 4 GiB.
    n, Hq, Hkv, D, far = 2100, 2, 2, 128, 1 << 20
    c = U.qkv_case(rng, n, Hq, Hkv, D, "bf16", D)
    c["num_pages"] = 5 * (1 << 30) // (Hkv * 2 * 16 * D * 2)
    c["words"] = (16 * c["num_pages"] - 1 - rng.permutation(4 * n)[:n]).astype(np.int32)
    c["positions"][:] = rng.integers(0, 9000, n)
    rows = torch.zeros(n, far, dtype=torch.bfloat16, device="cuda")
    rows[:, :6 * D] = dev(c["rows"])
    body = rows[:, :6 * D].view(n, 6, D)
    params = G.make_params(Hq, Hkv, D, c["num_pages"], "bf16")
    pool = G.empty_pool(params)
    transform = G.QKTransform(D, dev(c["inv_freq"]), False, *(dev(w) for w in c["weights"]), c["eps"])
    q = G.qkv_append(pool, *body.split([Hq, Hkv, Hkv], 1), dev(c["positions"]), dev(c["words"]), transform, params)
    every = np.ones(n, dtype=bool)
    U.check_rows(host(q), U.qkv_parts(c)[0], c, c["weights"][0], every)
    k, v = G.kv_read(pool, dev(c["words"]), params)
    U.check_rows(host(k), U.qkv_parts(c)[1], c, c["weights"][1], every)
    np.testing.assert_array_equal(host(v), U.qkv_parts(c)[2])


def test_two_calls_at_once():
    """The same call's arrays on two streams: calls keep nothing, so neither disturbs the other."""
    require_gpu()
    rng = np.random.default_rng(46)
    g = U.random_graph(rng, 12)
    a, b = (Logits(U.logits_case(rng, g, 600, 20001, "f32", rules="rfptb")) for _ in range(2))
    p, q = (U.slot_case(rng) for _ in range(2))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, x in zip(streams, (a, b)):
            x.call(s)
    torch.cuda.synchronize()
    for x in (a, b):
        U.check_logits(x.c, host(x.out_buffer), x.before)
    for c in (p, q):
        U.check_slots(c, *run_slots(c))


def test_captured_rules_of_large_slices():
    """Slices whose counts fill half of a CU's LDS, captured and replayed over new logits and positions."""
    require_gpu()
    rng = np.random.default_rng(47)
    g = U.random_graph(rng, 12)
    c = U.logits_case(rng, g, 520, 38001, "f32", rules="rfpt")
    s = Logits(c)
    s.call()
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured):
        s.call()
    for i in range(3):
        c["logits"] = U.stored(rng.standard_normal(c["logits"].shape), "f32")
        c["positions"] = rng.integers(-1, 100, 520).astype(np.int32)
        s.buffer.copy_(dev(c["logits"]))
        s.positions.copy_(dev(c["positions"]))
        s.out_buffer.fill_(9.0)
        captured.replay()
        torch.cuda.synchronize()
        got = s.out_buffer.clone()
        s.out_buffer.fill_(9.0)
        assert torch.equal(s.call(), got), i
    keep = rng.permutation(520)[:40]
    for k in ("logits", "branches", "positions", "rep", "freq", "pres", "temp"):
        c[k] = c[k][keep]
    U.check_logits(c, host(got)[keep], np.full((40, 38001), 9, np.float32))


def test_a_weight_stays_with_its_channel():
    """An infinite weight of a channel that does not turn reaches no other and is not multiplied by an angle."""
    require_gpu()
    rng = np.random.default_rng(48)
    for inter in (False, True):
        c = U.qkv_case(rng, 3, 2, 1, 64, "f32", 16, inter)
        c["positions"][:] = [0, 7, 900]
        c["weights"][0][40] = np.inf
        out = host(Qkv(c).call())
        assert np.isposinf(np.abs(out[:, :, 40])).all()
        c["weights"][0][40] = 0
        out[:, :, 40] = 0
        U.check_rows(out, U.qkv_parts(c)[0], c, c["weights"][0], np.ones(3, dtype=bool))


def test_an_infinite_penalty_bans_what_came_and_nothing_else():
    require_gpu()
    rng = np.random.default_rng(49)
    g = U.graph([30, 10], [[0, 1], [0]], rng)
    for name in ("freq", "pres", "rep"):
        c = U.logits_case(rng, g, 2, 300, "f32", rules="rfp", drafts=False, prompt=0)
        c["ids"][:] = rng.integers(0, 40, len(c["ids"]))
        c["logits"] = -np.abs(c["logits"]) - 1
        c["rep"][:], c["freq"][:], c["pres"][:] = 1, 0, 0
        c[name][:] = np.inf
        out = host(Logits(c).call())
        for r in range(2):
            came = {v for v, _ in S.context(U.oracle_graph(g), r, None, c["ids"], 0)}
            gone = np.isin(np.arange(300), list(came))
            assert (out[r, gone] == -np.inf).all() and (out[r, ~gone] == c["logits"][r, ~gone]).all(), name
