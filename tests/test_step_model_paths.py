"""The kernels between two attention calls on the CPU model of the device, as in test_step_model.py: calls of sizes and
values that take other ways through them."""
import numpy as np
import pytest

import step_util as U
from oracle import cache_oracle as C
from test_step_model import _run, driver, pytestmark  # noqa: F401 (the fixture and the mark)


def norm_cases(rng, D, dtype):
    """Heads whose squares leave float32's range: every size of value that the type has, one a head, with an eps of 0 and
    one below the smallest normal number, and with one that is far larger than the squares."""
    sizes = [1e-20, 1e-22, 3e-30, 1e-37, 1e18, 1e20, 3e37, 1.0] + ([3e-42] if dtype == "f32" else [])
    for eps in (0.0, 1e-40, 1e-6):
        for inter in (False, True):
            c = U.qkv_case(rng, 5, 9, 3, D, dtype, D // 2, inter, eps=eps, far=1000)
            c["positions"][:], c["words"][:] = rng.integers(0, 1000, 5), rng.permutation(16)[:5]
            if eps == 1e-6:
                sizes = [s for s in sizes if s >= 1e-30]      # (below, a result is no normal number)
            heads = rng.choice(sizes, (5, 15, 1))
            heads[0, :9, 0] = np.resize(sizes, 9)
            c["rows"] = U.stored((rng.standard_normal((5, 15, D)) * heads).reshape(5, -1), c["row"])
            yield c


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_of_values_whose_squares_leave_float32(driver, tmp_path, dtype, D):  # noqa: F811
    cases = list(norm_cases(np.random.default_rng(D), D, dtype))
    for c, (pool, q_out) in zip(cases, _run(driver, cases, str(tmp_path / "x"))):
        U.check_qkv(c, q_out.reshape(c["n"], 9, D), pool, 9)


def many_tokens(dtype, n):
    """So many tokens that a workgroup takes four, the last one fewer; some words and positions outside."""
    rng = np.random.default_rng(n)
    Hq, Hkv, D = {"bf16": (6, 2, 64), "f32": (5, 1, 64), "mxfp4": (2, 1, 128)}[dtype]
    c = U.qkv_case(rng, n, Hq, Hkv, D, "bf16" if dtype == "mxfp4" else dtype, D, n % 2 == 0, pad=8)
    c["positions"][rng.integers(0, n, 40)] = -1
    c["words"][rng.integers(0, n, 40)] = -1
    c["positions"][-1], c["words"][-1] = 77, 5 if 5 not in c["words"][:-1] else c["words"][-1]
    return c


@pytest.mark.parametrize("n", [4096, 4097, 4099])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_four_tokens_a_workgroup(driver, tmp_path, dtype, n):  # noqa: F811
    c = many_tokens(dtype, n)
    (pool, q_out), = _run(driver, [c], str(tmp_path / "x"))
    U.check_qkv(c, q_out.reshape(n, c["Hq"], c["D"]), pool, 9)


def test_four_tokens_a_workgroup_into_mxfp4(driver, tmp_path):  # noqa: F811
    c = many_tokens("mxfp4", 4099)
    (pool, q1), (codes, q2) = _run(driver, [c, dict(c, dtype="mxfp4")], str(tmp_path / "x"))
    np.testing.assert_array_equal(q1, q2)
    there = (c["positions"] >= 0) & (c["words"] >= 0) & (c["words"] < 16 * c["num_pages"])
    w = c["words"][there]
    k, v = (U.values(pool[w // 16, :, i, w % 16], "bf16") for i in (0, 1))
    np.testing.assert_array_equal(codes, C.append(np.full_like(codes, 9), k, v, w))


def many_branches(rng, bad):
    """More branches than workgroups of 256 threads take, with counts and without, and as many segments."""
    for counts in ("drawn", None):
        B, n_seg = 4097 + int(rng.integers(0, 900)), 300
        paths = [list(rng.integers(0, n_seg, rng.integers(1, 4))) for _ in range(B)]
        g = U.graph(list(rng.integers(1, 40, n_seg)), paths, rng)
        if bad:
            g["ps"][rng.integers(0, len(g["ps"]), 50)] = rng.choice([-1, n_seg, 2**31 - 1], 50)
            g["po"][rng.integers(0, B + 1, 20)] = rng.choice(np.array([-1, 2**40, 2**63 - 1]), 20)
        if counts is not None:
            counts = rng.integers(-1 if bad else 0, 9, B).astype(np.int32)
        yield U.slot_case(rng, g=g, counts=counts)


@pytest.mark.parametrize("bad", [False, True])
def test_slots_of_many_branches(driver, tmp_path, bad):  # noqa: F811
    cases = list(many_branches(np.random.default_rng(70 + bad), bad))
    for c, out in zip(cases, _run(driver, cases, str(tmp_path / "x"))):
        U.check_slots(c, *out)


def test_page_table_of_many_segments(driver, tmp_path):  # noqa: F811
    rng = np.random.default_rng(72)
    cases = [U.page_case(rng, 4097), U.page_case(rng, 4700, bad=True)]
    for c, out in zip(cases, _run(driver, cases, str(tmp_path / "x"))):
        U.check_page(c, *out)


def long_bias_lists(rng, dtype, wide, vocab=5003, rows=5):
    """Rows of as many biases as LDS holds, one more, and many more, some tokens twice, some outside the vocabulary; beside
    them a row of three and one of none."""
    c = U.logits_case(rng, U.random_graph(rng, 12), rows, vocab, dtype, wide, rules="rfptbm", drafts=True)
    lists = []
    for n in [512, 513, 2000, 3, 0][:rows]:
        tokens = rng.permutation(vocab)[:n]
        tokens[:n // 8] = tokens[n // 8:2 * (n // 8)]
        tokens[n // 3:n // 3 + min(n, 4) // 2] = -1
        tokens[n // 2:n // 2 + min(n, 4) // 2] = vocab
        lists.append(np.sort(tokens))
    off = np.concatenate([[0], np.cumsum([len(t) for t in lists])]).astype(np.int64)
    c["bias"] = (off, np.concatenate(lists).astype(np.int32), rng.normal(0, 4, int(off[-1])).astype(np.float32))
    return c


@pytest.mark.parametrize("dtype,wide", [("f32", False), ("bf16", False), ("bf16", True)])
def test_long_bias_lists(driver, tmp_path, dtype, wide):  # noqa: F811
    rng = np.random.default_rng(73)
    cases = [long_bias_lists(rng, dtype, wide), long_bias_lists(rng, dtype, wide, vocab=2501)]
    # (counts beyond 14 bits: the slice in two halves, the list beside both)
    long = U.graph([100, 20000, 5], [[0, 1], [0, 2]], rng)
    c = dict(long_bias_lists(rng, dtype, wide), graph=long, ids=rng.integers(0, 400, 16 * long["num_pages"]).astype(np.int32))
    c["branches"], c["positions"] = np.array([0, 0, 1, 0, 1], np.int32), np.array([20099, 16700, 99, 2**31 - 1, 60], np.int32)
    for c, (out,) in zip(cases + [c], _run(driver, cases + [c], str(tmp_path / "x"))):
        U.check_logits(c, out, np.full_like(out, 9))


def large_slices(rng, dtype, wide, rows=516, vocab=17001):
    """So many rows that each is one workgroup's, and so long that its threads load more than once."""
    g = U.random_graph(rng, 12)
    c = U.logits_case(rng, g, rows, vocab, dtype, wide, rules="rfptbm", biases=20, pad=3)
    c["positions"][rng.integers(0, rows, 9)] = -1
    return c


@pytest.mark.parametrize("dtype,wide", [("f32", False), ("bf16", False), ("bf16", True)])
def test_large_slices(driver, tmp_path, dtype, wide):  # noqa: F811
    c = large_slices(np.random.default_rng(74), dtype, wide)
    (out,), = _run(driver, [c], str(tmp_path / "x"))
    keep = np.random.default_rng(1).permutation(516)[:60]
    U.check_logits(rows_of(c, keep), out[keep], np.full_like(out[keep], 9))


def rows_of(c, keep):
    """The case of some of a case's rows."""
    c = dict(c, **{k: c[k][keep] for k in ("logits", "branches", "positions", "rep", "freq", "pres", "temp")})
    off, tokens, vals = c["bias"]
    pick = [np.arange(off[r], off[r + 1]) for r in keep]
    at = np.concatenate(pick + [np.zeros(0, np.int64)]).astype(np.int64)
    c["bias"] = (np.concatenate([[0], np.cumsum([len(p) for p in pick])]).astype(np.int64), tokens[at], vals[at])
    c["masks"] = (c["masks"][0], c["masks"][1][keep])
    return c
