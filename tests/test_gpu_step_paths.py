"""The calls between two attention calls on the GPU: sizes and values that take other ways through their kernels."""
import numpy as np
import pytest
import torch

import step_util as U
from gpu_util import require_gpu
from paper_2606_18954_amd import graphattn as G
from test_gpu_step import Logits, Qkv, dev, host, run_page, run_slots
from test_step_model_paths import large_slices, long_bias_lists, many_branches, many_tokens, norm_cases, rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_of_values_whose_squares_leave_float32(dtype, D):
    require_gpu()
    for c in norm_cases(np.random.default_rng(D), D, dtype):
        s = Qkv(c)
        U.check_qkv(c, host(s.call()), host(s.pool), 9)


@pytest.mark.parametrize("n", [4096, 4097, 4099])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_four_tokens_a_workgroup(dtype, n):
    require_gpu()
    c = many_tokens(dtype, n)
    s = Qkv(c)
    U.check_qkv(c, host(s.call()), host(s.pool), 9)


def test_four_tokens_a_workgroup_into_mxfp4():
    require_gpu()
    c = many_tokens("mxfp4", 4099)
    a, b = Qkv(c), Qkv(c, "mxfp4")
    assert torch.equal(a.call().view(torch.int16), b.call().view(torch.int16))
    there = (c["positions"] >= 0) & (c["words"] >= 0) & (c["words"] < 16 * c["num_pages"])
    words = dev(c["words"][there])
    k, v = G.kv_read(a.pool, words, a.params)
    want = torch.full_like(b.pool, 9)
    G.kv_append(want, k, v, words, b.params)
    assert torch.equal(b.pool, want)


@pytest.mark.parametrize("bad", [False, True])
def test_slots_of_many_branches(bad):
    require_gpu()
    for c in many_branches(np.random.default_rng(70 + bad), bad):
        U.check_slots(c, *run_slots(c))


def test_page_table_of_a_bad_old_table():
    """Old offsets outside the old pages, in a table that workgroups of 1024 threads make."""
    require_gpu()
    c = U.page_case(np.random.default_rng(72), 4700, bad=True)
    U.check_page(c, *run_page(c))


@pytest.mark.parametrize("dtype,wide", [("f32", False), ("bf16", False), ("bf16", True)])
def test_long_bias_lists(dtype, wide):
    require_gpu()
    rng = np.random.default_rng(73)
    cases = [long_bias_lists(rng, dtype, wide), long_bias_lists(rng, dtype, wide, vocab=2501)]
    long = U.graph([100, 20000, 5], [[0, 1], [0, 2]], rng)
    c = dict(long_bias_lists(rng, dtype, wide), graph=long, ids=rng.integers(0, 400, 16 * long["num_pages"]).astype(np.int32))
    c["branches"], c["positions"] = np.array([0, 0, 1, 0, 1], np.int32), np.array([20099, 16700, 99, 2**31 - 1, 60], np.int32)
    for c in cases + [c]:
        s = Logits(c)
        U.check_logits(c, host(s.call()), s.before)


@pytest.mark.parametrize("dtype,wide", [("f32", False), ("bf16", False), ("bf16", True)])
def test_large_slices(dtype, wide):
    require_gpu()
    c = large_slices(np.random.default_rng(74), dtype, wide)
    s = Logits(c)
    out = host(s.call())
    keep = np.random.default_rng(1).permutation(516)[:60]
    U.check_logits(rows_of(c, keep), out[keep], s.before[keep])
