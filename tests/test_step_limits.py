"""Sizes that one launch of the calls between two attention calls cannot take are refused by the call itself (CPU: a refused
call reads nothing)."""
import ctypes

import pytest

from paper_2606_18954_amd import graphattn as G

FAKE = 1 << 20                           # aligned, never dereferenced by a refused call


@pytest.mark.parametrize("rows,vocab,biases", [(1 << 22, 100, 0), ((1 << 31) - 1, 7, 0), (1 << 21, 38913, 0), (1 << 21, 36865, 5),
                                               (1 << 20, 152064, 0), (1024, (1 << 28) - 1, 0)])
def test_logits_of_more_workgroups_than_a_launch_has(rows, vocab, biases):
    """1024 threads a workgroup, fewer than 2^32 threads in a launch."""
    lib = G.load_library()
    rules = G.LogitRulesC(None, None, None, FAKE, 0, FAKE if biases else None, FAKE if biases else None,
                          FAKE if biases else None, biases, None, 0, 0, None)
    out = FAKE + 4 * rows * vocab
    got = lib.graphattn_process_logits(FAKE, vocab, rows, vocab, G.GA_F32, ctypes.byref(rules), None, None, None, None, out, vocab,
                                       0, None)
    assert got == G.GA_EUNSUPPORTED and "rows" in G.last_error()


@pytest.mark.parametrize("n", [(1 << 26) - 3, 1 << 26, 1 << 28])
def test_tokens_of_more_workgroups_than_a_launch_has(n):
    """256 threads for four tokens."""
    lib = G.load_library()
    p, t = G.make_params(1, 1, 64, 9, "bf16"), G.QKTransformC(0, 0, 0.0, 1.0, None, None, None)
    out = FAKE + 2 * 64 * n
    got = lib.graphattn_qkv_append(FAKE, FAKE, FAKE, FAKE, 64, 64, 64, FAKE, FAKE, n, out, ctypes.byref(t), ctypes.byref(p), None)
    assert got == G.GA_EUNSUPPORTED and "tokens" in G.last_error()
