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
