"""Outputs that a call of the binding makes itself are made on the stream that the call goes to: on another one a fill
could run after the call, and memory could be taken that earlier work there still uses (CPU: where each is made)."""
import contextlib
import types

import numpy as np
import pytest

from paper_2606_18954_amd import graphattn as G

torch = pytest.importorskip("torch")
STREAM = types.SimpleNamespace(cuda_stream=7)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def graph():
    """A device graph without its device: two branches of one segment."""
    g = object.__new__(G.DeviceGraph)
    g.tensors, g.num_segments, g.num_branches, g.num_pages, g.ref = (i32(1),), 1, 2, 3, None
    return g


def without(cls, **fields):
    """An object of the library without its device memory."""
    x = object.__new__(cls)
    x.handle, x.lib = None, G.load_library()
    for name, value in fields.items():
        setattr(x, name, value)
    return x


def calls(stream):
    """Every call that makes outputs; host tensors are refused after they were made."""
    p = G.make_params(4, 2, 64, 3, "bf16")
    pool, rows = G.empty_pool(p, "cpu"), torch.zeros(2, 8, 64, dtype=torch.bfloat16)
    q, k, v = rows.split([4, 2, 2], 1)
    host = G.HostGraph([20], [0, 2], [0, 1], [0, 1, 2], [0, 0])
    forest, z, labels = G.HostForest([-1, 0]), torch.zeros(2, 64, dtype=torch.bfloat16), i32(2)
    f = without(G.Forest, host=forest)
    e = without(G.Evict, offsets=np.array([0, 4]), num_pages=3)
    rules = object.__new__(G.LogitRules)
    rules.rows, rules.vocab, rules.counted, rules.ref, rules.device = None, None, False, None, None
    s, two, one, free, g = {"stream": stream}, i32(2), i32(1), i32(3), graph()
    x, mass, turn = torch.zeros(2, 9), torch.zeros(48), G.QKTransform(64)
    return {
        "decode": lambda: G.decode(q, pool, host, p, **s), "extend": lambda: G.extend(q, pool, host, [1, 1], p, **s),
        "kv_read": lambda: G.kv_read(pool, two, p, **s), "page_table": lambda: G.page_table(one, free, **s),
        "slot_map": lambda: G.slot_map(g, **s),
        "qkv_append": lambda: G.qkv_append(pool, q, k, v, two, two, turn, p, **s),
        "process_logits": lambda: G.process_logits(x, rules, **s),
        "equivalence_classes": lambda: G.equivalence_classes(z, forest, 0.9, **s),
        "graph_suffix": lambda: G.graph_suffix(labels, forest, **s), "classes": lambda: f.classes(z, 0.9, **s),
        "advantages": lambda: f.advantages(labels, z, None, 0.5, 0.5, **s), "select": lambda: e.select(mass, **s),
    }


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("name", sorted(calls(None)))
def test_outputs_are_made_on_the_stream_of_the_call(name, given, monkeypatch):
    call = calls(STREAM if given else None)[name]
    on, made = [], []

    @contextlib.contextmanager
    def use(stream):
        on.append(getattr(stream, "cuda_stream", stream))
        yield
        on.pop()

    def recorded(make):
        def wrapped(*a, **k):
            made.append(on[-1] if on else None)
            return make(*a, **k)
        return wrapped
    monkeypatch.setattr(torch.cuda, "stream", use)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, *a, **k: types.SimpleNamespace(cuda_stream=handle))
    monkeypatch.setattr(G, "_stream_handle", lambda stream, t=None: 0)
    for fn in ("empty", "zeros", "full"):
        monkeypatch.setattr(torch, fn, recorded(getattr(torch, fn)))
    with pytest.raises((ValueError, G.GraphAttnError)):
        call()
    assert made and set(made) == {7 if given else None}, made
