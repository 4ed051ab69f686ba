"""What the Python binding refuses before a pointer is taken (no GPU: these are tensors of the host, which the
binding refuses last)."""
import pytest

from paper_2606_18954_amd import graphattn as G

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("name", ["MXFP4", "fp4", "bfloat16", "float32", "", None, 2])
def test_a_type_that_is_none_is_refused(name):
    """(Taken for another type, the kernels would read past a smaller pool's end.)"""
    with pytest.raises(ValueError, match="mxfp4"):
        G.make_params(4, 2, 64, 3, name)


def _pool(p):
    return G.empty_pool(p, "cpu")


GRAPH = G.HostGraph([20], [0, 2], [0, 1], [0, 1], [0])
ROW = {"f32": torch.float32, "bf16": torch.bfloat16, "mxfp4": torch.bfloat16}


@pytest.fixture
def plan():
    """A plan's calls without its device memory."""
    def make(p, rows=1):
        pl = object.__new__(G.Plan)
        pl.handle, pl.lib, pl.params = None, G.load_library(), p
        pl._keep(p, rows)
        return pl
    return make


def _calls(p, pool, plan):
    """Every call that reads or writes a pool, with arguments that fit params p."""
    q = torch.zeros(1, 4, 64, dtype=ROW[_name(p)])
    kv, words = torch.zeros(2, 2, 64, dtype=q.dtype), torch.zeros(2, dtype=torch.int32)
    out, lse, mass = torch.zeros_like(q), torch.zeros(1, 4), torch.zeros(48)
    return [lambda: G.decode(q, pool, GRAPH, p), lambda: G.decode_static(q, pool, GRAPH, p, out, lse),
            lambda: G.extend(q, pool, GRAPH, [1], p), lambda: plan(p).run(q, pool, out, lse),
            lambda: plan(p).run_mass(q, pool, lse, mass), lambda: G.kv_append(pool, kv, kv, words, p),
            lambda: G.kv_copy(pool, words, words, p), lambda: G.kv_read(pool, words, p, kv, kv)]


def _name(p):
    return next(n for n, d in G.DTYPES.items() if d == p.dtype)


@pytest.mark.parametrize("params", ["f32", "bf16", "mxfp4"])
@pytest.mark.parametrize("pool", ["f32", "bf16", "mxfp4", "short"])
def test_a_pool_of_another_type_or_size_is_refused(params, pool, plan):
    p = G.make_params(4, 2, 64, 3, params)
    tensor = _pool(p)[:-1] if pool == "short" else _pool(G.make_params(4, 2, 64, 3, pool))
    for call in _calls(p, tensor, plan):
        # (the right pool is refused for being the host's, which comes last)
        with pytest.raises(ValueError, match="GPU" if params == pool else " pool is a "):
            call()


@pytest.mark.parametrize("params", ["f32", "bf16", "mxfp4"])
def test_rows_of_another_type_or_size_are_refused(params, plan):
    p = G.make_params(4, 2, 64, 3, params)
    pool, row = _pool(p), ROW[params]
    other = torch.bfloat16 if params == "f32" else torch.float32
    words = torch.zeros(2, dtype=torch.int32)
    good = {"q": torch.zeros(2, 4, 64, dtype=row), "out": torch.zeros(2, 4, 64, dtype=row), "lse": torch.zeros(2, 4)}
    two = G.HostGraph([20], [0, 2], [0, 1], [0, 1, 2], [0, 0])

    def attend(**new):
        a = {**good, **new}
        for call in (lambda: plan(p, 2).run(a["q"], pool, a["out"], a["lse"]),
                     lambda: G.decode(a["q"], pool, two, p, a["out"], a["lse"]),
                     lambda: G.decode_static(a["q"], pool, two, p, a["out"], a["lse"])):
            yield call
    for new, match in (({"q": good["q"].to(other)}, "rows beside"), ({"q": good["q"][:1]}, "of q"),
                       ({"out": good["out"].to(other)}, "out must be"), ({"out": good["out"][:1]}, "of out"),
                       ({"lse": good["lse"].double()}, "lse must be"), ({"lse": good["lse"][:1]}, "lse must be")):
        for call in attend(**new):
            with pytest.raises(ValueError, match=match):
                call()
    with pytest.raises(ValueError, match="of q"):
        G.extend(good["q"], pool, GRAPH, [3], p)
    wide = G.make_params(4, 2, 64, 3, params, out_f32=True)
    if params != "f32":
        with pytest.raises(ValueError, match="out must be"):
            plan(wide, 2).run(good["q"], pool, good["out"], good["lse"])
    with pytest.raises(ValueError, match="GPU"):
        plan(wide, 2).run(good["q"], pool, good["out"].float(), good["lse"])
    kv = torch.zeros(2, 2, 64, dtype=row)
    for k, v in ((kv.to(other), kv), (kv, kv.to(other))):
        with pytest.raises(ValueError, match="rows beside"):
            G.kv_append(pool, k, v, words, p)
    for k, v in ((kv[:, :1], kv), (kv, kv[..., :32])):
        with pytest.raises(ValueError, match="Hkv, D"):
            G.kv_append(pool, k, v, words, p)
    for call in (lambda: G.kv_append(pool, kv, kv, words.long(), p), lambda: G.kv_copy(pool, words.long(), words, p),
                 lambda: G.kv_copy(pool, words, words.long(), p)):
        with pytest.raises(ValueError, match="int32"):
            call()


@pytest.mark.parametrize("D", [64, 128])
def test_an_mxfp4_page_is_17_of_64_of_a_bf16_page(D):
    pages = {n: G.kv_page_bytes(G.make_params(4, 4, D, 1, n)) for n in ("bf16", "mxfp4")}
    assert 64 * pages["mxfp4"] == 17 * pages["bf16"]
