"""Tensors of two devices in one of the calls between two attention calls are refused, each tensor of each call (CPU:
tensors that say that they are on a device, and a library that must not be called)."""
import pytest

from paper_2606_18954_amd import graphattn as G

torch = pytest.importorskip("torch")


class On(torch.Tensor):
    """A tensor of the host that says that it is on a device."""
    at = 0
    is_cuda = property(lambda t: t.at >= 0)

    def get_device(t):
        return t.at


def on(t, device=0):
    t = t.as_subclass(On)
    t.at = device
    return t


def i32(*shape, at=0):
    return on(torch.zeros(shape, dtype=torch.int32), at)


def i64(*shape, at=0):
    return on(torch.zeros(shape, dtype=torch.int64), at)


def f32(*shape, at=0):
    return on(torch.zeros(shape), at)


class Library:
    def __getattr__(self, name):
        def called(*a):
            raise AssertionError(f"{name} was called")
        return called


@pytest.fixture(autouse=True)
def library(monkeypatch):
    monkeypatch.setattr(G, "_lib", Library())
    monkeypatch.setattr(G, "_stream_handle", lambda stream, t=None: 0)


def graph(**where):
    at = {k: where.get(k, 0) for k in ("seg_len", "off", "pages", "po", "ps")}
    return G.DeviceGraph(i32(3, at=at["seg_len"]), i64(4, at=at["off"]), i32(9, at=at["pages"]), i64(3, at=at["po"]),
                         i32(4, at=at["ps"]), 9)


def rules(**where):
    at = lambda k: where.get(k, 0)  # noqa: E731
    return G.LogitRules(f32(3, at=at("rep")), f32(3, at=at("freq")), f32(3, at=at("pres")), f32(3, at=at("temp")), 0,
                        i64(4, at=at("bo")), i32(2, at=at("bt")), f32(2, at=at("bv")), i32(2, 2, at=at("masks")),
                        i32(3, at=at("row_mask")))


def transform(**where):
    at = lambda k: where.get(k, 0)  # noqa: E731
    return G.QKTransform(64, on(torch.zeros(32, dtype=torch.float64), at("freq")), False, f32(64, at=at("qn")),
                         f32(64, at=at("kn")))


REFUSED = "device"


def check(make, names):
    """make(**where) reaches the library with every tensor on device 0, and is refused with any one of them on device 1."""
    for name in names:
        with pytest.raises(ValueError, match=REFUSED):
            make(**{name: 1})


@pytest.mark.parametrize("make,names", [(graph, ("off", "pages", "po", "ps", "seg_len")),
                                        (rules, ("freq", "pres", "temp", "bo", "bt", "bv", "masks", "row_mask", "rep")),
                                        (transform, ("qn", "kn", "freq"))])
def test_arrays_of_two_devices(make, names):
    make()
    check(make, names)


def reaches(call):
    """The call with every tensor on device 0, and on device 1, goes to the library."""
    for at in (0, 1):
        with pytest.raises(AssertionError, match="was called"):
            call(at)


def test_page_table():
    names = ("lens", "free", "old", "old_pages", "off", "pages")

    def call(base=0, **where):
        at = {k: where.get(k, base) for k in names}
        return G.page_table(i32(3, at=at["lens"]), i32(9, at=at["free"]), 0, i64(3, at=at["old"]), i32(4, at=at["old_pages"]),
                            i64(4, at=at["off"]), i32(13, at=at["pages"]))
    reaches(call)
    check(call, names)


def test_slot_map():
    names = ("counts", "off", "words", "pos", "branches", "graph")

    def call(base=0, **where):
        at = {k: where.get(k, base) for k in names}
        g = graph(**{k: at["graph"] for k in ("seg_len", "off", "pages", "po", "ps")})
        return G.slot_map(g, i32(2, at=at["counts"]), i32(3, at=at["off"]), i32(5, at=at["words"]), i32(5, at=at["pos"]),
                          i32(5, at=at["branches"]))
    reaches(call)
    check(call, names)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "mxfp4"])
def test_qkv_append(dtype):
    names = ("pool", "q", "k", "v", "pos", "words", "transform", "out")
    p, row = G.make_params(4, 2, 64, 3, dtype), torch.float32 if dtype == "f32" else torch.bfloat16
    pool = torch.zeros(3, 2, 17 * 64, dtype=torch.uint8) if dtype == "mxfp4" else torch.zeros(3, 2, 2, 16, 64, dtype=row)

    def call(base=0, **where):
        at = {k: where.get(k, base) for k in names}
        x = lambda name, heads: on(torch.zeros(5, heads, 64, dtype=row), at[name])  # noqa: E731
        t = transform(**{k: at["transform"] for k in ("freq", "qn", "kn")})
        return G.qkv_append(on(pool, at["pool"]), x("q", 4), x("k", 2), x("v", 2), i32(5, at=at["pos"]), i32(5, at=at["words"]), t,
                            p, x("out", 4))
    reaches(call)
    check(call, names)


def test_process_logits():
    names = ("logits", "rules", "graph", "ids", "branches", "pos", "out")

    def call(base=0, **where):
        at = {k: where.get(k, base) for k in names}
        r = rules(**{k: at["rules"] for k in ("rep", "freq", "pres", "temp", "bo", "bt", "bv", "masks", "row_mask")})
        g = graph(**{k: at["graph"] for k in ("seg_len", "off", "pages", "po", "ps")})
        return G.process_logits(f32(3, 64, at=at["logits"]), r, g, i32(144, at=at["ids"]), i32(3, at=at["branches"]),
                                i32(3, at=at["pos"]), f32(3, 64, at=at["out"]))
    reaches(call)
    check(call, names)


def test_tensors_of_the_host_are_refused_as_such():
    for make, name in ((graph, "ps"), (rules, "bv"), (transform, "kn")):
        with pytest.raises(ValueError, match="GPU"):
            make(**{name: -1})
