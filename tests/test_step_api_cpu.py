"""Host checks of the calls between two attention calls: the header's entry points are exported and plain C, malformed
arguments are refused before any device work, and the binding refuses tensors that do not fit."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2606_18954_amd import graphattn as G

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20                           # aligned, never dereferenced by a refused call
ODD = FAKE + 2


def test_every_declared_symbol_is_exported():
    lib = G.load_library()
    syms = G.header_symbols("graphattn_step.h")
    assert set(syms) == {"graphattn_page_table", "graphattn_slot_map", "graphattn_qkv_append",
                         "graphattn_process_logits"}
    for s in syms:
        assert hasattr(lib, s), s


def _refused(call, good, bad, statuses):
    """Every change of `bad` to the arguments `good` is refused with its status, and says why."""
    for (change, status) in zip(bad, statuses):
        assert call(**{**good, **change}) == status, change
        assert G.last_error(), change


def test_page_table_errors():
    lib = G.load_library()

    def call(lens=FAKE, S=5, spare=0, oo=FAKE, op=FAKE, So=3, nop=9, free=FAKE, nf=9, off=FAKE + 512, pages=FAKE + 1024,
             cap=9):
        return lib.graphattn_page_table(lens, S, spare, oo, op, So, nop, free, nf, off, pages, cap, None)
    bad = [dict(S=-1), dict(spare=-1), dict(nop=-1), dict(nf=-1), dict(cap=-1), dict(So=6), dict(So=-1), dict(lens=None),
           dict(oo=None), dict(op=None), dict(free=None), dict(off=None), dict(pages=None), dict(lens=ODD),
           dict(off=FAKE + 516), dict(oo=FAKE + 4), dict(pages=ODD), dict(pages=FAKE + 32), dict(off=FAKE + 16),
           dict(pages=FAKE + 520)]
    _refused(call, {}, bad, [G.GA_EINVAL] * len(bad))
    assert call(nop=1 << 31) == G.GA_EUNSUPPORTED


def _graph(**change):
    c = G.DeviceGraphC(3, 2, 9, 4, 9, FAKE, FAKE, FAKE, FAKE, FAKE)
    for k, v in change.items():
        setattr(c, k, v)
    return c


BAD_GRAPHS = [dict(num_segments=-1), dict(num_branches=-1), dict(num_table_pages=-1), dict(num_path_segs=-1),
              dict(num_pages=-1), dict(seg_len=None), dict(seg_page_offsets=None), dict(seg_pages=None),
              dict(path_offsets=None), dict(path_segs=None), dict(seg_len=ODD), dict(path_offsets=FAKE + 4)]


def test_slot_map_errors():
    lib = G.load_library()

    def call(g=_graph(), counts=FAKE, off=FAKE + 512, words=FAKE + 1024, pos=FAKE + 2048, branches=FAKE + 4096, cap=7):
        return lib.graphattn_slot_map(ctypes.byref(g) if g else None, counts, off, words, pos, branches, cap, None)
    bad = [dict(g=None), dict(off=None), dict(cap=-1), dict(off=ODD), dict(words=ODD), dict(counts=ODD),
           dict(words=FAKE), dict(pos=FAKE + 1048), dict(branches=FAKE + 520), dict(off=FAKE + 24)]
    bad += [dict(g=_graph(**x)) for x in BAD_GRAPHS]
    _refused(call, {}, bad, [G.GA_EINVAL] * len(bad))
    assert call(g=_graph(num_pages=(1 << 27) + 1)) == G.GA_EUNSUPPORTED


def test_qkv_append_errors():
    lib = G.load_library()
    p = G.make_params(8, 2, 64, 9, "bf16")

    def call(pool=FAKE, q=FAKE, k=FAKE, v=FAKE, qs=768, ks=768, vs=768, pos=FAKE, words=FAKE, n=3, out=FAKE + 4096, params=p,
             t={}, transform=True):
        c = G.QKTransformC(64, 0, 1e-6, 1.0, FAKE, FAKE, FAKE)
        for name, value in t.items():
            setattr(c, name, value)
        return lib.graphattn_qkv_append(pool, q, k, v, qs, ks, vs, pos, words, n, out,
                                        ctypes.byref(c) if transform else None, ctypes.byref(params) if params else None,
                                        None)
    bad = [dict(pool=None), dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(words=None), dict(out=None),
           dict(params=None), dict(transform=False), dict(n=-1), dict(qs=-8), dict(ks=9), dict(vs=4), dict(q=FAKE + 8),
           dict(out=FAKE + 8), dict(pos=ODD), dict(out=FAKE), dict(out=FAKE + 1024), dict(k=FAKE + 4112), dict(v=FAKE + 4096), dict(t=dict(rotary_dim=-2)), dict(t=dict(rotary_dim=66)),
           dict(t=dict(rotary_dim=31)), dict(t=dict(interleaved=2)), dict(t=dict(norm_eps=-1e-6)),
           dict(t=dict(norm_eps=float("nan"))), dict(t=dict(rotary_scale=float("inf"))), dict(t=dict(inv_freq=None)),
           dict(t=dict(inv_freq=FAKE + 4)), dict(t=dict(q_weight=FAKE + 4)), dict(t=dict(k_weight=FAKE + 8)),
           dict(params=G.make_params(8, 3, 64, 9, "bf16"))]
    _refused(call, {}, bad, [G.GA_EINVAL] * len(bad))
    for change in (dict(t=dict(rotary_dim=8)), dict(n=(1 << 28) + 1), dict(params=G.make_params(8, 2, 96, 9, "bf16"))):
        assert call(**change) == G.GA_EUNSUPPORTED, change
    assert call(n=0) == G.GA_OK and call(n=0, pool=None, q=None, pos=None, out=None) == G.GA_OK


def test_process_logits_errors():
    lib = G.load_library()

    def call(x=FAKE, si=100, rows=3, V=100, dtype=G.GA_F32, r={}, rules=True, g=_graph(), ids=FAKE, rb=FAKE, rp=FAKE,
             out=FAKE + 4096, so=100, wide=0):
        c = G.LogitRulesC(FAKE, FAKE, FAKE, FAKE, 1, FAKE, FAKE, FAKE, 5, FAKE, 2, 4, FAKE)
        for name, value in r.items():
            setattr(c, name, value)
        return lib.graphattn_process_logits(x, si, rows, V, dtype, ctypes.byref(c) if rules else None,
                                            ctypes.byref(g) if g else None, ids, rb, rp, out, so, wide, None)
    bad = [dict(x=None), dict(out=None), dict(rules=False), dict(g=None), dict(ids=None), dict(rows=-1), dict(V=0), dict(si=99),
           dict(so=99), dict(wide=2), dict(x=ODD), dict(out=ODD), dict(rb=ODD), dict(rp=ODD), dict(ids=ODD),
           dict(r=dict(prompt_segments=-1)), dict(r=dict(num_bias=-1)), dict(r=dict(num_masks=-1)),
           dict(r=dict(mask_words=3)), dict(r=dict(masks=None)), dict(r=dict(row_mask=None)), dict(r=dict(bias_tokens=None)),
           dict(r=dict(bias_offsets=None)), dict(r=dict(bias_values=None)), dict(r=dict(repetition=ODD)),
           dict(r=dict(bias_offsets=FAKE + 4)), dict(out=FAKE, so=200), dict(out=FAKE + 400), dict(out=FAKE, dtype=G.GA_BF16, wide=1)]
    bad += [dict(g=_graph(**x)) for x in BAD_GRAPHS]
    _refused(call, {}, bad, [G.GA_EINVAL] * len(bad))
    for change in (dict(dtype=G.GA_MXFP4), dict(dtype=7), dict(V=(1 << 28) + 1, si=1 << 31, so=1 << 31)):
        assert call(**change) == G.GA_EUNSUPPORTED, change
    assert call(rows=0) == G.GA_OK and call(rows=0, x=None, out=None) == G.GA_OK


def test_header_is_plain_c(tmp_path):
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "step.c"
    src.write_text('#include "graphattn_step.h"\n#include <stdio.h>\n'
                   "int main(void) { ga_logit_rules r = {0}; ga_qk_transform t = {0}; ga_device_graph g = {0};\n"
                   "  printf(\"%d %d %d\\n\", (int)sizeof r, (int)sizeof t, (int)sizeof g); return 0; }\n")
    exe = tmp_path / "step"
    r = subprocess.run([cc, "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src),
                        "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    sizes = [ctypes.sizeof(t) for t in (G.LogitRulesC, G.QKTransformC, G.DeviceGraphC)]
    assert [int(x) for x in r.stdout.split()] == sizes


# The binding: tensors of the host, which it refuses last ----------------------------------------------------

def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def i64(*shape):
    return torch.zeros(shape, dtype=torch.int64)


@pytest.fixture
def graph():
    """A device graph without its device."""
    g = object.__new__(G.DeviceGraph)
    g.tensors, g.c = (i32(3), i64(4), i32(9), i64(3), i32(4)), _graph()
    g.num_segments, g.num_branches, g.num_pages, g.ref = 3, 2, 9, ctypes.byref(g.c)
    return g


def test_device_graph_refusals():
    good = [i32(3), i64(4), i32(9), i64(3), i32(4)]
    with pytest.raises(ValueError, match="GPU"):
        G.DeviceGraph(*good, 9)
    for i, t, match in ((0, i64(3), "seg_len"), (1, i64(3), "seg_page_offsets"), (1, i32(4), "seg_page_offsets"),
                        (2, i64(9), "seg_pages"), (3, i32(3), "path_offsets"), (3, i64(0), "path_offsets"),
                        (4, i64(4), "path_segs"), (4, i32(8)[::2], "path_segs")):
        bad = list(good)
        bad[i] = t
        # (arrays are looked at one after the other, and the host's are refused where they stand)
        with pytest.raises(ValueError, match=match if i == 0 or match == "path_offsets" and not t.numel() else "GPU|" + match):
            G.DeviceGraph(*bad, 9)


def test_page_table_refusals():
    with pytest.raises(ValueError, match="seg_len"):
        G.page_table(i64(3), i32(9))
    with pytest.raises(ValueError, match="together"):
        G.page_table(i32(3), i32(9), 0, i64(3))
    with pytest.raises(ValueError, match="together"):
        G.page_table(i32(3), i32(9), 0, i64(0), i32(3))
    with pytest.raises(ValueError, match="GPU"):
        G.page_table(i32(3), i32(9))


def test_slot_map_refusals(graph, monkeypatch):
    monkeypatch.setattr(G, "_stream_handle", lambda *a: 0)       # (no device here)
    with pytest.raises(ValueError, match="capacity"):
        G.slot_map(graph, i32(2))
    with pytest.raises(ValueError, match="int32"):
        G.slot_map(graph, None, None, i32(3), capacity=4)
    for change, match in ((dict(counts=i64(2)), "counts"), (dict(counts=i32(1)), "counts")):
        with pytest.raises(ValueError, match=match):
            G.slot_map(graph, **change, capacity=4)
    with pytest.raises(ValueError, match="GPU"):
        G.slot_map(graph)


def test_transform_refusals():
    f64, f32 = torch.zeros(32, dtype=torch.float64), torch.zeros(64)
    with pytest.raises(ValueError, match="inv_freq"):
        G.QKTransform(64, f64.float())
    with pytest.raises(ValueError, match="rotated"):
        G.QKTransform(32, f64)
    with pytest.raises(ValueError, match="scale"):
        G.QKTransform(64, f64, scale=0.0)
    for norm in (f32[:32], f32.double(), torch.zeros(128)[::2]):
        with pytest.raises(ValueError, match="q_norm"):
            G.QKTransform(64, None, q_norm=norm)
    with pytest.raises(ValueError, match="GPU"):
        G.QKTransform(64, None, q_norm=f32)
    assert G.QKTransform(64).c.rotary_dim == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16", "mxfp4"])
def test_qkv_append_refusals(dtype):
    p, t = G.make_params(4, 2, 64, 3, dtype), G.QKTransform(64)
    pool, row = G.empty_pool(p, "cpu"), torch.float32 if dtype == "f32" else torch.bfloat16
    other = torch.bfloat16 if dtype == "f32" else torch.float32
    rows = torch.zeros(5, 8, 64, dtype=row)
    good = dict(pool=pool, q=rows[:, :4], k=rows[:, 4:6], v=rows[:, 6:], positions=i32(5), slot_words=i32(5), transform=t,
                params=p)
    with pytest.raises(ValueError, match="GPU"):
        G.qkv_append(**good)
    for change, match in ((dict(pool=pool[:2]), "pool"), (dict(pool=pool.to(torch.int8)), "pool"),
                          (dict(transform=G.QKTransform(128)), "transform")):
        with pytest.raises(ValueError, match=match):
            G.qkv_append(**{**good, **change})
    for t, n, h in ((rows[:, :4].to(other), 5, 4), (rows[:, :3], 5, 4), (rows[:4, :4], 5, 4), (rows[..., :32], 5, 8)):
        with pytest.raises(ValueError, match="rows beside"):
            G._rows(t, (n, h, 64), row)
    wide = torch.zeros(5, 4, 128, dtype=row)
    for t in (wide[..., ::2], wide[..., :64], torch.zeros(5, 64, 4, dtype=row).transpose(1, 2)):
        with pytest.raises(ValueError, match="one behind the other"):
            G._rows(t, (5, 4, 64), row)


def test_logits_refusals(graph):
    f, x = torch.zeros(3), torch.zeros(3, 64)
    for bad in (dict(bias_offsets=i64(4)), dict(bias_tokens=i32(2), bias_values=f), dict(masks=i32(2, 2)), dict(row_mask=i32(3)),
                dict(masks=i64(2, 2), row_mask=i32(3)), dict(masks=i32(4), row_mask=i32(3)), dict(repetition=f.double()),
                dict(masks=torch.zeros(2, 2), row_mask=i32(3))):
        with pytest.raises(ValueError):
            G.LogitRules(**bad)
    rules = object.__new__(G.LogitRules)
    rules.rows, rules.vocab, rules.counted, rules.c = 3, 64, True, G.LogitRulesC()
    rules.ref = ctypes.byref(rules.c)
    ids = i32(16 * 9)
    good = dict(logits=x, rules=rules, graph=graph, token_ids=ids)
    with pytest.raises(ValueError, match="GPU"):
        G.process_logits(**good)
    for change, match in ((dict(logits=x.double()), "logits must"), (dict(logits=x[0]), "logits must"),
                          (dict(logits=torch.zeros(4, 64)), "fewer rows"), (dict(logits=torch.zeros(3, 65)), "fewer tokens"),
                          (dict(graph=None), "graph"), (dict(token_ids=None), "graph"), (dict(token_ids=ids[1:]), "token_ids"),
                          (dict(token_ids=ids.long()), "token_ids"), (dict(out=torch.zeros(3, 63)), "out must"),
                          (dict(out=x.bfloat16()), "out must"), (dict(logits=torch.zeros(64, 3).T), "one behind")):
        with pytest.raises(ValueError, match=match):
            G.process_logits(**{**good, **change})
    rules.counted = False
    for change in (dict(row_branches=i32(2)), dict(row_positions=i64(3)), dict(row_branches=i32(6)[::2])):
        with pytest.raises(ValueError, match="row_branches"):
            G.process_logits(x, rules, **change)
