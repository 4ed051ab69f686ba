"""Host checks of the compressed cache: the header's entry points are exported, malformed arguments
are refused before any device work, and the header is plain C."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2606_18954_amd import graphattn as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(1 << 20)          # aligned, never dereferenced by a refused call


def test_every_declared_symbol_is_exported():
    lib = G.load_library()
    syms = G.header_symbols("graphattn_cache.h")
    assert set(syms) == {"graphattn_kv_page_bytes", "graphattn_kv_read", "graphattn_run_mass",
                         "graphattn_evict_create", "graphattn_evict_select",
                         "graphattn_evict_destroy"}
    for s in syms:
        assert hasattr(lib, s), s


def test_page_bytes():
    for hkv, dim, dtype, want in [(4, 128, "bf16", 4 * 2 * 16 * 128 * 2),
                                  (2, 64, "f32", 2 * 2 * 16 * 64 * 4),
                                  (4, 128, "mxfp4", 4 * (2 * 16 * 64 + 2 * 16 * 4)),
                                  (3, 64, "mxfp4", 3 * (2 * 16 * 32 + 2 * 16 * 2))]:
        p = G.make_params(hkv, hkv, dim, 7, dtype)
        assert G.kv_page_bytes(p) == want
        t = G.empty_pool(p, "cpu")
        assert t.numel() * t.element_size() == 7 * want
    p = G.make_params(4, 4, 96, 7, "mxfp4")
    with pytest.raises(G.GraphAttnError) as e:
        G.kv_page_bytes(p)
    assert e.value.status == G.GA_EUNSUPPORTED


def test_unknown_types_are_refused():
    for dtype in (3, -1):
        p = G.make_params(4, 4, 64, 7, "mxfp4")
        p.dtype = dtype
        assert G.load_library().graphattn_kv_page_bytes(ctypes.byref(p)) == G.GA_EUNSUPPORTED


def test_mxfp4_params_pass_validation():
    g = G.HostGraph([20], [0, 2], [0, 1], [0, 1], [0])
    p = G.make_params(8, 2, 64, 2, "mxfp4")
    assert G.validate_only(g, p) == G.GA_EINVAL          # only the device buffers are missing
    assert "non-NULL" in G.last_error()
    p = G.make_params(8, 2, 64, 1, "mxfp4")
    assert G.validate_only(g, p) == G.GA_ERANGE


def test_kv_read_errors():
    lib = G.load_library()
    p = G.make_params(4, 4, 64, 7, "mxfp4")

    def rd(pool=FAKE, words=FAKE, n=3, k=FAKE, v=FAKE, params=p):
        return lib.graphattn_kv_read(pool, words, n, k, v,
                                     ctypes.byref(params) if params else None, None)
    assert rd(pool=None) == G.GA_EINVAL and rd(words=None) == G.GA_EINVAL
    assert rd(k=None) == G.GA_EINVAL and rd(v=None) == G.GA_EINVAL
    assert rd(n=-1) == G.GA_EINVAL and rd(params=None) == G.GA_EINVAL
    odd = ctypes.c_void_p((1 << 20) + 8)
    assert rd(k=odd) == G.GA_EINVAL and rd(v=odd) == G.GA_EINVAL and rd(pool=odd) == G.GA_EINVAL
    assert rd(words=ctypes.c_void_p((1 << 20) + 2)) == G.GA_EINVAL
    assert rd(n=0) == G.GA_OK and rd(n=0, k=None, v=None, pool=None, words=None) == G.GA_OK


def _create(lens=(20, 7, 33), keep=(10, 7, 5), first=0, recent=0, num_pages=None, pages=None,
            offsets=None):
    lib = G.load_library()
    npg = [(n + 15) // 16 for n in lens]
    off = np.concatenate([[0], np.cumsum(npg)]) if offsets is None else np.asarray(offsets)
    pages = np.arange(int(off[-1])) if pages is None else pages
    g = G.HostGraph(lens, off, pages, [0], [])
    k = np.ascontiguousarray(keep, dtype=np.int32)
    h = ctypes.c_void_p(1)
    n = int(off[-1]) if num_pages is None else num_pages
    st = lib.graphattn_evict_create(ctypes.byref(g.st), k.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                                    first, recent, n, None, ctypes.byref(h))
    if st != G.GA_OK:
        assert not h.value and G.last_error()
    else:
        lib.graphattn_evict_destroy(h)
    return st


def test_evict_create_errors():
    lib = G.load_library()
    assert _create(keep=(21, 7, 5)) == G.GA_EINVAL
    assert _create(keep=(10, -1, 5)) == G.GA_EINVAL
    assert _create(first=-1) == G.GA_EINVAL and _create(recent=-1) == G.GA_EINVAL
    assert _create(first=3, recent=3) == G.GA_EINVAL                   # the last keeps 5 < 6 of 33
    assert "keeps 5" in G.last_error()
    assert _create(keep=(20, 6, 33), first=2**31 - 1, recent=2**31 - 1) == G.GA_EINVAL
    assert _create(lens=(20, 0, 33), keep=(1, 0, 1), offsets=[0, 2, 2, 5]) == G.GA_EINVAL
    assert _create(offsets=[0, 1, 2, 5]) == G.GA_EINVAL                # too few pages
    assert _create(offsets=[1, 2, 3, 6], pages=np.zeros(6)) == G.GA_EINVAL
    assert _create(num_pages=4) == G.GA_ERANGE
    assert _create(pages=[0, 1, 2, -3, 4, 5]) == G.GA_ERANGE
    assert _create(num_pages=-1) == G.GA_EINVAL
    assert _create(num_pages=(1 << 27) + 1) == G.GA_EUNSUPPORTED
    assert _create(lens=((1 << 30) + 1,), keep=(1,), offsets=[0, 5], num_pages=1 << 27) == G.GA_EUNSUPPORTED
    h = ctypes.c_void_p()
    k = np.zeros(3, dtype=np.int32)
    kp = k.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    assert lib.graphattn_evict_create(None, kp, 0, 0, 9, None, ctypes.byref(h)) == G.GA_EINVAL
    g = G.HostGraph([20], [0, 2], [0, 1], [0], [])
    assert lib.graphattn_evict_create(ctypes.byref(g.st), None, 0, 0, 9, None,
                                      ctypes.byref(h)) == G.GA_EINVAL
    assert lib.graphattn_evict_create(ctypes.byref(g.st), kp, 0, 0, 9, None, None) == G.GA_EINVAL
    assert lib.graphattn_evict_select(None, FAKE, FAKE, FAKE, None) == G.GA_EINVAL
    lib.graphattn_evict_destroy(None)
    with pytest.raises(ValueError):
        G.Evict(g, [1, 2], 0, 0, 9)


def test_evict_without_segments_needs_no_device():
    g = G.HostGraph([], [0], [], [0], [])
    lib = G.load_library()
    h = ctypes.c_void_p()
    assert lib.graphattn_evict_create(ctypes.byref(g.st), None, 0, 0, 0, None,
                                      ctypes.byref(h)) == G.GA_OK
    assert lib.graphattn_evict_select(h, None, None, None, None) == G.GA_OK
    lib.graphattn_evict_destroy(h)


def test_evict_is_refused_without_a_gpu():
    import torch
    if torch.cuda.device_count():
        pytest.skip("a GPU is visible")
    assert _create() in (G.GA_ENOMEM, G.GA_EHIP)


def test_run_mass_errors():
    lib = G.load_library()
    assert lib.graphattn_run_mass(None, FAKE, FAKE, FAKE, None, 1.0, FAKE, None) == G.GA_EINVAL
    assert "plan" in G.last_error()


def test_header_is_plain_c(tmp_path):
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "abi.c"
    src.write_text(r'''
#include "graphattn_cache.h"
int main(void) {
  ga_params p = {8, 2, 128, 16, 4, GA_MXFP4, 0.0f, 0};
  ga_evict* h = 0;
  return graphattn_kv_page_bytes(&p) == 2 * 17 * 128 &&
         graphattn_evict_create(0, 0, 0, 0, 0, 0, &h) == GA_EINVAL && h == 0 ? 0 : 1;
}
''')
    lib = os.path.join(ROOT, "paper_2606_18954_amd")
    exe = tmp_path / "abi"
    r = subprocess.run([cc, "-std=c99", "-Wall", "-Werror", "-pedantic", "-I",
                        os.path.join(ROOT, "include"), str(src), "-L", lib, "-lgraphattn",
                        "-Wl,-rpath," + lib, "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert subprocess.run([str(exe)]).returncode == 0


def test_binding_refuses_tensors_of_other_types_and_sizes():
    """(Before any pointer is taken: these are tensors of the host.)"""
    torch = pytest.importorskip("torch")
    p = G.make_params(4, 2, 64, 3, "mxfp4")
    pool, words = G.empty_pool(p, "cpu"), torch.zeros(2, dtype=torch.int32)
    kv = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    for bad in (pool[:-1], torch.zeros(3, 2, 2, 16, 64, dtype=torch.bfloat16)):
        for call in (lambda: G.kv_append(bad, kv, kv, words, p), lambda: G.kv_copy(bad, words, words, p),
                     lambda: G.kv_read(bad, words, p, kv, kv)):
            with pytest.raises(ValueError, match="MXFP4 pool"):
                call()
    for k, v in ((kv.float(), kv), (kv, kv.to(torch.float8_e4m3fn))):
        with pytest.raises(ValueError, match="bf16"):
            G.kv_append(pool, k, v, words, p)
    with pytest.raises(ValueError, match="must be"):
        G.kv_read(pool, words, p, kv.half(), kv)
    with pytest.raises(ValueError, match="int32"):
        G.kv_read(pool, words.long(), p, kv, kv)
    with pytest.raises(ValueError, match="Hkv, D"):
        G.kv_read(pool, words, p, kv[:1], kv)
    g = G.HostGraph([20], [0, 2], [0, 1], [0, 1], [0])
    with pytest.raises(ValueError, match="bf16"):
        G.decode_static(torch.zeros(1, 4, 64), pool, g, p, None, None)


def test_binding_refuses_a_tensor_of_another_device(monkeypatch):
    """Where no stream is given: the call would go to the current device's."""
    torch = pytest.importorskip("torch")

    class Far:
        dtype, is_cuda, shape = torch.int32, True, (2, 2, 64)

        def get_device(self):
            return 1

        def numel(self):
            return 2

        def is_contiguous(self):
            return True

        def data_ptr(self):
            return 1 << 20
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    p, t = G.make_params(4, 2, 64, 3, "bf16"), Far()
    for call in (lambda: G.kv_append(t, t, t, t, p), lambda: G.kv_copy(t, t, t, p)):
        with pytest.raises(ValueError, match="device 1"):
            call()
