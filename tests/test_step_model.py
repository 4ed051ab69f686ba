"""The kernels between two attention calls on the CPU: their own sources, compiled for the host against the model of the
device (tests/host/model) under AddressSanitizer, every array of exactly its size, against the oracle.

Cases hold what the headers allow: indices outside their arrays, empty paths, segments and vocabularies, padding, odd
sizes.  An access out of range ends the run; waves go in a drawn order, so that a missing barrier shows.
"""
import os
import platform
import re
import struct
import subprocess
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest

import step_util as U
from oracle import cache_oracle as C

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_18954_amd", "csrc")
MODEL = os.path.join(ROOT, "tests", "host", "model")
CXX = "/opt/rocm/llvm/bin/clang++"
SOURCES = ["slots.hip", "qkv.hip", "logits.hip", "step_api.cpp"]
HEADERS = ["step_internal.hpp", "ga_internal.hpp", "mxfp4.hpp", "pool_load.hpp"]

pytestmark = pytest.mark.skipif(not os.path.exists(CXX) or platform.machine() != "x86_64",
                                reason="needs ROCm's clang on x86-64")

SHIM = """
#include <hip/hip_runtime.h>
#include <cmath>
template <class T> T atomicOr(T* p, T v) { const T o = *p; *p = o | v; return o; }
inline void sincospif(float x, float* s, float* c) {
  *s = (float)std::sin(M_PI * (double)x);
  *c = (float)std::cos(M_PI * (double)x);
}
#define __builtin_amdgcn_rsqf(x) (1.f / sqrtf(x))
"""


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    out = tmp_path_factory.mktemp("step_model")
    for name in SOURCES + HEADERS:
        with open(os.path.join(CSRC, name)) as f:
            text = f.read().replace('#include "../../include/', '#include "')
        text = re.sub(r"extern __shared__ (unsigned|int64_t) (\w+)\[\];",
                      r"\1* \2 = static_cast<\1*>(emu::dynamic_lds());", text)
        text = re.sub(r'asm volatile\(""[^;]*;', ";", text)
        assert "asm volatile" not in text, name
        (out / name).write_text(text)
    (out / "shim.hpp").write_text(SHIM)
    flags = ["-std=c++17", "-O1", "-g", "-w", "-fno-pie", "-mf16c", "-fsanitize=address", "-mllvm", "-asan-stack=0",
             "-fno-omit-frame-pointer", "-I", MODEL, "-I", os.path.join(ROOT, "include"), "-I", str(out),
             "-include", str(out / "shim.hpp")]
    jobs = [str(out / s) for s in SOURCES] + [os.path.join(MODEL, s) for s in ("emu.cpp", "step_driver.cpp")]

    def compile_one(path):
        obj = str(out / (os.path.basename(path) + ".o"))
        r = subprocess.run([CXX, *flags, "-x", "c++", "-c", path, "-o", obj], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        return obj

    with ThreadPoolExecutor(8) as ex:
        objs = list(ex.map(compile_one, jobs))
    exe = str(out / "driver")
    r = subprocess.run([CXX, "-no-pie", "-fsanitize=address", *objs, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return exe


NOTHING = np.zeros(0, dtype=np.uint8)


def _blobs(c):
    """(sizes, arrays, indices and shapes of the outputs) of a case, as the driver takes them."""
    arr = lambda a: NOTHING if a is None else np.ascontiguousarray(a)  # noqa: E731
    if c["op"] == 0:
        n = len(c["lens"])
        sizes = [n, c["spare"], max(len(c["old"]) - 1, 0), len(c["old_pages"]), len(c["free"]), c["capacity"]]
        return sizes, [c["lens"], c["old"], c["old_pages"], c["free"], np.zeros(n + 1, np.int64),
                       np.full(c["capacity"], -77, np.int32)]
    if c["op"] in (1, 3):
        g = c["graph"]
        gs = [len(g["seg_len"]), len(g["po"]) - 1, len(g["pages"]), len(g["ps"]), g["num_pages"]]
        ga = [g["seg_len"], g["off"], g["pages"], g["po"], g["ps"]]
    if c["op"] == 1:
        n = c["capacity"]
        return gs + [n], ga + [arr(c["counts"]), np.zeros(gs[1] + 1, np.int32)] + [np.full(n, -77, np.int32)] * 3
    if c["op"] == 2:
        q, k, v = U.qkv_parts(c)
        n, Hq, Hkv, D = c["n"], c["Hq"], c["Hkv"], c["D"]
        dtype = {"f32": 0, "bf16": 1, "mxfp4": 2}[c["dtype"]]
        width = c["rows"].shape[1]
        pool = (np.full((c["num_pages"], Hkv, 17 * D), 9, np.uint8) if c["dtype"] == "mxfp4"
                else np.full((c["num_pages"], Hkv, 2, 16, D), 9, c["rows"].dtype))
        # q, k and v as blobs that end with their last token's last value
        def strided(a, first):
            flat = c["rows"].reshape(-1)[first * D:]
            return np.ascontiguousarray(flat[:(n - 1) * width + a.shape[1] * D]) if n else NOTHING
        if c["in_place"]:
            qa, qs = np.ascontiguousarray(q), Hq * D
        else:
            qa, qs = strided(q, 0), width
        sizes = [n, Hq, Hkv, D, dtype, c["num_pages"], qs, width, width, 2 * len(c["inv_freq"]), int(c["interleaved"]),
                 int(c["in_place"])]
        return sizes, [np.array([c["eps"], c["scale"]]), pool, qa, strided(k, Hq), strided(v, Hq + Hkv), c["positions"],
                       c["words"], np.full((n, Hq, D), 9, c["rows"].dtype), c["inv_freq"], arr(c["weights"][0]),
                       arr(c["weights"][1])]
    bias, masks = c["bias"] or (None,) * 3, c["masks"] or (None, None)
    rows, V = len(c["logits"]), c["vocab"]
    wide = np.float32 if c["out_f32"] or c["dtype"] == "f32" else np.uint16
    counted = any(c[k] is not None for k in ("rep", "freq", "pres"))
    sizes = [rows, V, 0 if c["dtype"] == "f32" else 1, int(c["out_f32"]), V + c["pad"], V + c["pad"], c["prompt"],
             0 if bias[1] is None else len(bias[1]), 0 if masks[0] is None else len(masks[0]),
             0 if masks[0] is None else masks[0].shape[1]] + gs + [int(c["in_place"]), int(counted or c["branches"] is None)]
    return sizes, [c["logits"], np.full((rows, V + c["pad"]), 9, wide)] + ga + [
        c["ids"], arr(c["branches"]), arr(c["positions"]), arr(c["rep"]), arr(c["freq"]), arr(c["pres"]), arr(c["temp"]),
        arr(bias[0]), arr(bias[1]), arr(bias[2]), arr(masks[0]), arr(masks[1])]


def _run(driver, cases, path, seed=1):
    """Outputs of every case, in order."""
    shapes = []
    with open(path + ".in", "wb") as f:
        for c in cases:
            sizes, arrays = _blobs(c)
            outs = {0: (4, 5), 1: (6, 7, 8, 9), 2: (1, 2 if c.get("in_place") else 7),
                    3: (0 if c.get("in_place") else 1,)}[c["op"]]
            shapes.append([arrays[i] for i in outs])
            for a in [np.array([c["op"], len(arrays)] + [int(x) for x in sizes], dtype=np.int64)] + arrays:
                data = np.ascontiguousarray(a).tobytes()
                f.write(struct.pack("q", len(data)) + data)
    r = subprocess.run([driver, path + ".in", path + ".out", str(seed)], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, (r.stdout[-500:], r.stderr[-3000:])
    got = []
    with open(path + ".out", "rb") as f:
        for like in shapes:
            one = []
            for a in like:
                n, = struct.unpack("q", f.read(8))
                one.append(np.frombuffer(f.read(n), dtype=a.dtype).reshape(a.shape))
            got.append(one)
    return got


@pytest.mark.parametrize("seed", range(4))
def test_page_tables(driver, tmp_path, seed):
    rng = np.random.default_rng(seed)
    cases = [U.page_case(rng, bad=i % 4 == 3) for i in range(25)] + [U.page_case(rng, n) for n in (0, 1, 600, 1100)]
    for c, out in zip(cases, _run(driver, cases, str(tmp_path / "x"), seed + 1)):
        U.check_page(c, *out)


@pytest.mark.parametrize("seed", range(4))
def test_slot_maps(driver, tmp_path, seed):
    rng = np.random.default_rng(10 + seed)
    cases = [U.slot_case(rng, bad=i % 3 == 2) for i in range(30)]
    one = U.graph([70000], [[0]], rng)
    cases.append(U.slot_case(rng, g=one, counts=np.array([70000], np.int32)))
    many = U.graph(list(rng.integers(1, 5, 700)), [[i] for i in range(700)], rng)
    cases.append(U.slot_case(rng, g=many))
    cases.append(U.slot_case(rng, g=U.graph([5], [], rng), counts=None))
    for c, out in zip(cases, _run(driver, cases, str(tmp_path / "x"), seed + 1)):
        U.check_slots(c, *out)


SHAPES = [(28, 4, 128), (16, 2, 64), (5, 5, 64), (3, 1, 128), (12, 12, 64), (1, 1, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", SHAPES)
def test_qkv(driver, tmp_path, dtype, Hq, Hkv, D):
    rng = np.random.default_rng(D + Hq)
    cases = []
    for rotary, inter in ((D, False), (D, True), (16, False), (6, True), (0, False), (D // 2, False), (D - 2, True)):
        cases.append(U.qkv_case(rng, int(rng.integers(1, 12)), Hq, Hkv, D, dtype, rotary, inter,
                                (rng.random() < 0.6, rng.random() < 0.6), rng.choice([1.0, 1.3]),
                                int(rng.choice([3, 5000, 2**31 - 1])), int(rng.choice([0, 8, 24])),
                                in_place=rng.random() < 0.3))
    for c, (pool, q_out) in zip(cases, _run(driver, cases, str(tmp_path / "x"))):
        U.check_qkv(c, q_out.reshape(c["n"], Hq, D), pool, 9)


@pytest.mark.parametrize("Hq,Hkv,D", SHAPES)
def test_qkv_into_mxfp4_is_append_of_its_bf16_rows(driver, tmp_path, Hq, Hkv, D):
    rng = np.random.default_rng(D + Hq)
    for rotary, inter in ((D, False), (16, True)):
        c = U.qkv_case(rng, 9, Hq, Hkv, D, "bf16", rotary, inter)
        c["positions"][:] = rng.integers(0, 1000, 9)              # (all stored, but for the words outside)
        c["rows"][4, (Hq + Hkv) * D + 7] = 0x7F80                 # an infinity in v, a NaN in k
        c["rows"][5, Hq * D + 3] = 0x7FC0
        f = dict(c, dtype="mxfp4")
        (pool, q1), (codes, q2) = _run(driver, [c, f], str(tmp_path / "x"))
        np.testing.assert_array_equal(q1, q2)
        there = (c["words"] >= 0) & (c["words"] < 16 * c["num_pages"])
        w = c["words"][there]
        k, v = (U.values(pool[w // 16, :, i, w % 16], "bf16") for i in (0, 1))
        want = C.append(np.full_like(codes, 9), k, v, w)
        np.testing.assert_array_equal(codes, want)


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("dtype,wide", [("f32", False), ("bf16", False), ("bf16", True)])
def test_logits(driver, tmp_path, dtype, wide, seed):
    rng = np.random.default_rng(20 + seed)
    cases = []
    for i in range(8):
        bad = i % 4 == 3
        g = U.random_graph(rng, 12, bad=bad)
        rows = int(rng.integers(1, 9)) if i else 0
        rules = "".join(x for x in "rfptbm" if rng.random() < 0.7)
        drafts = bad or rng.random() < 0.6
        if not drafts:
            rows = min(rows, len(g["po"]) - 1)
        cases.append(U.logits_case(rng, g, rows, int(rng.choice([1, 7, 31, 33, 500, 2049, 5000])), dtype, wide, rules,
                                   int(rng.integers(0, 3)), drafts, int(rng.choice([0, 1, 5])),
                                   in_place=not wide and rng.random() < 0.4, bad=bad))
    for c, (out,) in zip(cases, _run(driver, cases, str(tmp_path / "x"), seed + 1)):
        U.check_logits(c, out, c["logits"] if c["in_place"] else np.full_like(out, 9))


def test_logits_of_long_contexts_and_paths(driver, tmp_path):
    """Counts beyond 14 bits (the slice in halves of 32 bits a token) and paths of more segments than are taken at once."""
    rng = np.random.default_rng(5)
    long = U.graph([100, 20000, 5], [[0, 1], [0, 2]], rng)
    paths = U.graph(list(rng.integers(0, 4, 150)), [list(range(150)), list(range(149, 19, -1)), [3]], rng)
    cases = []
    for g, vocab, rows in ((long, 4100, 2), (long, 333, 2), (paths, 700, 3)):
        c = U.logits_case(rng, g, rows, vocab, "f32", rules="rfptbm", drafts=False)
        if g is long:
            c["ids"][:] = np.where(rng.random(len(c["ids"])) < 0.95, 300, c["ids"])
        cases.append(c)
    half = U.logits_case(rng, long, 3, 333, "f32", rules="fp")
    half["branches"][:], half["positions"][:] = 0, [16482, 16483, 99]       # 16383 and 16384 counted tokens, none
    half["ids"][:] = 7
    cases.append(half)
    deep = U.logits_case(rng, paths, 4, 90, "bf16", rules="rfp", prompt=70)
    deep["branches"][:], deep["positions"][:] = [0, 0, 1, 1], [40, 130, 100, 2**31 - 1]
    cases.append(deep)
    for c, (out,) in zip(cases, _run(driver, cases, str(tmp_path / "x"))):
        U.check_logits(c, out, np.full_like(out, 9))


@pytest.mark.parametrize("seed", range(3))
def test_rows_of_one_branch_go_on_with_its_counts(driver, tmp_path, seed):
    """More rows than workgroups take one each: drafts in order, out of order, again, beyond the path, with padding, other
    branches and biases between them, and counts that pass 14 bits on the way."""
    rng = np.random.default_rng(40 + seed)
    cases = []
    for rules in ("rfp", "rfptbm", "f"):
        g = U.random_graph(rng, 12)
        c = U.logits_case(rng, g, 1100, 37, "bf16", rules=rules, biases=1)
        B = len(g["po"]) - 1
        c["branches"][:] = np.repeat(rng.integers(-1, B, 220), 5)
        first = rng.integers(0, 60, 220)
        c["positions"][:] = (first[:, None] + np.cumsum(rng.choice([0, 1, 1, 2, 40, -3], (220, 5)), 1)).reshape(-1)
        cases.append(c)
    long = U.graph([100, 17000], [[0, 1], [0]], rng)
    c = U.logits_case(rng, long, 1030, 40, "f32", rules="rfp")
    c["branches"][:] = np.arange(1030) // 500
    c["positions"][:] = np.where(np.arange(1030) < 500, 99 + 16380 + np.arange(1030) // 40, np.arange(1030) % 130)
    c["ids"][:] = 3
    cases.append(c)
    for c, (out,) in zip(cases, _run(driver, cases, str(tmp_path / "x"), seed + 1)):
        U.check_logits(c, out, np.full_like(out, 9))
