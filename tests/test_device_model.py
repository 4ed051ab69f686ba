"""The compressed cache's kernels on the CPU: their own sources, compiled for the host against a model of the
device (tests/host/model), under AddressSanitizer.

Every array has exactly the size the headers ask for, so an index out of range ends the run; results are
compared with sums in 64 bits, waves run in a drawn order, and direct-to-LDS copies land once when they are
issued and once as late as their waits allow, so that a missing barrier or wait shows as a wrong value.  What
the model cannot show are wait states of the hardware (test_isa_wait_states.py).
"""
import os
import platform
import random
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest

from perf import operators

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_18954_amd", "csrc")
MODEL = os.path.join(ROOT, "tests", "host", "model")
CXX = "/opt/rocm/llvm/bin/clang++"
SOURCES = ["api.cpp", "sched.hip", "seg_attn.hip", "mq_attn.hip", "mq_fp4_attn.hip", "fp4_attn.hip", "merge.hip",
           "kv_write.hip", "mass.hip", "evict.hip", "evict_api.cpp"]

pytestmark = pytest.mark.skipif(not os.path.exists(CXX) or platform.machine() != "x86_64",
                                reason="needs ROCm's clang on x86-64")


def _once(pattern, new, text, count):
    out, n = re.subn(pattern, new, text)
    assert n == count, (pattern, n)
    return out


def _for_the_host(name, text):
    """A source with its inline assembly, LDS pointers and dynamic LDS put in the model's terms."""
    text = re.sub(r"__attribute__\(\(address_space\(\d\)\)\)", "", text)
    text = text.replace('#include "../../include/', '#include "')
    if name == "mass.hip":
        text = _once(r"extern __shared__ float (\w+)\[\];", r"float* \1 = static_cast<float*>(emu::dynamic_lds());",
                     text, 1)
    if name == "attn_dev.hpp":
        text = _once(r'asm volatile\("s_mov_b32 m0, %2[^;]*;', "emu::dma16(off, base, lds_base);", text, 2)
        text = _once(r'asm volatile\("global_store[^;]*;', "*p = v;", text, 2)
    if name == "mq_attn.hpp":
        # A wave's lanes write rows to LDS and read each other's without a barrier: they go together.
        rounds = r"(for \(int p = 0; p < 2; \+\+p\) \{\n)(#pragma unroll\n +for \(int t = 0; t < C::NC / 2; \+\+t\))"
        reads = (r"#pragma unroll\n( +for \(int k = 0; k < NI; \+\+k\) \{\n[^\n]*\n +st\[p\]\[k\])")
        text = _once(rounds, r"\1emu::together();\n\2", text, 1)
        text = _once(reads, r"emu::together();\n\1", text, 1)
    text = re.sub(r'asm volatile\(""[^;]*;', ";", text)
    assert "asm volatile" not in text, name
    return text


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    out = tmp_path_factory.mktemp("model")
    src = out / "csrc"
    src.mkdir()
    for name in os.listdir(CSRC):
        if not name.startswith(("equiv", "reward")):
            with open(os.path.join(CSRC, name)) as f:
                (src / name).write_text(_for_the_host(name, f.read()))
    # (no position-independent code: LDS addresses are 32 bits)
    flags = ["-std=c++17", "-O1", "-g", "-w", "-fno-pie", "-mf16c", "-fsanitize=address", "-mllvm", "-asan-stack=0",
             "-fno-omit-frame-pointer", "-I", MODEL, "-I", os.path.join(ROOT, "include"), "-I", str(src)]
    jobs = [str(src / s) for s in SOURCES] + [os.path.join(MODEL, s) for s in ("emu.cpp", "driver.cpp")]

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


def _run(driver, *args):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1")
    r = subprocess.run([driver, *map(str, args)], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, (args, r.stdout[-1500:], r.stderr[-3000:])
    return r.stdout


@pytest.mark.parametrize("kind,cases,seeds", [("attn", 12, 4), ("mass", 12, 4), ("evict", 40, 2), ("cache", 30, 2)])
def test_random_calls(driver, kind, cases, seeds):
    with ThreadPoolExecutor(8) as ex:
        for text in ex.map(lambda seed: _run(driver, kind, cases, seed), range(1, seeds + 1)):
            assert "ok, " in text


def _write_case(case, path):
    """The case's graph as the driver reads it; how many pages its kernels read."""
    lens, paths, counts = operators._structure(case)
    off, pages, total = operators._pages(lens, 3)
    kind = {"attn": 0, "mass": 1, "evict": 2}[case["op"]]
    dtype = {"f32": 0, "bf16": 1, "mxfp4": 2}[case.get("dtype", "mxfp4")]
    parts = [[kind, case.get("hq", 1), case.get("hkv", 1), case.get("dim", 64), dtype, total, len(lens), len(paths)],
             lens, off, pages]
    if kind == 2:
        n = np.asarray(lens)
        parts += [np.maximum(np.ceil(n * case["share"]).astype(np.int64),
                             np.minimum(n, case["first"] + case["recent"])), [case["first"], case["recent"]]]
    else:
        many = case["queries"] or case["graph"] == "prompt"
        parts += [np.concatenate([[0], np.cumsum([len(p) for p in paths])]), np.concatenate(paths),
                  counts if many else [0] * len(paths)]
    np.concatenate([np.asarray(p, dtype=np.int64) for p in parts]).tofile(path)
    return total * case.get("hkv", 1) * max(1, sum(counts) // 256)


def test_calls_of_a_rollout_stay_in_their_arrays(driver, tmp_path):
    """Calls drawn over the sizes of the performance cases, on a device of 256 CUs."""
    rng, todo = random.Random(11), []
    while len(todo) < 24:
        case = operators.draw(rng)
        path = str(tmp_path / f"{len(todo)}.bin")
        if case["op"] != "append" and _write_case(case, path) < 30000:
            todo.append(path)
    with ThreadPoolExecutor(8) as ex:
        for text in ex.map(lambda path: _run(driver, "file", path), todo):
            assert text.startswith("ok")
