"""Builds that need no GPU: the eviction's host code under AddressSanitizer and UBSan, and properties
of the assembly of the compressed cache's kernels."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_18954_amd", "csrc")
HIPCC = "/opt/rocm/bin/hipcc"

needs_hipcc = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")


@needs_hipcc
def test_eviction_host_code_under_sanitizers(tmp_path):
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-omit-frame-pointer"]
    objs = []
    for src in (os.path.join(CSRC, "evict_api.cpp"),
                os.path.join(ROOT, "tests", "host", "evict_driver.cpp")):
        obj = tmp_path / (os.path.basename(src) + ".o")
        r = subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
                            *san, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src,
                            "-o", str(obj)], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        objs.append(str(obj))
    exe = tmp_path / "evict_driver"
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", *san, *objs, "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", HIP_VISIBLE_DEVICES="")
    r = subprocess.run([str(exe), "300"], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "ok" in r.stdout, (r.stdout + r.stderr)[-4000:]


def _assembly(name, tmp_path):
    from paper_2606_18954_amd import build_lib     # compile exactly as the library build does
    out = tmp_path / (name + ".s")
    flags = [f for f in build_lib.CFLAGS if f != "-fPIC"]
    subprocess.run([HIPCC, *flags, "-x", "hip", "-S", "--cuda-device-only",
                    os.path.join(CSRC, name), "-o", str(out)], check=True, capture_output=True)
    return out.read_text()


@needs_hipcc
@pytest.mark.parametrize("name,kernels", [("fp4_attn.hip", 4), ("mq_fp4_attn.hip", 2), ("mass.hip", 6), ("evict.hip", 3)])
def test_kernels_keep_to_their_registers(name, kernels, tmp_path):
    text = _assembly(name, tmp_path)
    sizes = re.findall(r"; ScratchSize: (\d+)", text)
    assert len(sizes) >= kernels and set(sizes) == {"0"}, (name, sizes)


@needs_hipcc
def test_every_m0_write_feeds_a_direct_to_lds_copy(tmp_path):
    text = _assembly("fp4_attn.hip", tmp_path)
    lines = [x.strip() for x in text.splitlines() if x.strip() and not x.strip().startswith((";", "."))]
    copies = 0
    for i, x in enumerate(lines):
        if re.search(r"\bm0\b", x):
            assert re.match(r"s_mov_b32 m0, (s\d+|vcc_lo|vcc_hi)$", x), x
            assert lines[i + 1].startswith("global_load_lds_dwordx4"), lines[i + 1]
            copies += 1
    assert copies and copies == sum(x.startswith("global_load_lds_dwordx4") for x in lines)
