"""The host side of the calls on 8-bit integers under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): sizes, plans and refusals over random and edge-case
arguments. The library's host code alone is compiled, with empty images in place of the GPU code."""
import os
import re
import subprocess

import pytest

from test_sanitizers import ENV, ROOT, SAN, SRC, _run

pytestmark = pytest.mark.slow


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="hipcc not installed")
def test_int8_host_code_under_sanitizers(tmp_path):
    objs, procs = [], []
    for f in ("runtime", "gemm", "gemm_dl", "rowwise", "attention", "ceiling"):
        o = str(tmp_path / f"{f}.o")
        objs.append(o)
        procs.append(subprocess.Popen(
            ["/opt/rocm/bin/hipcc", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-g", "-fPIC",
             "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
             "-Xarch_host", "-fno-sanitize-recover=all",
             "-I", SRC, "-c", os.path.join(SRC, f + ".hip"), "-o", o],
            stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True))
    for p in procs:
        out, err = p.communicate()
        assert p.returncode == 0, err[-3000:]
    images = sorted(set(re.findall(r"U (__hip_fatbin\w*)", _run(["nm", *objs]))))
    (tmp_path / "images.c").write_text("".join(f"char {i}[16];\n" for i in images))
    _run(["gcc", "-c", str(tmp_path / "images.c"), "-o", str(tmp_path / "images.o")])
    drv, exe = str(tmp_path / "driver.o"), str(tmp_path / "qint")
    _run(["g++", "-std=c++17", "-O1", "-g", *SAN, "-c",
          os.path.join(ROOT, "tests", "sanitize", "qint_driver.cpp"), "-o", drv])
    _run(["g++", *SAN, "-o", exe, drv, *objs, str(tmp_path / "images.o"), "-L/opt/rocm/lib", "-lamdhip64",
          "-Wl,-rpath,/opt/rocm/lib"])
    assert "0 failures" in _run([exe], env=ENV)
