"""The host side of the 4-bit calls under AddressSanitizer and UndefinedBehaviorSanitizer
(CPU only): sizes, plans and refusals over random and edge-case arguments. GPU code is not
sanitized: the hipcc lines instrument the host pass only."""
import os

import pytest

from test_sanitizers import ENV, ROOT, SAN, SRC, _run

pytestmark = pytest.mark.slow


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="hipcc not installed")
def test_four_bit_host_code_under_sanitizers(tmp_path):
    import subprocess
    objs, procs = [], []
    for f in ("runtime", "gemm", "gemm_dl", "rowwise", "attention", "ceiling"):
        o = str(tmp_path / f"{f}.o")
        objs.append(o)
        procs.append(subprocess.Popen(
            ["/opt/rocm/bin/hipcc", "--offload-arch=gfx950", "-O1", "-g", "-fPIC", "-std=c++17",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
             "-Xarch_host", "-fno-sanitize-recover=all",
             "-I", SRC, "-c", os.path.join(SRC, f + ".hip"), "-o", o],
            stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True))
    for p in procs:
        out, err = p.communicate()
        assert p.returncode == 0, err[-3000:]
    drv, exe = str(tmp_path / "driver.o"), str(tmp_path / "mx")
    _run(["g++", "-std=c++17", "-O1", "-g", *SAN, "-c",
          os.path.join(ROOT, "tests", "sanitize", "mx_driver.cpp"), "-o", drv])
    _run(["g++", *SAN, "-o", exe, *objs, drv, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"])
    assert "0 failures" in _run([exe], env=ENV)
