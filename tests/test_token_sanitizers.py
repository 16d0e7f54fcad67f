"""The host side of the token operators built with AddressSanitizer and
UndefinedBehaviorSanitizer on its host code only (the device code is compiled as
usual), driven by tests/sanitize/token_abi_check.cpp on the CPU."""
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_32628_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
       "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer"]
FLAGS = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++20", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument", *SAN]


def _compile(args):
    src, out, lang = args
    r = subprocess.run([HIPCC, *FLAGS, "-x", lang, "-c", src, "-o", str(out)], capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, (src, r.stderr[-3000:])
    return str(out)


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="CPU-only check (the driver expects no device)")
def test_token_operators_under_asan_and_ubsan(tmp_path):
    jobs = [(os.path.join(CSRC, f), tmp_path / (f + ".o"), "hip")
            for f in ("host_token.cpp", "norm.hip", "rope.hip", "diff_fwd.hip", "diff_bwd.hip")]
    jobs.append((os.path.join(ROOT, "tests", "sanitize", "token_abi_check.cpp"), tmp_path / "driver.o", "c++"))
    with ThreadPoolExecutor(max_workers=4) as pool:
        objs = list(pool.map(_compile, jobs))
    exe = tmp_path / "token_abi_check"
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", *SAN, *objs, "-o", str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-4000:])
    assert "token ABI checks passed" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr
