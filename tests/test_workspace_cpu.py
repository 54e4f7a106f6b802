"""The device buffers that the library keeps for the kernels of a call, on the
host (no GPU): gdn_workspace.hip against a fake runtime, with AddressSanitizer
and UndefinedBehaviorSanitizer."""
import glob
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "sanitize")
CSRC = os.path.join(ROOT, "paper_2607_06763_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CLANGXX = "/opt/rocm/llvm/bin/clang++"
NM = shutil.which("nm")

pytestmark = pytest.mark.skipif(not (shutil.which(HIPCC) and shutil.which(CLANGXX) and NM), reason="needs hipcc and nm")


def run_driver(tmp_path, driver, sources):
    """Builds the host side of the sources with the driver, which brings the runtime they call, and runs it."""
    flags = ["--offload-arch=gfx950", "--offload-host-only", "-O1", "-g", "-std=c++17", "-Xarch_host",
             "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    objs = []
    for src in [os.path.join(SAN, driver), *(os.path.join(CSRC, s) for s in sources)]:
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        r = subprocess.run([HIPCC, *flags, "-c", "-x", "hip", src, "-o", objs[-1]], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr
    exe = str(tmp_path / "driver")
    r = subprocess.run([CLANGXX, "-fsanitize=address,undefined", *objs, "-lpthread", "-o", exe], capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "0 failed checks" in out and "runtime error" not in out, out


def test_buffers_that_were_handed_out_stay(tmp_path):
    run_driver(tmp_path, "workspace_driver.cpp", ["gdn_workspace.hip"])


def test_calls_of_two_threads_on_one_stream(tmp_path):
    """The whole library's host side: kernels that share a stream's workspace are enqueued call by call."""
    objs = []
    flags = ["--offload-arch=gfx950", "--offload-host-only", "-O0", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    for src in [os.path.join(SAN, "threads_driver.cpp"), *glob.glob(os.path.join(CSRC, "*.hip"))]:
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        r = subprocess.run([HIPCC, *flags, "-c", "-x", "hip", src, "-o", objs[-1]], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr
    # the device code that the host side names: there is none here
    r = subprocess.run([NM, "-u", *objs], capture_output=True, text=True, timeout=60)
    absent = sorted({w for w in r.stdout.split() if w.startswith("__hip_fatbin")})
    exe = str(tmp_path / "driver")
    r = subprocess.run([CLANGXX, *objs, *(f"-Wl,--defsym={s}=0" for s in absent), "-lpthread", "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "0 failed checks" in r.stdout, r.stdout + r.stderr
