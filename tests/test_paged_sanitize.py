"""The paged cache's host layer under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only): the entry
points with sizes at and past every limit. Compiled by g++ with stand-ins for the kernel launchers."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_03235_amd", "csrc")
HERE = os.path.join(ROOT, "tests", "sanitize")


def _gpu():
    try:
        import torch
        return torch.cuda.is_available()
    except Exception:
        return False


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/lib/libamdhip64.so"),
                    reason="needs g++ and the HIP host runtime")
@pytest.mark.skipif(_gpu(), reason="host-only run: the device entry points are driven through validation only")
def test_paged_host_under_sanitizers(tmp_path):
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g", "-O1"]
    exe = str(tmp_path / "paged_driver")
    sources = [os.path.join(CSRC, f) for f in ("sgdkv_host.cpp", "paged_host.cpp", "profile.cpp")]
    sources += [os.path.join(HERE, f) for f in ("launch_stubs.cpp", "paged_driver.cpp")]
    subprocess.run(["g++", "-std=c++17", *san, "-ffp-contract=off", "-fno-fast-math", "-D__HIP_PLATFORM_AMD__",
                    "-isystem", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", CSRC, *sources, "-o",
                    exe, "-L/opt/rocm/lib", "-Wl,-rpath,/opt/rocm/lib", "-lamdhip64", "-lm"], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, f"sanitizer run failed (rc {r.returncode}):\n{r.stdout[-3000:]}\n{r.stderr[-6000:]}"
    assert "SANITIZE PASS" in r.stdout
