"""The host code of attention, embedding and optimiser under AddressSanitizer
and UndefinedBehaviorSanitizer: the tests of their refusals and forms against
the sanitized build (see test_abi_hostsan.py)."""
import os
import subprocess
import sys

from test_abi_hostsan import ROOT, hostsan_lib  # noqa: F401  (a fixture)

FILES = ("test_operators_cpu.py", "test_grids_cpu.py", "test_attention_forms_cpu.py", "test_optimizer_range_cpu.py",
         "test_owners_devices_cpu.py", "test_aliases_cpu.py")


def test_refusals_clean_under_asan_ubsan(hostsan_lib):  # noqa: F811
    lib_path, runtime = hostsan_lib
    env = dict(os.environ, DMTX_LIB=lib_path, LD_PRELOAD=runtime, PYTHONDONTWRITEBYTECODE="1",
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    cmd = [sys.executable, "-m", "pytest", "-q", "-s", "-p", "no:cacheprovider",
           *[os.path.join(ROOT, "tests", f) for f in FILES]]
    r = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert "ERROR: AddressSanitizer" not in out, out[-4000:]
    assert "runtime error:" not in out, out[-4000:]
    assert r.returncode == 0 and " passed" in out, out[-4000:]
