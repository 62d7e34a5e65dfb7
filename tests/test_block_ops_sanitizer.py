"""The host code of the group norm, the feed-forward block and the 8-bit projection (argument checks, plans,
workspace layouts) under AddressSanitizer and UndefinedBehaviorSanitizer, without a GPU:
tests/sanitize/block_ops_driver.cpp against the sanitized copy of the library."""
import os
import subprocess

from paper_2609_36522_amd import build as B
from test_host_sanitizer import SUPP, _driver


def test_sanitized_block_operators_without_gpu(tmp_path):
    _driver()                                 # the sanitized library is built with it
    exe = tmp_path / "block_ops_driver"
    src = os.path.join(os.path.dirname(__file__), "sanitize", "block_ops_driver.cpp")
    subprocess.run([B.hipcc(), "-O1", "-g", "-std=c++17", *B._HOST_SAN, "-I", B.INCLUDE, src, "-L", B.SAN_DIR, "-lparaanya_san",
                    f"-Wl,-rpath,{B.SAN_DIR}", "-o", str(exe)], check=True, timeout=300)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1:abort_on_error=0:exitcode=23",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", LSAN_OPTIONS=f"suppressions={SUPP}:exitcode=23")
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300, env=env)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "block_ops_driver ok" in r.stdout, out[-4000:]
    assert "Sanitizer" not in out and "runtime error" not in out, out[-4000:]
