"""The host code of the operators around the layer step under AddressSanitizer and UndefinedBehaviorSanitizer: its sources, with
both on their host code, and a driver that replays the calls over the range of sizes and takes note of their launches (see
host_sanitizer_policy.cpp).  No GPU is touched."""
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2512_23353_amd import build as libbuild

TESTS = os.path.dirname(os.path.abspath(__file__))
SOURCES = ("policy_api.cpp", "linear.hip", "linear_tile.hip", "linear_f32.hip", "act_backward.hip", "token_logprob.hip", "adamw.hip")
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
       "-Xarch_host", "-fno-omit-frame-pointer"]


def test_host_code_of_the_policy_operators(tmp_path):
    if shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    base = ["hipcc", *[f for f in libbuild.FLAGS if f != "-O3"], "-O1", "-g", *SAN]

    def one(src):
        obj = os.path.join(str(tmp_path), os.path.basename(src) + ".o")
        r = subprocess.run([*base, "-x", "hip", "-c", src, "-o", obj], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
        return obj

    with ThreadPoolExecutor(max_workers=8) as ex:
        objs = list(ex.map(one, [*(os.path.join(libbuild.CSRC, s) for s in SOURCES), os.path.join(TESTS, "host_sanitizer_policy.cpp")]))
    exe = os.path.join(str(tmp_path), "driver")
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize", "-o", exe, *objs],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    report = r.stdout[-3000:] + r.stderr[-6000:]
    assert r.returncode == 0 and "done failures=0" in r.stdout and "FAIL" not in r.stdout, report
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, report
    assert int(r.stdout.split("calls=")[1].split()[0]) > 1000
