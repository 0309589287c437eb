"""The host code of rotary positions, the cache in 8 bits and the pages of a cache under sanitizers, without a GPU."""
import os
import re
import subprocess


def test_host_code_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    """Validation, the choice of forms and the launchers, driven by tests/serving_host_check.cpp with sizes at the edges of int and of
    their limits: a sanitizer report aborts the run."""
    from paper_2602_11562_amd.build import build_serving_host_check
    exe = build_serving_host_check(str(tmp_path / "serving_host_check"))
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    print(r.stdout[-500:])
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    accepted, refused = map(int, re.search(r"0 failure\(s\), (\d+) calls accepted, (\d+) refused", r.stdout).groups())
    assert accepted > 1000 and refused > 1000
