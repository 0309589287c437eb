"""The steps of the pages' kernels over users, on the host, without a GPU."""
import os
import subprocess

from paper_2602_11562_amd import build


def test_users_up_to_the_last_of_an_int(tmp_path):
    """Tables of one page may have 2^31 - 1 users: the step behind the last of them does not fit an int."""
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "pages_users_check.cpp")
    obj, exe = str(tmp_path / "check.o"), str(tmp_path / "check")
    sanitizer = ["-fsanitize=undefined", "-fno-sanitize-recover=undefined"]
    host = [x for f in sanitizer for x in ("-Xarch_host", f)]
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-Xclang", "-target-feature", "-packed-fp32-ops")]
    for cmd in ([build._hipcc(), "-x", "hip", "--offload-host-only", *flags, *host, "-c", src, "-o", obj],
                ["/opt/rocm/lib/llvm/bin/clang++", *sanitizer, "-o", exe, obj]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "every user in order" in r.stdout, r.stdout + r.stderr[-3000:]
