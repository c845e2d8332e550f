"""C++ exceptions at the output-head entry points (no GPU needed)."""
import subprocess

from test_apply_plan_host import build_host


def test_no_exception_and_no_older_message(tmp_path):
    r = subprocess.run([build_host(tmp_path, "exception_host.cpp")], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])
