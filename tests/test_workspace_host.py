"""The library's workspace across graph captures (no GPU needed): a C++ program that stands in for the runtime's calls."""
import subprocess

from test_apply_plan_host import build_host


def test_buffers_of_captured_calls_stay(tmp_path):
    r = subprocess.run([build_host(tmp_path, "workspace_host.cpp")], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])
