"""Host check of the adapters' planner (no GPU needed): a C++ program linked against the library."""
import subprocess

from test_apply_plan_host import build_host


def test_places_of_partial_gradients(tmp_path):
    r = subprocess.run([build_host(tmp_path, "adapter_plan_host.cpp")], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])
