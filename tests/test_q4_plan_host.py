"""Host checks of the 4-bit product's planner (no GPU needed): a C++ program linked against the library plans batches
of whole and of partial panels."""
import subprocess

from test_apply_plan_host import build_host


def test_batches_of_whole_panels_are_planned(tmp_path):
    r = subprocess.run([build_host(tmp_path, "q4_plan_host.cpp")], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])
