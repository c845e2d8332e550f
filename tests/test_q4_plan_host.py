"""Host checks of the 4-bit product's planner (no GPU needed): a C++ program linked against the library plans batches
of whole and of partial panels."""
import subprocess

from test_apply_plan_host import build_host


def test_batches_of_whole_panels_are_planned(tmp_path):
    r = subprocess.run([build_host(tmp_path, "q4_plan_host.cpp")], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])


def test_quantizing_refuses_rows_that_no_launch_takes():
    from paper_2607_12969_amd import lrc
    L, n = lrc.lib(), 2 ** 34 + 1
    assert L.lrc_q4_quantize(1 << 50, n, 2, n, 32, lrc.FP16, 1 << 40, 1 << 44, lrc.FP16, None, None) == -2
    assert b"2^34" in L.lrc_last_error()
