"""Refusals of the output-head binding beyond those of test_head_host.py (no GPU needed)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_12969_amd import lrc  # noqa: E402


@pytest.mark.parametrize("group", [0, -32, 48, 1024])
def test_q4_apply_refuses_other_groups(group):
    codes, scales = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 2, dtype=torch.float16)
    with pytest.raises(ValueError, match="group must"):
        lrc.q4_apply(codes, scales, torch.zeros(2, 40, dtype=torch.float16), group)
