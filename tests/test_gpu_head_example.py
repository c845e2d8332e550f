"""The output-head calls together, as examples/compressed_head.py runs them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("vocab,hidden,rank", [(2048, 512, 17), (1001, 333, 8)])
def test_compressed_head_example(vocab, hidden, rank):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "compressed_head.py")
    spec = importlib.util.spec_from_file_location("compressed_head", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    r = mod.run(vocab, hidden, rank, tokens=128, top=32)
    assert 0 < r["error_compensated"] < r["error_4bit"] < 0.2
    assert 0 <= r["loss_after"] < r["loss_before"]
    assert r["bytes_of_16_bit"] < 0.45
    assert len(r["tokens"]) == 4 and all(0 <= t < vocab for t in r["tokens"])
