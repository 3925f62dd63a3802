"""The example that teaches a local head: its loss falls, both loss calls agree, and the teacher's tokens become likely."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("rank", [32, 256])
def test_example_teaches_the_head(rank):
    spec = importlib.util.spec_from_file_location("distill_head", os.path.join(ROOT, "examples", "distill_head.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.run(rows=256, vocab=5003, rank=rank, top_k=20, steps=40, quiet=True)
    assert got["losses"][-1] < 0.5 * got["losses"][0], got
    assert abs(got["losses"][-1] - got["stored"]) < 1e-4 * (1 + abs(got["stored"]))   # the same bf16 weights, float32 logits
    assert got["after"][0] > got["before"][0] + 1.0, got
