"""The speculative decoding example end to end: prefill, sealed handoff, drafted trees, accepted rows, a manipulated table."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

from paper_2608_25431_amd import gift  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_speculative_decode():
    spec = importlib.util.spec_from_file_location("speculative_decode", os.path.join(ROOT, "examples", "speculative_decode.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(steps=6, verbose=False)
    assert r["tokens"] >= 6 * 4 and r["per_step"] > 1.2  # drafts are accepted
    # two bfloat16 roundings a layer (K or V, and the output) move a logit by some 2^-8 of its deviation each
    assert r["gap"] <= 8 * 2.0 ** -8
    assert r["verdicts"] == [gift.SEG_OWNER_MIXED, gift.SEG_OK, gift.SEG_OK, gift.SEG_OK] and r["zeroed"]
    assert r["sealed"] == [gift.SEG_OK] * 3
