"""The example that runs the operators together: quantization costs, distillation lowers its loss."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def test_score_and_recover():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "score_and_recover.py")
    spec = importlib.util.spec_from_file_location("score_and_recover", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    out = mod.main(["--tokens", "600", "--vocabulary", "1003", "--steps", "10"])
    s = out["scores"]
    # the tokens were drawn from the bf16 model: nothing scores better on them by more than chance
    assert s["bf16"] < s["4-bit microscaled"] + 0.05
    assert s["bf16"] < s["2-bit frames"]
    assert out["distill"][-1] < out["distill"][0]
    assert all(b < a * 1.001 for a, b in zip(out["distill"], out["distill"][1:]))
