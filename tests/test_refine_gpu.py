"""The example that runs draws, their loss, kept activation and gradients together, on a small population."""

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "refine_networks.py")


def test_networks_learn_from_their_answers():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("refine_networks", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    before, after, parents = example.main(["--genomes", "100", "--updates", "100"])
    # (many random networks reach an output by no path that tells the inputs apart, and answer by chance)
    assert after.mean() > before.mean() + 0.02
    assert before.max() < 0.6 and after.max() > 0.8
    assert torch.isfinite(after).all()
    fit = torch.argsort(after, descending=True, stable=True)[:20]
    assert torch.isin(parents[0].long(), fit).all()
