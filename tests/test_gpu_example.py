"""The example of the head's operators in a federated round: both losses fall,
the groups end with the same head, and a second run gives the same bits."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "federated_distillation.py")


def test_federated_distillation():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("federated_distillation", PATH)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    a, b = ex.run(), ex.run()
    for g in range(ex.G):
        for k in range(2):
            print("[gpu-example]", g, k, a["first"][g][k], a["last"][g][k], flush=True)
            assert a["last"][g][k] < 0.9 * a["first"][g][k]
    assert torch.equal(a["heads"][0], a["heads"][1])
    for x, y in zip(a["heads"], b["heads"]):
        assert torch.equal(x, y)
    assert a["first"] == b["first"] and a["last"] == b["last"]
