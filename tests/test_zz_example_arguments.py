"""The example hands the library pointers: tensors that are not what these are taken for (another type, order, shape or device) are refused before any call."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TOKENS, K, E, H, F = 6, 2, 3, 8, 12


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("expert_layer", os.path.join(ROOT, "examples", "expert_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _arguments(**change):
    ok = dict(x=torch.zeros(TOKENS, H), ids=torch.zeros(TOKENS, K, dtype=torch.int32), weight=torch.zeros(TOKENS, K), dy=torch.zeros(TOKENS, H))
    return {**ok, **change}


BAD = {
    "x of another width": dict(x=torch.zeros(TOKENS, H + 1)), "x of every second column": dict(x=torch.zeros(TOKENS, 2 * H)[:, ::2]), "x transposed": dict(x=torch.zeros(H, TOKENS).t()),
    "x of another type": dict(x=torch.zeros(TOKENS, H, dtype=torch.float64)), "ids of 64 bits": dict(ids=torch.zeros(TOKENS, K, dtype=torch.int64)),
    "ids transposed": dict(ids=torch.zeros(K, TOKENS, dtype=torch.int32).t()), "ids of fewer tokens": dict(ids=torch.zeros(TOKENS - 1, K, dtype=torch.int32)),
    "weights of 16 bits": dict(weight=torch.zeros(TOKENS, K, dtype=torch.bfloat16)), "fewer weights": dict(weight=torch.zeros(TOKENS, K - 1)),
    "weights elsewhere": dict(weight=torch.zeros(TOKENS, K, device="meta")),
}
BAD_TRAINING = {"dy of another type": dict(dy=torch.zeros(TOKENS, H, dtype=torch.bfloat16)), "dy of fewer tokens": dict(dy=torch.zeros(TOKENS - 1, H)),
                "dy of every second token": dict(dy=torch.zeros(2 * TOKENS, H)[::2]), "tokens of another type than the weights": dict(x=torch.zeros(TOKENS, H, dtype=torch.bfloat16))}


@pytest.mark.parametrize("what", list(BAD) + list(BAD_TRAINING))
def test_tensors_that_are_something_else(example, what):
    layer = example.ExpertLayer.__new__(example.ExpertLayer)
    layer.experts, layer.inner, layer.width, layer.up, layer.down = E, F, H, torch.zeros(E, F, H), torch.zeros(E, H, F)
    a = _arguments(**{**BAD, **BAD_TRAINING}[what])
    with pytest.raises(ValueError):
        layer.train(a["x"], a["ids"], a["weight"], a["dy"])
    if what in BAD:
        with pytest.raises(ValueError):
            layer.serve(a["x"], a["ids"], a["weight"])


def test_projections_that_do_not_fit(example):
    for up, down in ((torch.zeros(E, F, H), torch.zeros(E, F, H)), (torch.zeros(E, F, H), torch.zeros(E + 1, H, F)),
                     (torch.zeros(E, F, H), torch.zeros(E, H, F, dtype=torch.bfloat16)), (torch.zeros(E, F, H, dtype=torch.int8), torch.zeros(E, H, F, dtype=torch.int8))):
        with pytest.raises(ValueError):
            example.ExpertLayer(up, down)
