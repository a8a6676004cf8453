"""Serving with a weight that was laid out once: what changes the weight ends it."""
import copy

import pytest

from stage_util import torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def served(layer, x):
    with torch_mod().no_grad():
        return layer(x)


def optimizer(make):
    def change(A, layer, x):
        torch = torch_mod()
        opt = make(torch, layer.parameters())
        layer(x).float().square().mean().backward()
        opt.step()
    return change


def given_gradient(make):
    """An optimizer's step without a call of the layer."""
    def change(A, layer, x):
        torch = torch_mod()
        layer.weight.grad = torch.ones_like(layer.weight)
        make(torch, layer.parameters()).step()
    return change


def load(A, layer, x):
    layer.load_state_dict(A.stage.BlockLinear(layer.weight.shape[1], layer.weight.shape[0]).state_dict())


def assign(A, layer, x):
    layer.load_state_dict(A.stage.BlockLinear(layer.weight.shape[1], layer.weight.shape[0]).state_dict(), assign=True)


def replace(A, layer, x):
    layer.weight = torch_mod().nn.Parameter(layer.weight.detach() * 3)


def in_place(A, layer, x):
    with torch_mod().no_grad():
        layer.weight.mul_(3)


def other_type(A, layer, x):
    layer.to(torch_mod().bfloat16)


CHANGES = {
    "sgd": optimizer(lambda torch, p: torch.optim.SGD(p, lr=1.0)),
    "adamw": optimizer(lambda torch, p: torch.optim.AdamW(p, lr=0.1)),
    "fused": optimizer(lambda torch, p: torch.optim.AdamW(p, lr=0.1, fused=True)),
    "given": given_gradient(lambda torch, p: torch.optim.AdamW(p, lr=0.1)),
    "load": load, "assign": assign, "replace": replace, "in_place": in_place, "other_type": other_type,
}


@pytest.mark.parametrize("change", CHANGES)
def test_a_changed_weight_is_served_as_it_is(A, change):
    torch = torch_mod()
    layer = A.stage.BlockLinear(300, 130)
    x = torch.randn(3, 300, device="cuda")
    fresh = lambda: served(copy.deepcopy(layer).unfreeze(), x)
    first = fresh()
    layer.freeze()
    assert torch.equal(served(layer, x), first)
    CHANGES[change](A, layer, x)
    now = fresh()
    if change != "other_type":
        assert not torch.equal(now, first)
    assert torch.equal(served(layer, x), now)
    assert torch.equal(served(layer.freeze(), x), now) and torch.equal(served(layer, x), now)


def test_frozen_codes_are_kept_and_not_made_again(A, monkeypatch):
    torch = torch_mod()
    layer = A.stage.BlockLinear(300, 130).freeze()
    x = torch.randn(3, 300, device="cuda")
    calls = []
    quantize = A.stage.quantize_weight
    monkeypatch.setattr(A.stage, "quantize_weight", lambda *a, **k: calls.append(1) or quantize(*a, **k))
    y = served(layer, x)
    assert torch.equal(served(layer, x), y) and not calls
    twin = copy.deepcopy(layer)
    assert torch.equal(served(twin, x), y)
    with torch.inference_mode():
        assert torch.equal(layer(x), y)
        inside = A.stage.BlockLinear(300, 130).freeze()      # its weight has no count of its changes
        z = inside(x)
        calls.clear()
        assert torch.equal(inside(x), z) and not calls
