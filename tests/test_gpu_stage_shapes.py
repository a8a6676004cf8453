"""The autograd form at shapes beside the usual ones: no tokens, one vector."""
import pytest

from stage_util import torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def layers(A):
    return {"linear": A.stage.BlockLinear(96, 40), "entry": A.stage.NormLinear(96, 40), "serving": A.stage.NormLinear(96, 40).eval()}


@pytest.mark.parametrize("frozen", [False, True])
@pytest.mark.parametrize("name", ["linear", "entry", "serving"])
@pytest.mark.parametrize("shape", [(0, 96), (0, 7, 96), (5, 0, 96)])
def test_no_tokens(A, shape, name, frozen):
    torch = torch_mod()
    layer = layers(A)[name]
    if frozen:
        (layer if name == "linear" else layer.linear).freeze()
    x = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
    with torch.no_grad():
        assert layer(x).shape == (*shape[:-1], 40)
    x.requires_grad_(True)
    y = layer(x)
    assert y.shape == (*shape[:-1], 40)
    y.sum().backward()
    assert x.grad.shape == x.shape
    for p in layer.parameters():
        assert p.grad.shape == p.shape and torch.all(p.grad == 0)


@pytest.mark.parametrize("name", ["linear", "entry", "serving"])
def test_one_vector(A, name):
    torch = torch_mod()
    layer = layers(A)[name]
    x = torch.randn(96, device="cuda")
    with torch.no_grad():
        assert torch.equal(layer(x), layer(x[None])[0]) and layer(x).shape == (40,)
    x.requires_grad_(True)
    layer(x).sum().backward()
    assert x.grad.shape == (96,)


@pytest.mark.parametrize("shape", [(96,), (1, 96), (1, 1, 96), (96, 1)])
def test_gradients_have_their_parameters_shapes(A, shape):
    """Weights and biases of as many elements as a row may be of any shape; so are their gradients."""
    torch = torch_mod()
    torch.manual_seed(1)
    x, w, b, dy = (torch.randn(s, device="cuda") for s in ((5, 96), (96,), (96,), (5, 96)))
    got = []
    for s in ((96,), shape):
        leaves = [x.clone().requires_grad_(True), w.clone().view(s).requires_grad_(True), b.clone().view(s).requires_grad_(True)]
        A.stage.layer_norm(*leaves).backward(dy)
        assert leaves[1].grad.shape == leaves[2].grad.shape == s
        got.append([leaves[0].grad, *(t.grad.reshape(-1) for t in leaves[1:])])
    for p, q in zip(*got):
        assert torch.equal(p, q)
