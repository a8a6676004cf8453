"""The autograd form of the stage operators, and the example that runs them between boundaries."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import stage_oracle as orc
from stage_util import HALF_BF16, U, f64, torch_mod

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def blocks(v, group, code):
    c, e = orc.quantize(v, group, code)
    return c * orc.spread(e, *v.shape, group)


def test_layer_norm_through_autograd(A):
    """A sum of its outputs with random factors: the gradients are those of the formula at float32's precision (the bounds of the
    operator's own tests, 64 U of the terms, are below 2e-5 of the largest for rows of 300 values of size 1)."""
    torch = torch_mod()
    rng = np.random.default_rng(1)
    x64, w64, b64 = rng.standard_normal((4, 7, 300)), 1 + 0.1 * rng.standard_normal(300), rng.standard_normal(300)
    f64s = rng.standard_normal((4, 7, 300))
    x, w, b, f = (torch.tensor(v, dtype=torch.float32, device="cuda") for v in (x64, w64, b64, f64s))
    for t in (x, w, b):
        t.requires_grad_(True)
    y = A.stage.layer_norm(x, w, b, 1e-5)
    (y * f).sum().backward()
    x64, w64, b64, f64s = f64(x).reshape(-1, 300), f64(w), f64(b), f64(f).reshape(-1, 300)
    want, mean, rstd = orc.layer_norm(x64, w64, b64, 1e-5)
    dx, dw, db = orc.layer_norm_backward(f64s, x64, w64, mean, rstd)
    for got, ref in ((y, want), (x.grad, dx), (w.grad, dw), (b.grad, db)):
        assert np.all(np.abs(f64(got).reshape(ref.shape) - ref) <= 2e-5 * np.abs(ref).max())
    y = A.stage.layer_norm(x.detach(), None, None)
    assert not y.requires_grad


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_block_linear_through_autograd(A, name):
    """The three products are those of the quantized operands: y and dx with the squares of the weight, dw with columns."""
    torch = torch_mod()
    dtype = torch.float32 if name == "f32" else torch.bfloat16
    rng = np.random.default_rng(2)
    m, k, n = 90, 200, 260
    layer = A.stage.BlockLinear(k, n)
    x = torch.tensor(rng.standard_normal((2, m // 2, k)), dtype=dtype, device="cuda", requires_grad=True)
    dy = torch.tensor(1e-3 * rng.standard_normal((2, m // 2, n)), dtype=dtype, device="cuda")
    y = layer(x)
    assert y.shape == (2, m // 2, n) and y.dtype == dtype
    y.backward(dy)
    x64, w64, dy64 = f64(x).reshape(m, k), f64(layer.weight), f64(dy).reshape(m, n)
    qw = blocks(w64, 128, 0)
    gt, xt = blocks(np.ascontiguousarray(dy64.T), 1, 1), blocks(np.ascontiguousarray(x64.T), 1, 0)

    def check(got, a, b, low):
        want, terms = a @ b.T, np.abs(a) @ np.abs(b).T
        bound = (a.shape[1] * U + (2.0 ** -10 if low else 0)) * terms
        got = f64(got).reshape(want.shape)
        assert np.all(np.abs(got - want) <= bound + (HALF_BF16 if low else U) * (np.abs(want) + bound))

    check(y, blocks(x64, 1, 0), qw, name == "bf16")
    check(x.grad, blocks(dy64, 1, 1), np.ascontiguousarray(qw.T), name == "bf16")
    check(layer.weight.grad, gt, xt, False)
    assert layer.weight.grad.dtype == torch.float32


def test_what_needs_no_gradient_gets_none(A):
    torch = torch_mod()
    layer = A.stage.BlockLinear(96, 64)
    x = torch.randn(10, 96, device="cuda")
    layer(x).sum().backward()
    assert x.grad is None and layer.weight.grad is not None
    layer.weight.grad = None
    layer.weight.requires_grad_(False)
    x.requires_grad_(True)
    layer(x).sum().backward()
    assert x.grad is not None and layer.weight.grad is None


def test_serving_uses_the_weight_as_it_is_unless_frozen(A):
    torch = torch_mod()
    entry = A.stage.NormLinear(300, 130)
    x = torch.randn(3, 300, device="cuda").bfloat16()
    with torch.no_grad():
        y = entry(x)
        entry.linear.weight.data.mul_(2)          # behind autograd's back
        assert torch.equal(entry(x), 2 * y)
        entry.linear.freeze()
        entry.linear.weight.data.mul_(2)
        assert torch.equal(entry(x), 2 * y)
        assert torch.equal(entry.linear.unfreeze()(x), entry.linear(x))
        assert torch.equal(entry(x), 4 * y)
        # rows do not depend on each other: one token alone gives the same codes, and its product the same bits as three's
        assert torch.equal(entry(x[:1]), entry(x)[:1])
    assert entry(x).requires_grad


def test_example(A):
    """A student behind a compressed boundary comes nearer to its teacher, and serves what it learned."""
    torch = torch_mod()
    spec = importlib.util.spec_from_file_location("pipeline_stage", os.path.join(ROOT, "examples", "pipeline_stage.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, entry, out = example.train(256, 136, 264, 40, say=lambda line: None)
    assert all(np.isfinite(losses)) and losses[-1] < 0.8 * losses[0]
    x = torch.randn(5, 136, device="cuda").bfloat16()
    y = example.serve(entry, out, x)
    with torch.no_grad():
        assert torch.equal(y, out(torch.relu(entry(x))))
