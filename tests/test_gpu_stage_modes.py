"""The same arithmetic with and without gradients in training mode, and the norm that writes codes in evaluation mode."""
import pytest

from stage_util import torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def make(A, dtype):
    torch = torch_mod()
    torch.manual_seed(3)
    entry = A.stage.NormLinear(768, 300)
    with torch.no_grad():
        entry.norm_weight.add_(0.1 * torch.randn(768, device="cuda"))
        entry.norm_bias.add_(0.1 * torch.randn(768, device="cuda"))
    return entry, torch.randn(200, 768, device="cuda").to(dtype)


@pytest.mark.parametrize("frozen", [False, True])
@pytest.mark.parametrize("name", ["float32", "bfloat16"])
def test_training_mode_has_one_arithmetic(A, name, frozen):
    torch = torch_mod()
    entry, x = make(A, getattr(torch, name))
    if frozen:
        entry.linear.freeze()
    with torch.no_grad():
        quiet = entry(x)
    assert torch.equal(entry(x), quiet)


@pytest.mark.parametrize("reentrant", [True, False])
def test_checkpointing_changes_nothing(A, reentrant):
    from torch.utils.checkpoint import checkpoint

    torch = torch_mod()
    entry, x = make(A, torch.bfloat16)
    dy = torch.randn(200, 300, device="cuda").bfloat16()
    results = []
    for through in (False, True):
        entry.zero_grad()
        leaf = x.clone().requires_grad_(True)
        y = checkpoint(entry, leaf, use_reentrant=reentrant) if through else entry(leaf)
        y.backward(dy)
        results.append((y.detach(), leaf.grad, entry.norm_weight.grad.clone(), entry.norm_bias.grad.clone(), entry.linear.weight.grad.clone()))
    for p, q in zip(*results):
        assert torch.equal(p, q)


def test_evaluation_mode_goes_straight_to_codes(A):
    torch = torch_mod()
    entry, x = make(A, torch.bfloat16)
    entry.eval()
    d = A.make_norm_desc(200, 768, x_dtype=A.BF16)
    codes, scales, _ = A.accept_layer_norm_quantize(d, x, entry.norm_weight, entry.norm_bias)
    w, ws = A.stage.quantize_weight(entry.linear.weight, colwise=False)[:2]
    want = A.accept_block_matmul(A.make_matmul_desc(200, 300, 768, out_dtype=A.BF16), codes, scales, w, ws)
    with torch.no_grad():
        assert torch.equal(entry(x), want)
        entry.linear.freeze()
        assert torch.equal(entry(x), want)
    assert entry(x).requires_grad
