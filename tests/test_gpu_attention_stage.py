"""Rotation, attention and the cache as a stage uses them: through autograd, packed, served, and the example."""
import importlib.util
import os

import numpy as np
import pytest

from attention_util import check_forward, ints, orc
from stage_util import HALF_BF16, f64, torch_mod

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def frequencies(rotated):
    torch = torch_mod()
    return torch.tensor(10000.0 ** (-np.arange(0, rotated, 2) / rotated), dtype=torch.float32, device="cuda")


def plain(q, k, v, f, ends, neighbours=False):
    """Rotation and causal attention of packed sequences, PyTorch in 64 bits on the host."""
    torch = torch_mod()

    def turn(x, n):
        angle = torch.arange(n, dtype=torch.float64)[:, None, None] * f.double().cpu()
        c, s = angle.cos(), angle.sin()
        half = f.numel()
        if neighbours:
            a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            turned = torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
        else:
            a, b = x[..., :half], x[..., half:2 * half]
            turned = torch.cat((a * c - b * s, a * s + b * c), -1)
        return torch.cat((turned, x[..., 2 * half:]), -1)

    group, out = q.shape[1] // k.shape[1], []
    for b, e in zip(ends, ends[1:]):
        n = e - b
        tq, tk = turn(q[b:e], n).transpose(0, 1), turn(k[b:e], n).repeat_interleave(group, 1).transpose(0, 1)
        s = (tq @ tk.transpose(1, 2)) * q.shape[2] ** -0.5
        s = s.masked_fill(~torch.ones(n, n, dtype=torch.bool).tril(), float("-inf"))
        out.append((torch.softmax(s, -1) @ v[b:e].repeat_interleave(group, 1).transpose(0, 1)).transpose(0, 1))
    return torch.cat(out)


@pytest.mark.parametrize("neighbours", [False, True])
def test_through_autograd(A, neighbours):
    """Packed sequences in float32: outputs and gradients of a sum with random factors against 64 bits.  (For rows of 70 scores of size 1 and
    heads of 32 values the bounds of the operators' own tests are below 2e-5 of the largest.)"""
    torch = torch_mod()
    rng = np.random.default_rng(1)
    ends, f = [0, 30, 31, 101], frequencies(16)
    x64 = [torch.tensor(rng.standard_normal((101, h, 32)), requires_grad=True) for h in (4, 2, 2)]
    factors = torch.tensor(rng.standard_normal((101, 4, 32)))
    (plain(*x64, f, ends, neighbours) * factors).sum().backward()
    x = [t.detach().float().cuda().requires_grad_(True) for t in x64]
    off = ints(ends)
    o = A.stage.attention(A.stage.rotate(x[0], f, off, neighbours=neighbours), A.stage.rotate(x[1], f, off, neighbours=neighbours), x[2], off)
    (o * factors.float().cuda()).sum().backward()
    with torch.no_grad():
        want = plain(*x64, f, ends, neighbours)
    assert float((o.detach().cpu().double() - want).abs().max()) <= 2e-5 * float(want.abs().max())
    for got, ref in zip(x, x64):
        assert float((got.grad.cpu().double() - ref.grad).abs().max()) <= 2e-5 * float(ref.grad.abs().max())


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_a_batch_is_packed_sequences(A, name):
    """(batch, n, heads, head), views that are no plain rows among them, gives what its tokens with offsets give, bit for bit."""
    torch = torch_mod()
    dtype = torch.float32 if name == "f32" else torch.bfloat16
    f, off = frequencies(64), ints([0, 50, 100, 150])
    whole = torch.randn(3, 50, 9, 64, device="cuda", dtype=dtype)
    parts = [whole[:, :, :4], whole[:, :, 4:6], torch.randn(3, 2, 50, 64, device="cuda", dtype=dtype).transpose(1, 2)]
    factors = torch.randn(3, 50, 4, 64, device="cuda", dtype=dtype)
    results = []
    for flat in (False, True):
        q, k, v = (p.reshape(-1, *p.shape[2:]).contiguous().requires_grad_(True) if flat else p.detach().requires_grad_(True) for p in parts)
        o = A.stage.attention(A.stage.rotate(q, f, off if flat else None), A.stage.rotate(k, f, off if flat else None), v, off if flat else None)
        (o * factors.view(o.shape)).sum().backward()
        results.append([t.reshape(150, -1) for t in (o, q.grad, k.grad, v.grad)])
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("packed", [False, True])
def test_one_function_for_all_three(A, packed):
    """SelfAttention's function against rotate and attention one by one: the same kernels, the same bits, and gradients side by side."""
    torch = torch_mod()
    heads, kv, head, n = 4, 2, 64, 120
    off = ints([0, 70, 71, 110]) if packed else None
    x = torch.randn(n, heads + 2 * kv, head, device="cuda").bfloat16()
    f, factors = frequencies(32), torch.randn(n, heads, head, device="cuda").bfloat16()
    a, b = x.clone().requires_grad_(True), x.clone().requires_grad_(True)
    one = A.stage._TurnedAttention.apply(a, f, off, 3 if packed else 1, heads, kv, A.ROTATE_HALVES)
    turned = A.stage.rotate(b[:, :heads + kv], f, off)
    two = A.stage.attention(turned[:, :heads], turned[:, heads:], b[:, heads + kv:], off)
    assert torch.equal(one, two)
    one.backward(factors)
    two.backward(factors)
    assert torch.equal(a.grad, b.grad)
    if packed:
        assert torch.all(one[110:] == 0) and torch.all(a.grad[110:] == 0) and torch.isfinite(a.grad).all()


def test_what_needs_no_gradient(A):
    torch = torch_mod()
    q, k, v = (torch.randn(2, 20, 2, 64, device="cuda") for _ in range(3))
    assert not A.stage.attention(q, k, v).requires_grad
    k.requires_grad_(True)
    A.stage.attention(q, k, v, causal=False, scale=0.2).sum().backward()
    assert k.grad is not None and q.grad is None


@pytest.mark.parametrize("frozen", [False, True])
def test_a_stage_served_from_a_cache(A, frozen):
    """A prompt and tokens after it through a cache against the whole sequence at once.  Attention's results differ by the rounding of
    both, at most 2 * 2^-8 and what the weights' rounding adds, as much again; where that moves a value over the border of two codes its code moves by
    up to a step, 2^-3 of it: so the product's results agree to (2^-3 + 2^-5) of the sum of its terms' magnitudes."""
    torch = torch_mod()
    torch.manual_seed(3)
    layer = A.stage.SelfAttention(256, 4, 2, 64).eval()
    if frozen:
        layer.entry.linear.freeze(), layer.out.freeze()
    x = torch.randn(3, 40, 256, device="cuda").bfloat16()
    with torch.no_grad():
        want = layer(x)
        cache = layer.cache(3, 50, page_size=16)
        got = [layer(x[:, :25], cache=cache)]
        got += [layer(x[:, i:i + 1], cache=cache) for i in range(25, 40)]
        assert cache.lengths.tolist() == [40] * 3
    got = torch.cat(got, 1)
    qkv = layer.entry(x).view(120, 8, 64)
    o = A.stage._TurnedAttention.apply(qkv, layer.frequencies, None, 3, 4, 2, A.ROTATE_HALVES).detach().float().abs()
    terms = (o.reshape(120, 256) @ layer.out.weight.detach().abs().t()).view(3, 40, 256)
    assert torch.all((got.float() - want.float()).abs() <= (2 ** -3 + 2 ** -5) * terms + 2 ** -6 * want.float().abs())
    with pytest.raises(ValueError):
        layer(x, cache=cache)   # with gradients


def test_a_block_with_bfloat16_weights(A):
    """The same float32 weights, rounded: trained and served as the block whose weights hold those values in float32 (its gradients, but for their rounding)."""
    torch = torch_mod()
    torch.manual_seed(5)
    layer = A.stage.SelfAttention(128, 2, 1, 64).bfloat16()
    same = A.stage.SelfAttention(128, 2, 1, 64)
    same.load_state_dict(layer.state_dict())
    x = torch.randn(2, 30, 128, device="cuda").bfloat16()
    y, want = layer(x), same(x)
    assert torch.equal(y, want)
    y.backward(x)
    want.backward(x)
    for a, b in zip(layer.parameters(), same.parameters()):
        assert a.grad.dtype == torch.bfloat16
        assert torch.all((a.grad.float() - b.grad).abs() <= HALF_BF16 * b.grad.abs())
    with torch.no_grad():
        cache, other = layer.eval().cache(2, 64), same.eval().cache(2, 64)
        assert torch.equal(layer(x, cache=cache), same(x, cache=other))


def test_drafts_and_what_is_accepted(A):
    """A tree of drafted tokens attends without making the sequence longer; the accepted ones, appended again, give what their path in the
    tree gave: the same keys in the same order for every row but for where they lie, to the bounds of both."""
    torch = torch_mod()
    heads, kv, head, context = 4, 2, 64, 37
    f = frequencies(head)
    cache = A.stage.Cache(1, 80, kv, head, page_size=16)
    x = torch.randn(context + 5, heads + 2 * kv, head, device="cuda").bfloat16()

    def step(t, **kw):
        return cache.step(t[:, :heads], t[:, heads:heads + kv], t[:, heads + kv:], frequencies=f, **kw)

    step(x[:context])
    # nodes: 0 - 1 - 3 is the path that is accepted; 2 and 4 branch off
    tree = torch.tensor([[0b00001], [0b00011], [0b00101], [0b01011], [0b10001]], device="cuda")
    positions = ints([context, context + 1, context + 1, context + 2, context + 1])
    o = step(x[context:], tree=tree, positions=positions)
    assert cache.lengths.tolist() == [context]
    path = [0, 1, 3]
    again = step(x[context:][path])
    assert cache.lengths.tolist() == [context + 3]
    k = cache.k[cache.table[0].long()].transpose(1, 2).reshape(-1, kv, head)[:context + 3]
    v = cache.v[cache.table[0].long()].transpose(1, 2).reshape(-1, kv, head)[:context + 3]
    q = A.stage.rotate(x[context:][path][:, :heads], f, positions=ints([context, context + 1, context + 2]))
    seen = orc.causal(3, context + 3)
    for h in range(heads):
        args = ("bf16", f64(q[:, h]), f64(k[:, h // 2]), f64(v[:, h // 2]), seen, head ** -0.5)
        check_forward(*args, f64(o[path][:, h]))
        check_forward(*args, f64(again[:, h]))
    with pytest.raises(ValueError):
        step(x[:2], tree=tree[:2])


def test_two_passes_of_a_stage_captured(A):
    """A training step of the stage as a graph, replayed with other inputs: the gradients of an eager step."""
    torch = torch_mod()
    torch.manual_seed(4)
    layer = A.stage.SelfAttention(128, 2, 1, 64)
    x = torch.randn(90, 128, device="cuda").bfloat16()
    off = ints([0, 40, 90])
    dy = torch.randn(90, 128, device="cuda").bfloat16()
    parameters = list(layer.parameters())

    def grads():
        return torch.autograd.grad(layer(x, off), parameters, dy)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        grads()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = grads()
    for turn in range(3):
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, grads())), turn


def test_one_token_of_any_stride(A):
    """A single token's stride says nothing: 13 values here, which no operator takes."""
    torch = torch_mod()
    x = torch.randn(3, 2, 13, device="cuda")[:1, :, :8].transpose(0, 1)[1:2]   # (1, 1, 8), not whole vectors apart
    y = torch.randn(5, 24, device="cuda")[2:3, None, :8]
    f = frequencies(8)
    for t in (x, y):
        whole = t.clone(memory_format=torch.contiguous_format)
        assert torch.equal(A.stage.rotate(t, f), A.stage.rotate(whole, f))
        assert torch.equal(A.stage.attention(t, t, t), A.stage.attention(whole, whole, whole))
        one, other = (A.stage.Cache(1, 16, 1, 8, 16, torch.float32) for _ in range(2))
        assert torch.equal(one.step(t, t, t, frequencies=f), other.step(whole, whole, whole, frequencies=f))


@pytest.mark.parametrize("shape", [(0, 2, 64), (0, 5, 2, 64), (3, 0, 2, 64)])
def test_nothing_there(A, shape):
    torch = torch_mod()
    x = torch.zeros(shape, device="cuda", requires_grad=True)
    y = A.stage.attention(*(A.stage.rotate(x, frequencies(64)) for _ in range(2)), x)
    y.sum().backward()
    assert y.shape == shape and x.grad.shape == shape
    cache = A.stage.Cache(0, 16, 2, 64, 16, torch.float32)
    assert cache.step(x[:0].detach(), x[:0].detach(), x[:0].detach()).numel() == 0


def test_gradients_that_are_one_number(A):
    """The gradient of a sum has no strides: it is taken as what it stands for."""
    torch = torch_mod()
    torch.manual_seed(4)
    x = torch.randn(2, 9, 4, 64, device="cuda", requires_grad=True)
    got = []
    for of in (lambda y: y.sum(), lambda y: (y * torch.ones_like(y)).sum()):
        y = A.stage.attention(A.stage.rotate(x, frequencies(32)), x[:, :, :2], x[:, :, 2:])
        got.append(torch.autograd.grad(of(y), x)[0])
    assert torch.equal(*got)


def test_example(A):
    """It runs: losses, the gradient that goes back and all parameters' are finite, and served tokens are those of one pass over all."""
    torch = torch_mod()
    spec = importlib.util.spec_from_file_location("attention_stage", os.path.join(ROOT, "examples", "attention_stage.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, back, block = example.train(200, 128, 4, 2, 264, 3, say=lambda line: None)
    assert all(np.isfinite(losses)) and torch.isfinite(back).all() and float(back.abs().max()) > 0
    assert all(p.grad is not None and torch.isfinite(p.grad).all() for p in block.parameters())
    x = torch.randn(20, 128, device="cuda").bfloat16()
    y = example.serve(block, x, 12)
    assert y.shape == x.shape and torch.isfinite(y).all()
