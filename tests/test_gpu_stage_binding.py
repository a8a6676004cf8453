"""The stage operators' calls on real device tensors: outputs that are given, tensors that are refused, and the two ways that a
call can take (native code, or the checks written in Python) with the same results."""
import pytest

from stage_util import torch_mod

pytestmark = pytest.mark.gpu
R, C, N = 20, 300, 70


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def calls(A):
    """name -> (function of keyword arguments, its good arguments, the names of its outputs in order)."""
    torch = torch_mod()
    x, w, b = torch.randn(R, C, device="cuda"), torch.randn(C, device="cuda"), torch.randn(C, device="cuda")
    nd, bd = A.make_norm_desc(R, C), A.make_block_desc(R, C)
    stats = A.accept_layer_norm(nd, x, w, b)[1]
    a, sa, _, _ = A.accept_block_quantize(bd, x)
    v, sv, _, _ = A.accept_block_quantize(A.make_block_desc(N, C, group=128), torch.randn(N, C, device="cuda"))
    f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    empty = lambda *size, dtype=torch.float32: torch.empty(*size, dtype=dtype, device="cuda")
    codes = lambda rows, cols: empty(rows, A.accept_block_stride(cols), dtype=f8)[:, :cols]
    return {
        "layer_norm": (A.accept_layer_norm, dict(desc=nd, x=x, weight=w, bias=b),
                       dict(y=empty(R, C), stats=empty(2, R))),
        "quantized": (A.accept_layer_norm_quantize, dict(desc=nd, x=x, weight=w, bias=b),
                      dict(codes=codes(R, C), scales=empty(3, R, dtype=e8), stats=empty(2, R))),
        "backward": (A.accept_layer_norm_backward, dict(desc=nd, dy=torch.randn(R, C, device="cuda"), x=x, weight=w, stats=stats),
                     dict(dx=empty(R, C), dweight=empty(C), dbias=empty(C))),
        "quantize": (A.accept_block_quantize, dict(desc=bd, x=x, rowwise=True, colwise=True),
                     dict(codes=codes(R, C), scales=empty(3, R, dtype=e8), codes_t=codes(C, R), scales_t=empty(1, C, dtype=e8))),
        "matmul": (A.accept_block_matmul, dict(desc=A.make_matmul_desc(R, N, C), a=a, a_scales=sa, b=v, b_scales=sv),
                   dict(y=empty(R, N))),
    }


NAMES = ["layer_norm", "quantized", "backward", "quantize", "matmul"]


def as_tuple(r):
    return r if isinstance(r, tuple) else (r,)


def same(p, q):
    torch = torch_mod()
    bits = lambda t: t.contiguous().view(torch.uint8)
    return p.shape == q.shape and p.dtype == q.dtype and torch.equal(bits(p), bits(q))


class _Nothing:
    def __getattr__(self, name):
        return lambda *args: -1


@pytest.mark.parametrize("name", NAMES)
def test_outputs_made_and_given_natively_and_not(A, name, monkeypatch):
    function, good, outs = calls(A)[name]
    first = as_tuple(function(**good))
    assert [tuple(t.shape) for t in first] == [tuple(t.shape) for t in outs.values()]
    given = as_tuple(function(**good, **outs))
    for f, g, o in zip(first, given, outs.values()):
        assert g.data_ptr() == o.data_ptr() and same(f, o)
    assert A.stage_binding._native.__name__.endswith("_native") and hasattr(A.stage_binding._native, "block_matmul")
    monkeypatch.setattr(A.stage_binding, "_native", _Nothing())
    for o in outs.values():
        o.contiguous()
    for f, g in zip(first, as_tuple(function(**good))):
        assert same(f, g)
    for f, g, o in zip(first, as_tuple(function(**good, **outs)), outs.values()):
        assert g is o and same(f, o)


@pytest.mark.parametrize("kind", ["parameter", "subclass", "requires_grad"])
def test_other_tensors(A, kind):
    torch = torch_mod()

    class Tagged(torch.Tensor):
        pass

    for function, good, _ in calls(A).values():
        want = as_tuple(function(**good))
        other = dict(good)
        for key in ("x", "weight"):
            if key in other:
                t = other[key]
                other[key] = (torch.nn.Parameter(t) if kind == "parameter" else t.as_subclass(Tagged) if kind == "subclass"
                              else t.detach().clone().requires_grad_(True))
        for p, q in zip(want, as_tuple(function(**other))):
            assert same(p, q)


def spoiled(torch, t):
    """What no call may take in t's place."""
    yield None
    yield t.cpu()
    yield t.flatten()[:-1]
    yield torch.zeros(t.shape, dtype=torch.float16 if t.dtype != torch.float16 else torch.float32, device="cuda")
    if t.dim() == 2 and t.shape[0] > 1:
        yield t.t()                                                    # another shape (or, square, another order)
        wide = torch.zeros(t.shape[0], t.shape[1] * 2 + 256, dtype=t.dtype, device="cuda")
        yield wide[:, 1:2 * t.shape[1]:2]                             # elements apart
        yield wide[:, :t.shape[1]]                                    # rows further apart than the descriptor says
    if t.dim() == 1:
        yield torch.zeros(2 * t.shape[0], dtype=t.dtype, device="cuda")[::2]


OPTIONAL = {"weight", "bias", "y", "stats", "codes", "scales", "codes_t", "scales_t", "dx", "dweight", "dbias"}


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("name", NAMES)
def test_refused_tensors(A, name, native, monkeypatch):
    torch = torch_mod()
    function, good, outs = calls(A)[name]
    if not native:
        monkeypatch.setattr(A.stage_binding, "_native", _Nothing())
    for key, t in {**good, **outs}.items():
        if not isinstance(t, torch.Tensor):
            continue
        for bad in spoiled(torch, t):
            if bad is None and key in OPTIONAL and not (name == "backward" and key == "stats"):
                continue
            with pytest.raises(A.AcceptError):
                function(**{**good, **outs, key: bad})
    torch.cuda.synchronize()


@pytest.mark.parametrize("native", [True, False])
def test_refused_codes_and_workspaces(A, native, monkeypatch):
    torch = torch_mod()
    function, good, _ = calls(A)["matmul"]
    if not native:
        monkeypatch.setattr(A.stage_binding, "_native", _Nothing())
    f8 = torch.float8_e4m3fn
    stride = A.accept_block_stride(C)
    short = torch.zeros((R - 1) * stride + C, dtype=f8, device="cuda")          # the last row ends at C, not at a multiple of 16
    odd = torch.zeros(R * stride + 16, dtype=f8, device="cuda")[8:]
    for bad in (torch.as_strided(short, (R, C), (stride, 1)), torch.as_strided(odd, (R, C), (stride, 1), 8), good["a"].to(torch.float8_e5m2)):
        with pytest.raises(A.AcceptError):
            function(**{**good, "a": bad})
    function, good, outs = calls(A)["quantize"]
    short = torch.zeros((R - 1) * stride + C, dtype=f8, device="cuda")
    with pytest.raises(A.AcceptError):
        function(**{**good, **outs, "codes": torch.as_strided(short, (R, C), (stride, 1))})
    with pytest.raises(A.AcceptError):
        function(**{**good, "rowwise": False, "colwise": False})
    d = A.make_matmul_desc(100, 100, 8192)
    a = torch.zeros(100, 8192, dtype=f8, device="cuda")
    sa = torch.zeros(64, 100, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    sb = torch.zeros(64, 1, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    nbytes = A.accept_matmul_workspace_size(d)
    for ws in (torch.zeros(nbytes - 1, dtype=torch.uint8, device="cuda"), torch.zeros(nbytes, dtype=torch.uint8),
               torch.zeros(2 * nbytes, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(A.AcceptError):
            A.accept_block_matmul(d, a, sa, a, sb, workspace=ws)
    nd = A.make_norm_desc(R, C)
    _, good, _ = calls(A)["backward"]
    nbytes = A.accept_norm_workspace_size(nd)
    with pytest.raises(A.AcceptError):
        A.accept_layer_norm_backward(**good, workspace=torch.zeros(nbytes - 1, dtype=torch.uint8, device="cuda"))
    for bad in (A.make_norm_desc(R, C, eps=-1), A.make_norm_desc(R + 1, C), A.make_norm_desc(R, C, x_stride=C - 1)):
        with pytest.raises(A.AcceptError):
            A.accept_layer_norm(bad, good["x"])
        with pytest.raises(A.AcceptError):
            A.accept_layer_norm(A.make_block_desc(R, C), good["x"])
    torch.cuda.synchronize()
