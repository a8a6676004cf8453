"""Layer norm where a workgroup has several rows, one after the other, and several wavefronts share a row: their sums' places in shared
memory alternate, and the next row's values are asked for during this one.  More rows than workgroups (1024) in every form: one
wavefront a row, four, eight, rows that registers do not hold, and rows shorter than a vector.  Bounds and checks are those of the other tests of
the norm."""
import numpy as np
import pytest

import test_gpu_stage_norm as norm
from oracle import stage_oracle as orc
from stage_util import code_values, exponents, f64, torch_mod

pytestmark = pytest.mark.gpu
A = norm.A
SIZES = [(4500, 300), (5001, 5), (2600, 2049), (1531, 5003), (2100, 8200), (1100, 16385), (3000, 3)]


@pytest.mark.parametrize("types", [("bf16", "bf16", "f32"), ("f32", "f32", "bf16")])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward_of_many_rows(A, rows, cols, types):
    _, x, x64, w, w64, b, b64 = norm.make(rows, cols, types, rows)
    y, stats = A.accept_layer_norm(norm.desc_of(A, rows, cols, types), x, w, b)
    norm.check_forward(y, stats, x64, w64, b64, types[1])


@pytest.mark.parametrize("x_type", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantized_many_rows(A, rows, cols, x_type):
    """Scales: those of the exact output's largest value, give or take its bound; values: half a step of the code and the bound."""
    types = (x_type, "f32", "f32")
    _, x, x64, w, w64, b, b64 = norm.make(rows, cols, types, rows + 1)
    codes, scales, stats = A.accept_layer_norm_quantize(norm.desc_of(A, rows, cols, types), x, w, b)
    want, mean, rstd = orc.layer_norm(x64, w64, b64, norm.EPS)
    norm.check_stats(stats, x64, mean, rstd)
    bound = norm.forward_bound(x64, w64, b64, want, mean, rstd)
    blocks = -(-cols // 128)
    e = exponents(scales)
    pad = ((0, 0), (0, blocks * 128 - cols))
    lo, hi = (np.pad(v, pad).reshape(rows, blocks, 128).max(axis=2).T for v in (np.maximum(np.abs(want) - bound, 0), np.abs(want) + bound))
    assert np.all(orc.exponent(lo, 0) <= e) and np.all(e <= orc.exponent(hi, 0))
    scale = orc.spread(e, rows, cols, 1)
    assert np.all(np.abs(code_values(codes, 0) * scale - want) <= 0.5 * orc.step((np.abs(want) + bound) / scale, 0) * scale + bound)


@pytest.mark.parametrize("rows,cols", [(4500, 300), (5001, 5), (2600, 2049), (1531, 5003), (1100, 16385), (1100, 20001)])
def test_backward_of_many_rows(A, rows, cols):
    types = ("bf16", "bf16", "f32")
    d, x, x64, w, w64, dy, dy64, stats = norm.backward_case(A, rows, cols, types)
    norm.check_backward(A.accept_layer_norm_backward(d, dy, x, w, stats), dy64, x64, w64, stats, types, rows)


@pytest.mark.parametrize("rows,cols", SIZES)
def test_rows_do_not_depend_on_each_other(A, rows, cols):
    """The same bits whichever workgroup and turn a row falls to: the rows in another order, and one alone."""
    torch = torch_mod()
    x = torch.randn(rows, cols, device="cuda").bfloat16()
    order = torch.randperm(rows, device="cuda")
    d = A.make_norm_desc(rows, cols, x_dtype=A.BF16, y_dtype=A.BF16)
    y, stats = A.accept_layer_norm(d, x)
    z, other = A.accept_layer_norm(d, x[order].contiguous())
    assert torch.equal(z, y[order]) and torch.equal(other, stats[:, order])
    codes, scales, _ = A.accept_layer_norm_quantize(d, x)
    c, s, _ = A.accept_layer_norm_quantize(d, x[order].contiguous())
    bits = lambda t: t.contiguous().view(torch.uint8)
    assert torch.equal(bits(c), bits(codes)[order]) and torch.equal(bits(s), bits(scales)[:, order])
    one = A.make_norm_desc(1, cols, x_dtype=A.BF16, y_dtype=A.BF16)
    last = A.accept_layer_norm(one, x[-1:])[0]
    assert torch.equal(last[0], y[-1])
