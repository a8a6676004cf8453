"""Layer norm, its form that writes codes, and its gradients, against the formulas in 64 bits.

Bounds.  A row's sums are trees of float32 additions at most 64 deep (a lane's values, 64 lanes, at most 16 wavefronts), so a
sum of terms t is off by at most 64 U sum|t|, U = 2^-24; what follows it is a handful of roundings of U each.
"""
import numpy as np
import pytest

from oracle import stage_oracle as orc
from stage_util import U, code_values, dtype_of, exponents, f64, hidden, matrix, rounding, torch_mod, vector

pytestmark = pytest.mark.gpu
EPS = 1e-5
DEPTH = 64

# columns around what a vector, a block, one, four and eight wavefronts and a workgroup's registers hold
COLS = [1, 3, 7, 8, 63, 127, 128, 129, 256, 500, 767, 768, 1024, 1025, 1536, 2048, 2049, 4096, 4100, 5003, 8192, 8193, 12290, 16384, 16385, 20001]
TYPES = [("f32", "f32", "f32"), ("bf16", "bf16", "f32"), ("bf16", "f32", "bf16"), ("f32", "bf16", "bf16")]


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def code_of(A, name):
    return A.F32 if name == "f32" else A.BF16


def desc_of(A, rows, cols, types, **more):
    return A.make_norm_desc(rows, cols, x_dtype=code_of(A, types[0]), y_dtype=code_of(A, types[1]),
                            param_dtype=code_of(A, types[2]), **{"eps": EPS, **more})


def make(rows, cols, types, seed, pad=0, offset=0, shift=0.0):
    rng = np.random.default_rng(seed)
    x, x64 = matrix(hidden(rng, rows, cols) + shift, types[0], pad, offset)
    w, w64 = vector(1 + 0.1 * rng.standard_normal(cols), types[2])
    b, b64 = vector(0.1 * rng.standard_normal(cols), types[2])
    return rng, x, x64, w, w64, b, b64


def forward_bound(x, w, b, y, mean, rstd):
    d = np.abs(x - mean[:, None])
    return DEPTH * U * (np.abs(w) * rstd[:, None] * (np.abs(x).mean(axis=1)[:, None] + d) + np.abs(b) + np.abs(y))


def check_stats(stats, x, mean, rstd):
    got = f64(stats)
    size = np.abs(x).mean(axis=1)
    assert np.all(np.abs(got[0] - mean) <= DEPTH * U * (size + np.abs(mean)))
    # the variance is off by DEPTH U of itself, and by the square of the mean's error; a root halves that
    assert np.all(np.abs(got[1] - rstd) <= rstd * (DEPTH * U + (DEPTH * U * size * rstd) ** 2))


def check_forward(y, stats, x, w, b, out):
    want, mean, rstd = orc.layer_norm(x, w, b, EPS)
    check_stats(stats, x, mean, rstd)
    got = f64(y).reshape(want.shape)
    bound = forward_bound(x, w, b, want, mean, rstd)
    assert np.all(np.abs(got - want) <= bound + rounding(out, np.abs(want) + bound))


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_forward(A, cols, types):
    rows = 5
    _, x, x64, w, w64, b, b64 = make(rows, cols, types, cols)
    y, stats = A.accept_layer_norm(desc_of(A, rows, cols, types), x, w, b)
    assert y.shape == x.shape and y.dtype == dtype_of(types[1])
    check_forward(y, stats, x64, w64, b64, types[1])


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 63, 2049, 8200])
def test_forward_rows(A, rows):
    types = ("bf16", "bf16", "f32")
    _, x, x64, w, w64, b, b64 = make(rows, 130, types, rows)
    y, stats = A.accept_layer_norm(desc_of(A, rows, 130, types), x, w, b)
    check_forward(y, stats, x64, w64, b64, "bf16")


@pytest.mark.parametrize("types", TYPES[:2])
@pytest.mark.parametrize("cols,pad,offset", [(768, 8, 0), (767, 1, 1), (130, 3, 5), (5003, 7, 3), (20001, 9, 1)])
def test_strided_and_unaligned(A, cols, pad, offset, types):
    rows = 6
    torch = torch_mod()
    _, x, x64, w, w64, b, b64 = make(rows, cols, types, 7, pad, offset)
    d = desc_of(A, rows, cols, types, x_stride=cols + pad, y_stride=cols + 5)
    held = torch.full((rows, cols + 5), -7.0, dtype=dtype_of(types[1]), device="cuda")
    y, stats = A.accept_layer_norm(d, x, w, b, y=held[:, :cols])
    check_forward(y, stats, x64, w64, b64, types[1])
    assert torch.all(held[:, cols:] == -7)      # what lies between the rows stays


def test_without_weight_or_bias(A):
    types = ("f32", "f32", "f32")
    _, x, x64, w, w64, b, b64 = make(4, 300, types, 1)
    d = desc_of(A, 4, 300, types)
    for ww, bb in ((None, None), (w, None), (None, b)):
        y, stats = A.accept_layer_norm(d, x, ww, bb)
        check_forward(y, stats, x64, w64 if ww is not None else np.ones(300), b64 if bb is not None else np.zeros(300), "f32")


def test_large_mean_and_constant_rows(A):
    """The variance is that of the differences: a mean a thousand deviations away costs digits of x, not of the variance; a
    constant row has none."""
    types = ("f32", "f32", "f32")
    _, x, x64, w, w64, b, b64 = make(5, 1000, types, 2, shift=1000.0)
    y, stats = A.accept_layer_norm(desc_of(A, 5, 1000, types), x, w, b)
    check_forward(y, stats, x64, w64, b64, "f32")
    torch = torch_mod()
    x = torch.full((3, 256), 2.0, device="cuda")
    d = desc_of(A, 3, 256, types)
    y, stats = A.accept_layer_norm(d, x, None, None)
    assert torch.all(y == 0) and torch.all(stats[0] == 2)
    assert np.all(np.abs(f64(stats[1]) - EPS ** -0.5) <= 4 * U * EPS ** -0.5)


def test_values_that_are_not_finite_stay_in_their_rows(A):
    types = ("bf16", "f32", "f32")
    torch = torch_mod()
    _, x, x64, w, w64, b, b64 = make(6, 700, types, 3)
    d = desc_of(A, 6, 700, types)
    y0, s0 = A.accept_layer_norm(d, x, w, b)
    x[1, 5], x[3, 699], x[4, 0] = float("nan"), float("inf"), float("-inf")
    y, s = A.accept_layer_norm(d, x, w, b)
    for row in (0, 2, 5):
        assert torch.equal(y[row], y0[row]) and torch.equal(s[:, row], s0[:, row])
    for row in (1, 3, 4):
        assert torch.isnan(y[row]).all()


def test_no_rows(A):
    torch = torch_mod()
    d = desc_of(A, 0, 64, ("f32", "f32", "f32"))
    x = torch.empty(0, 64, device="cuda")
    y, stats = A.accept_layer_norm(d, x)
    assert y.shape == (0, 64) and stats.shape == (2, 0)
    codes, scales, _ = A.accept_layer_norm_quantize(d, x)
    assert codes.shape == (0, 64) and scales.shape == (1, 0)
    dx, dw, db = A.accept_layer_norm_backward(d, x, x, None, stats)
    assert dx.shape == (0, 64) and torch.all(dw == 0) and torch.all(db == 0)


# ------------------------------------------------------------------------------------- to codes
@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("x_type", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1, 5, 127, 128, 129, 300, 768, 1025, 4096, 5003, 8200, 16385, 20001])
def test_quantized(A, cols, x_type, code):
    rows = 5
    types = (x_type, "f32", "f32")
    torch = torch_mod()
    _, x, x64, w, w64, b, b64 = make(rows, cols, types, cols, pad=3)
    codes, scales, stats = A.accept_layer_norm_quantize(desc_of(A, rows, cols, types, code=code, x_stride=cols + 3), x, w, b)
    want, mean, rstd = orc.layer_norm(x64, w64, b64, EPS)
    check_stats(stats, x64, mean, rstd)
    bound = forward_bound(x64, w64, b64, want, mean, rstd)
    blocks = -(-cols // 128)
    e = exponents(scales)
    assert e.shape == (blocks, rows)
    up = np.zeros((rows, blocks * 128))
    lo, hi = up.copy(), up.copy()
    lo[:, :cols], hi[:, :cols] = np.maximum(np.abs(want) - bound, 0), np.abs(want) + bound
    lo, hi = (v.reshape(rows, blocks, 128).max(axis=2).T for v in (lo, hi))
    assert np.all(orc.exponent(lo, code) <= e) and np.all(e <= orc.exponent(hi, code))
    scale = orc.spread(e, rows, cols, 1)
    got = code_values(codes, code) * scale
    assert np.all(np.abs(got - want) <= 0.5 * orc.step((np.abs(want) + bound) / scale, code) * scale + bound)
    whole = torch.as_strided(codes, (rows, blocks * 128), (blocks * 128, 1))
    assert torch.all(whole.contiguous().view(torch.uint8)[:, cols:] == 0)   # the rest of the last block


# ------------------------------------------------------------------------------------ gradients
def check_backward(got, dy, x, w, stats, types, rows):
    mean, rstd = f64(stats)
    dx, dw, db = orc.layer_norm_backward(dy, x, w, mean, rstd)
    h = (x - mean[:, None]) * rstd[:, None]
    g = dy * w
    size = np.abs(g) + np.abs(g).mean(axis=1)[:, None] + np.abs(h) * np.abs(g * h).mean(axis=1)[:, None]
    # h itself is off by U of x's and the mean's size
    size = size + (np.abs(x) + np.abs(mean[:, None])) * rstd[:, None] * np.abs((g * h).mean(axis=1))[:, None]
    off_h = 2 * U * (np.abs(x) + np.abs(mean[:, None])) * rstd[:, None]
    bound = DEPTH * U * rstd[:, None] * size + rstd[:, None] * np.abs(h) * (np.abs(g) * off_h).mean(axis=1)[:, None]
    got_dx = f64(got[0]).reshape(dx.shape)
    assert np.all(np.abs(got_dx - dx) <= bound + rounding(types[0], np.abs(dx) + bound))
    deep = (rows / 512 + 128) * U
    if got[1] is not None:
        b = deep * np.abs(dy * h).sum(axis=0) + (np.abs(dy) * off_h).sum(axis=0)
        assert np.all(np.abs(f64(got[1]) - dw) <= b + rounding(types[2], np.abs(dw) + b))
    if got[2] is not None:
        b = deep * np.abs(dy).sum(axis=0)
        assert np.all(np.abs(f64(got[2]) - db) <= b + rounding(types[2], np.abs(db) + b))


def backward_case(A, rows, cols, types, pad=0, offset=0):
    rng, x, x64, w, w64, b, b64 = make(rows, cols, types, rows + cols, pad, offset)
    dy, dy64 = matrix(1e-3 * rng.standard_normal((rows, cols)), types[1], pad, offset)
    d = desc_of(A, rows, cols, types, x_stride=cols + pad, y_stride=cols + pad, dx_stride=cols + pad)
    _, stats = A.accept_layer_norm(d, x, w, b)
    return d, x, x64, w, w64, dy, dy64, stats


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_backward(A, cols, types):
    rows = 9
    d, x, x64, w, w64, dy, dy64, stats = backward_case(A, rows, cols, types)
    got = A.accept_layer_norm_backward(d, dy, x, w, stats)
    assert got[0].dtype == x.dtype and got[1].dtype == got[2].dtype == w.dtype
    check_backward(got, dy64, x64, w64, stats, types, rows)


@pytest.mark.parametrize("cols", [96, 1100, 9000])
@pytest.mark.parametrize("rows", [1, 3, 64, 65, 515, 4099])
def test_backward_rows(A, rows, cols):
    types = ("bf16", "bf16", "f32")
    d, x, x64, w, w64, dy, dy64, stats = backward_case(A, rows, cols, types)
    check_backward(A.accept_layer_norm_backward(d, dy, x, w, stats), dy64, x64, w64, stats, types, rows)


@pytest.mark.parametrize("cols,pad,offset", [(768, 8, 0), (767, 1, 1), (130, 3, 5), (5003, 7, 3), (20001, 9, 1)])
def test_backward_strided(A, cols, pad, offset):
    types = ("bf16", "bf16", "f32")
    d, x, x64, w, w64, dy, dy64, stats = backward_case(A, 7, cols, types, pad, offset)
    check_backward(A.accept_layer_norm_backward(d, dy, x, w, stats), dy64, x64, w64, stats, types, 7)


@pytest.mark.parametrize("cols", [300, 9000])
def test_backward_of_what_is_wanted(A, cols):
    types = ("f32", "f32", "f32")
    torch = torch_mod()
    d, x, x64, w, w64, dy, dy64, stats = backward_case(A, 20, cols, types)
    full = A.accept_layer_norm_backward(d, dy, x, w, stats)
    for weight, bias in ((False, False), (True, False), (False, True)):
        got = A.accept_layer_norm_backward(d, dy, x, w, stats, need_weight=weight, need_bias=bias)
        assert torch.equal(got[0], full[0])
        assert (got[1] is None) == (not weight) and (not weight or torch.equal(got[1], full[1]))
        assert (got[2] is None) == (not bias) and (not bias or torch.equal(got[2], full[2]))
    got = A.accept_layer_norm_backward(d, dy, x, None, stats)   # no weight: ones
    check_backward(got, dy64, x64, np.ones(cols), stats, types, 20)


def test_gradient_against_differences(A):
    """The directional derivative of sum(dy * y) along every input, by central differences of the kernel's own forward pass.

    With x of size 1 and steps of h = 2^-7 the third-order term is about h^2 of the derivative, and forward's rounding
    (64 U, over 2 h, summed at random over the outputs) some 1e-3 of it at most."""
    torch = torch_mod()
    rows, cols, h = 12, 200, 2.0 ** -7
    types = ("f32", "f32", "f32")
    rng = np.random.default_rng(11)
    dev = lambda v: torch.from_numpy(v.astype(np.float32)).cuda()
    x, dy = dev(rng.standard_normal((rows, cols))), dev(rng.standard_normal((rows, cols)))
    w, b = dev(1 + 0.1 * rng.standard_normal(cols)), dev(rng.standard_normal(cols))
    d = desc_of(A, rows, cols, types)
    _, stats = A.accept_layer_norm(d, x, w, b)
    dx, dw, db = A.accept_layer_norm_backward(d, dy, x, w, stats)
    value = lambda x, w, b: float((dy.double() * A.accept_layer_norm(d, x, w, b)[0].double()).sum())
    for i, g in enumerate((dx, dw, db)):
        args = [x, w, b]
        # along the gradient itself, so that the derivative is its norm and far from 0
        v = g / g.norm() * g.numel() ** 0.5
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + h * v, args[i] - h * v
        want = (value(*up) - value(*down)) / (2 * h)
        got = float((g.double() * v.double()).sum())
        assert abs(got - want) <= 1e-2 * abs(want)


# ------------------------------------------------------------------------- streams, repeats, size
def test_same_bits_again_and_on_another_stream(A):
    torch = torch_mod()
    types = ("bf16", "bf16", "f32")
    d, x, x64, w, w64, dy, dy64, stats = backward_case(A, 3000, 768, types)
    first = [*A.accept_layer_norm(d, x, w, None), *A.accept_layer_norm_backward(d, dy, x, w, stats)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        late = torch.zeros_like(x)
        late.copy_(x)                     # on that stream just before: a call on another one would miss it
        again = [*A.accept_layer_norm(d, late, w, None), *A.accept_layer_norm_backward(d, dy, late, w, stats)]
    s.synchronize()
    for p, q in zip(first, again):
        assert torch.equal(p, q)


def test_offsets_beyond_32_bits(A):
    torch = torch_mod()
    rows, cols, stride = 3, 300, (1 << 31) + 8
    rng = np.random.default_rng(5)
    held = torch.empty(2 * stride + cols, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(held, (rows, cols), (stride, 1))
    values = torch.from_numpy(hidden(rng, rows, cols)).bfloat16().cuda()
    for r in range(rows):
        x[r].copy_(values[r])
    types = ("bf16", "bf16", "f32")
    y, stats = A.accept_layer_norm(desc_of(A, rows, cols, types, x_stride=stride), x)
    y0, stats0 = A.accept_layer_norm(desc_of(A, rows, cols, types), values)
    assert torch.equal(y, y0) and torch.equal(stats, stats0)
    dy = torch.randn(rows, cols, device="cuda").bfloat16()
    dx = A.accept_layer_norm_backward(desc_of(A, rows, cols, types, x_stride=stride), dy, x, None, stats)[0]
    dx0 = A.accept_layer_norm_backward(desc_of(A, rows, cols, types), dy, values, None, stats)[0]
    assert torch.equal(dx, dx0)
