"""Quantization to blocks of 128 in 8-bit floating point (codes and scales are exact), and the products of such operands.

Bound of a product.  A term is a product of two codes of at most 4 significant bits times a power of two, so it is exact in
float32, and k of them are added in some order in float32: at most k U sum|terms| off, U = 2^-24, and one rounding to the output's type.
For bfloat16 results a term may also lose what is below 2^-13 of the largest of its eight, so eight terms 8 * 2^-13 of that largest one,
which is at most the sum of their magnitudes: 2^-10 sum|terms|.
"""
import numpy as np
import pytest

from oracle import stage_oracle as orc
from stage_util import U, code_values, dtype_of, exponents, f64, hidden, matrix, rounding, torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def code_of(A, name):
    return A.F32 if name == "f32" else A.BF16


# ----------------------------------------------------------------------------------- quantization
def check_codes(codes, scales, x, group, code):
    want, e = orc.quantize(x, group, code)
    assert np.array_equal(exponents(scales), e)
    assert np.array_equal(code_values(codes, code), want)
    torch = torch_mod()
    rows, cols = x.shape
    stride = -(-cols // 128) * 128
    whole = torch.as_strided(codes, (rows, stride), (stride, 1)).contiguous().view(torch.uint8)
    assert torch.all(whole[:, cols:] == 0)


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [1, 128])
@pytest.mark.parametrize("ways", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 300), (5, 128), (127, 129), (128, 128), (129, 127), (257, 515), (300, 64)])
def test_quantize(A, rows, cols, ways, group, dtype, code):
    rng = np.random.default_rng(rows * 1000 + cols)
    x, x64 = matrix(hidden(rng, rows, cols) * np.exp(rng.standard_normal((rows, 1))), dtype, pad=rows % 4, offset=cols % 3)
    d = A.make_block_desc(rows, cols, group=group, in_dtype=code_of(A, dtype), code=code, x_stride=cols + rows % 4)
    codes, scales, codes_t, scales_t = A.accept_block_quantize(d, x, rowwise=ways[0], colwise=ways[1])
    if ways[0]:
        check_codes(codes, scales, x64, group, code)
    else:
        assert codes is None and scales is None
    if ways[1]:
        check_codes(codes_t, scales_t, np.ascontiguousarray(x64.T), group, code)
    else:
        assert codes_t is None and scales_t is None


@pytest.mark.parametrize("code", [0, 1])
def test_every_bfloat16_value_is_rounded_to_the_nearest(A, code):
    """Each finite bfloat16, beside the largest value of the code so that the scale is 1; ties go to even."""
    torch = torch_mod()
    top = orc.LARGEST[code]
    every = (torch.arange(65536, dtype=torch.int32) << 16).view(torch.float32)
    every = every[torch.isfinite(every) & (every.abs() <= top)]
    n = -(-len(every) // 127)
    x = torch.zeros(n, 128)
    x[:, 0] = top
    x[:, 1:] = torch.nn.functional.pad(every, (0, n * 127 - len(every))).view(n, 127)
    codes, scales, _, _ = A.accept_block_quantize(A.make_block_desc(n, 128, code=code), x.cuda())
    assert np.all(exponents(scales) == 0)
    assert np.array_equal(code_values(codes, code), orc.nearest(x.double().numpy(), code))


@pytest.mark.parametrize("code", [0, 1])
def test_scales_at_their_limits(A, code):
    """The largest magnitude exactly on, just under and just over a power of two times the largest code; zeros; the smallest and
    largest floats."""
    torch = torch_mod()
    c = []
    for e in (-99, -20, 0, 1, 60):
        v = np.float32(orc.LARGEST[code] * 2.0 ** e)
        c += [v, np.nextafter(v, np.float32(0)), np.nextafter(v, np.float32(np.inf))]
    c += [0.0, np.float32(1e-45), np.float32(2.0 ** -126), np.float32(2.0 ** -100), np.finfo(np.float32).max, 1.0]
    x = np.zeros((len(c), 256), dtype=np.float32)
    x[:, 3] = c
    x[:, 200] = -np.asarray(c, dtype=np.float32) / 3
    for group in (1, 128):
        codes, scales, codes_t, scales_t = A.accept_block_quantize(A.make_block_desc(*x.shape, group=group, code=code),
                                                                   torch.from_numpy(x).cuda(), colwise=True)
        check_codes(codes, scales, x.astype(np.float64), group, code)
        check_codes(codes_t, scales_t, np.ascontiguousarray(x.T).astype(np.float64), group, code)


@pytest.mark.parametrize("code", [0, 1])
def test_quantize_values_that_are_not_finite(A, code):
    """A NaN stays one and does not touch its block; an infinity takes the block's scale to its largest, and its own code is NaN
    (E4M3) or an infinity (E5M2)."""
    torch = torch_mod()
    rng = np.random.default_rng(3)
    x = rng.standard_normal((6, 384)).astype(np.float32)
    clean, _, _, _ = A.accept_block_quantize(A.make_block_desc(6, 384, code=code), torch.from_numpy(x).cuda())
    clean = code_values(clean, code)
    x[1, 130], x[2, 5] = np.nan, -np.inf
    for colwise in (False, True):
        codes, scales, _, _ = A.accept_block_quantize(A.make_block_desc(6, 384, code=code), torch.from_numpy(x).cuda(), colwise=colwise)
        got, e = code_values(codes, code), exponents(scales)
        same = np.ones(x.shape, dtype=bool)
        same[2, :128] = False
        same[1, 128:256] = False      # its largest value may have been the one
        assert np.array_equal(got[same], clean[same])
        assert np.isnan(got[1, 130]) and np.isfinite(np.delete(got[1], 130)).all()
        row = x[1, 128:256].astype(np.float64)
        row[2] = 0
        want, ee = orc.quantize(row[None], 1, code)
        assert e[1, 1] == ee[0, 0] and np.array_equal(np.delete(got[1, 128:256], 2), np.delete(want[0], 2))
        assert e[0, 2] == (120 if code == 0 else 113)
        assert np.isnan(got[2, 5]) if code == 0 else got[2, 5] == -np.inf
        assert np.all(np.delete(got[2, :128], 5) == 0)


def test_quantize_nothing(A):
    torch = torch_mod()
    for rows, cols in ((0, 200), (200, 0), (0, 0)):
        x = torch.empty(rows, cols, device="cuda")
        codes, scales, codes_t, scales_t = A.accept_block_quantize(A.make_block_desc(rows, cols), x, colwise=True)
        assert codes.shape == (rows, cols) and codes_t.shape == (cols, rows)
        assert scales.shape == (-(-cols // 128), rows) and scales_t.shape == (-(-rows // 128), cols)


# ----------------------------------------------------------------------------------------- products
def operand(rng, rows, k, group, code, pad=0, small=False):
    """Codes, scales, and their values.  What lies behind column k of a row is NaN."""
    torch = torch_mod()
    if small:
        v = rng.integers(-8, 9, size=(rows, k)).astype(np.float64)
        e = rng.integers(-2, 3, size=(-(-k // 128), -(-rows // group)))
    else:
        v, e = orc.quantize(hidden(rng, rows, k) if rows and k else np.zeros((rows, k)), group, code)
    stride = -(-k // 16) * 16 + 16 * pad
    held = torch.full((rows, stride), float("nan"), device="cuda").to((torch.float8_e4m3fn, torch.float8_e5m2)[code])
    held[:, :k] = torch.from_numpy(v).float().cuda().to(held.dtype)
    scales = torch.from_numpy(np.ascontiguousarray(e + 127).astype(np.uint8)).cuda().view(torch.float8_e8m0fnu)
    return held[:, :k], scales, v * orc.spread(e, rows, k, group)


def multiply(A, rng, m, n, k, out="f32", codes=(0, 0), groups=(1, 128), pads=(0, 0), small=False, y_pad=0):
    a, sa, a64 = operand(rng, m, k, groups[0], codes[0], pads[0], small)
    b, sb, b64 = operand(rng, n, k, groups[1], codes[1], pads[1], small)
    d = A.make_matmul_desc(m, n, k, out_dtype=code_of(A, out), a_code=codes[0], b_code=codes[1], a_group=groups[0],
                           b_group=groups[1], a_stride=a.stride(0), b_stride=b.stride(0), y_stride=n + y_pad if y_pad else 0)
    return A.accept_block_matmul(d, a, sa, b, sb), a64, b64


def check_product(y, a, b, out):
    want = a @ b.T
    bound = (max(a.shape[1], 1) * U + (2.0 ** -10 if out == "bf16" else 0)) * (np.abs(a) @ np.abs(b).T)
    assert y.dtype == dtype_of(out) and y.shape == want.shape
    assert np.all(np.abs(f64(y) - want) <= bound + rounding(out, np.abs(want) + bound))


@pytest.mark.parametrize("m,n,k", [
    (1, 1, 1), (1, 16, 128), (1, 17, 300), (1, 4096, 2048), (2, 100, 1000), (15, 64, 129), (16, 33, 4100), (17, 48, 640),
    (32, 130, 100), (33, 16, 257), (48, 512, 2048), (63, 65, 1023), (64, 96, 128), (65, 64, 128), (65, 1, 5), (100, 130, 300),
    (127, 129, 2000), (128, 128, 128), (129, 127, 384), (256, 256, 1024), (257, 300, 8144), (300, 1000, 100), (640, 1030, 515)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_product(A, m, n, k, out):
    y, a, b = multiply(A, np.random.default_rng(m + n + k), m, n, k, out)
    check_product(y, a, b, out)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 20, 16500), (9, 33, 20001), (20, 130, 4200), (64, 40, 5000), (130, 140, 2100), (1, 1, 16400)])
def test_product_in_parts(A, m, n, k, out):
    """Few results over a long axis: parts of it, of unequal length, the last one with an incomplete block."""
    assert A.accept_matmul_workspace_size(A.make_matmul_desc(m, n, k, out_dtype=code_of(A, out))) > 0
    y, a, b = multiply(A, np.random.default_rng(k), m, n, k, out)
    check_product(y, a, b, out)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(40, 8200, 300), (64, 8300, 1100), (17, 8192, 129)])
def test_product_of_few_rows_with_many(A, m, n, k, out):
    """Up to 64 rows and enough columns for 32 of them a workgroup."""
    y, a, b = multiply(A, np.random.default_rng(n), m, n, k, out)
    check_product(y, a, b, out)


@pytest.mark.parametrize("m,n,k", [(3600, 3500, 130), (4000, 3400, 1), (3585, 3585, 400)])
def test_product_of_large_tiles(A, m, n, k):
    """Enough results for tiles of 256 x 256, none of them whole at the edges."""
    y, a, b = multiply(A, np.random.default_rng(m), m, n, k, "bf16")
    check_product(y, a, b, "bf16")


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("codes", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("m,n,k", [(3, 50, 200), (40, 300, 1500), (200, 150, 700)])
def test_product_of_types(A, m, n, k, codes, out):
    y, a, b = multiply(A, np.random.default_rng(7), m, n, k, out, codes)
    check_product(y, a, b, out)


@pytest.mark.parametrize("groups", [(1, 1), (1, 128), (128, 1), (128, 128)])
@pytest.mark.parametrize("m,n,k", [(20, 300, 400), (300, 400, 513)])
def test_product_of_groups(A, m, n, k, groups):
    y, a, b = multiply(A, np.random.default_rng(9), m, n, k, groups=groups)
    check_product(y, a, b, "f32")


@pytest.mark.parametrize("m,n,k", [(1, 300, 700), (60, 257, 1025), (200, 131, 5000), (300, 300, 200)])
def test_product_of_small_integers_is_exact(A, m, n, k):
    """Codes that are whole numbers up to 8 and scales of 2^-2 .. 2^2: every sum is a multiple of 2^-4 below 2^24 of them."""
    y, a, b = multiply(A, np.random.default_rng(13), m, n, k, small=True, pads=(1, 3), y_pad=5)
    assert np.array_equal(f64(y), a @ b.T)
    assert y.stride(0) == n + 5


def test_product_over_nothing_and_of_nothing(A):
    torch = torch_mod()
    for m, n in ((3, 40), (200, 70)):
        for out in ("f32", "bf16"):
            y, _, _ = multiply(A, np.random.default_rng(1), m, n, 0, out)
            assert y.shape == (m, n) and torch.all(y == 0)
    for m, n in ((0, 40), (40, 0)):
        y, _, _ = multiply(A, np.random.default_rng(1), m, n, 300)
        assert y.shape == (m, n)


def test_scales_far_apart(A):
    """Each block's scales far from 1, their products near it; and products beyond the largest float32."""
    torch = torch_mod()
    rng = np.random.default_rng(17)
    for m in (5, 150):
        k, n = 384, 200
        v = rng.integers(-8, 9, size=(m, k)).astype(np.float32)
        w = rng.integers(-8, 9, size=(n, k)).astype(np.float32)
        ea = np.tile(np.array([[-100], [90], [0]]), (1, m))
        eb = np.tile(np.array([[101], [-90], [1]]), (1, n))
        dev = lambda t: torch.from_numpy(t).cuda().to(torch.float8_e4m3fn)
        byte = lambda e: torch.from_numpy((e + 127).astype(np.uint8)).cuda().view(torch.float8_e8m0fnu)
        d = A.make_matmul_desc(m, n, k, b_group=1)
        y = A.accept_block_matmul(d, dev(v), byte(ea), dev(w), byte(eb))
        v64, w64 = v.astype(np.float64), w.astype(np.float64)
        want = sum(v64[:, 128 * q:128 * q + 128] @ w64[:, 128 * q:128 * q + 128].T * 2.0 ** (ea[q, 0] + eb[q, 0]) for q in range(3))
        assert np.array_equal(f64(y), want)
        big = A.accept_block_matmul(d, dev(np.ones_like(v)), byte(np.full_like(ea, 100)), dev(np.ones_like(w)), byte(np.full_like(eb, 100)))
        assert torch.isinf(big).all()


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("codes", [(0, 0), (1, 0), (0, 1), (1, 1)])
@pytest.mark.parametrize("m", [4, 130])
def test_product_of_every_code(A, m, codes, out):
    """Rows of one code each (all finite ones in turn) against rows with one 1 in them: every code as it is, subnormal ones too."""
    torch = torch_mod()
    finite = [v for v in range(256) if np.isfinite(orc.decode(v, codes[0]))]
    rows = torch.tensor([finite[i % len(finite)] for i in range(m * 70)], dtype=torch.uint8).view(m, 70)
    a = torch.zeros(m, 128, dtype=torch.uint8)
    a[:, :70] = rows
    b = torch.eye(70, 128).to((torch.float8_e4m3fn, torch.float8_e5m2)[codes[1]])
    types = (torch.float8_e4m3fn, torch.float8_e5m2)
    one = lambda r: torch.full((1, r), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    d = A.make_matmul_desc(m, 70, 128, out_dtype=code_of(A, out), a_code=codes[0], b_code=codes[1], b_group=1)
    y = A.accept_block_matmul(d, a.cuda().view(types[codes[0]]), one(m), b.cuda(), one(70))
    assert np.array_equal(f64(y), orc.decode(rows.numpy(), codes[0]))


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m", [3, 150])
def test_codes_that_are_not_finite_stay_in_their_rows(A, m, out):
    torch = torch_mod()
    rng = np.random.default_rng(19)
    a, sa, _ = operand(rng, m, 500, 1, 0)
    b, sb, _ = operand(rng, 90, 500, 128, 0)
    d = A.make_matmul_desc(m, 90, 500, out_dtype=code_of(A, out), a_stride=a.stride(0), b_stride=b.stride(0))
    y0 = A.accept_block_matmul(d, a, sa, b, sb)
    nan = torch.full((), float("nan"), device="cuda").to(a.dtype)
    a[1, 490], b[7, 0] = nan, nan
    y = A.accept_block_matmul(d, a, sa, b, sb)
    bad = torch.zeros(m, 90, dtype=torch.bool, device="cuda")
    bad[1], bad[:, 7] = True, True
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], y0[~bad])


def test_training_products(A):
    """The three products of a linear layer from one quantization of each tensor: y = x w^T, dx = dy w, dw = dy^T x."""
    torch = torch_mod()
    rng = np.random.default_rng(23)
    m, k, n = 300, 200, 260
    x, x64 = matrix(hidden(rng, m, k), "bf16")
    w, w64 = matrix(rng.standard_normal((n, k)) * k ** -0.5, "f32")
    dy, dy64 = matrix(1e-3 * rng.standard_normal((m, n)), "bf16")
    xc, xs, xct, xst = A.accept_block_quantize(A.make_block_desc(m, k, in_dtype=A.BF16), x, colwise=True)
    wc, ws, wct, wst = A.accept_block_quantize(A.make_block_desc(n, k, group=128), w, colwise=True)
    gc, gs, gct, gst = A.accept_block_quantize(A.make_block_desc(m, n, in_dtype=A.BF16, code=A.E5M2), dy, colwise=True)

    def values(v, group, code):
        c, e = orc.quantize(v, group, code)
        return c * orc.spread(e, *v.shape, group)

    y = A.accept_block_matmul(A.make_matmul_desc(m, n, k), xc, xs, wc, ws)
    check_product(y, values(x64, 1, 0), values(w64, 128, 0), "f32")
    dx = A.accept_block_matmul(A.make_matmul_desc(m, k, n, a_code=A.E5M2), gc, gs, wct, wst)
    check_product(dx, values(dy64, 1, 1), values(np.ascontiguousarray(w64.T), 128, 0), "f32")
    dw = A.accept_block_matmul(A.make_matmul_desc(n, k, m, a_code=A.E5M2, b_group=1), gct, gst, xct, xst)
    check_product(dw, values(np.ascontiguousarray(dy64.T), 1, 1), values(np.ascontiguousarray(x64.T), 1, 0), "f32")


@pytest.mark.parametrize("m,n,k", [(1, 64, 8000), (300, 200, 3000)])
def test_same_bits_again_on_another_stream_and_with_a_given_workspace(A, m, n, k):
    torch = torch_mod()
    rng = np.random.default_rng(29)
    a, sa, _ = operand(rng, m, k, 1, 0)
    b, sb, _ = operand(rng, n, k, 128, 0)
    d = A.make_matmul_desc(m, n, k, a_stride=a.stride(0), b_stride=b.stride(0))
    y = A.accept_block_matmul(d, a, sa, b, sb)
    nbytes = A.accept_matmul_workspace_size(d)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ws = torch.full((max(nbytes, 1),), 255, dtype=torch.uint8, device="cuda")   # NaN, if it were read before it is written
        again = A.accept_block_matmul(d, a, sa, b, sb, workspace=ws)
    s.synchronize()
    assert torch.equal(y, again)


def test_codes_beyond_32_bits(A):
    torch = torch_mod()
    rng = np.random.default_rng(31)
    k, n, stride = 300, 80, (1 << 31) + 16
    for m in (3,):
        held = torch.empty((m - 1) * stride + 304, dtype=torch.float8_e4m3fn, device="cuda")
        a, sa, a64 = operand(rng, m, k, 1, 0)
        b, sb, b64 = operand(rng, n, k, 128, 0)
        far = torch.as_strided(held, (m, k), (stride, 1))
        for r in range(m):
            far[r].copy_(a[r])
        y = A.accept_block_matmul(A.make_matmul_desc(m, n, k, a_stride=stride, b_stride=b.stride(0)), far, sa, b, sb)
        check_product(y, a64, b64, "f32")
        # and as the other operand, through the tiles
        c, sc, c64 = operand(rng, 100, k, 1, 0)
        y = A.accept_block_matmul(A.make_matmul_desc(100, m, k, a_stride=c.stride(0), b_stride=stride, b_group=1), c, sc, far, sa)
        check_product(y, c64, a64, "f32")


def test_in_a_graph(A):
    """Captured and replayed with other work between, the outputs are those of the calls themselves."""
    torch = torch_mod()
    x = torch.randn(40, 700, device="cuda")
    w = torch.randn(130, 700, device="cuda")
    nd = A.make_norm_desc(40, 700)
    wd, md = A.make_block_desc(130, 700, group=128), A.make_matmul_desc(40, 130, 700)
    bd, gd = A.make_block_desc(40, 130, code=A.E5M2), A.make_matmul_desc(40, 700, 130, a_code=A.E5M2)

    def step():
        codes, scales, stats = A.accept_layer_norm_quantize(nd, x)
        wc, ws, wct, wst = A.accept_block_quantize(wd, w, colwise=True)
        y = A.accept_block_matmul(md, codes, scales, wc, ws)
        gc, gs, _, _ = A.accept_block_quantize(bd, y)
        dh = A.accept_block_matmul(gd, gc, gs, wct, wst)
        return (y, *A.accept_layer_norm_backward(nd, dh, x, None, stats))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        x.copy_(torch.randn(40, 700, device="cuda") * (i + 1))
        w.copy_(torch.randn(130, 700, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        for p, q in zip(got, step()):
            assert torch.equal(p, q)
        torch.cuda.synchronize()
