"""Products whose scales reach the ends of their range, 2^-100 to 2^120, where a code times its scale is beyond float32 and the
product of both operands is not.

The codes are whole multiples of one power of two (the largest codes of their type) against -1, 0 and 1, so every sum of them is exact in
float32 and in the 8-bit instruction (multiples within 2^4 of each other), and so is its product with the scales: the results are compared for
equality, rounded once where they are bfloat16.
"""
import numpy as np
import pytest

from oracle import stage_oracle as orc
from stage_util import torch_mod

pytestmark = pytest.mark.gpu
# unit, from, to.  E4M3: 256 .. 448, E5M2: 32768 .. 57344
TOPS = ((32.0, 8, 14), (8192.0, 4, 7))


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def device(values, code):
    torch = torch_mod()
    return torch.from_numpy(values).float().cuda().to((torch.float8_e4m3fn, torch.float8_e5m2)[code])


def scales(e):
    torch = torch_mod()
    return torch.from_numpy(np.ascontiguousarray(e + 127).astype(np.uint8)).cuda().view(torch.float8_e8m0fnu)


def large(rng, rows, k, code):
    """The largest codes of the type, of either sign, and zeros."""
    unit, low, high = TOPS[code]
    return unit * rng.integers(low, high + 1, size=(rows, k)) * rng.choice([-1.0, 0.0, 1.0], size=(rows, k))


def product(A, a, ea, b, eb, out, codes):
    m, k = a.shape
    n = b.shape[0]
    whole = A.accept_block_stride(k)
    held = [device(np.pad(v, ((0, 0), (0, whole - k))), c) for v, c in zip((a, b), codes)]
    d = A.make_matmul_desc(m, n, k, out_dtype=A.F32 if out == "f32" else A.BF16, a_code=codes[0], b_code=codes[1], b_group=1)
    return A.accept_block_matmul(d, held[0][:, :k], scales(ea), held[1][:, :k], scales(eb))


def rounded(want, out):
    """float64 to the type: float32 first where both are exact, infinities beyond its largest."""
    torch = torch_mod()
    with np.errstate(over="ignore"):
        t = torch.from_numpy(want.astype(np.float32))
    return t if out == "f32" else t.to(torch.bfloat16)


# few rows (one to four of 16, whole chip or not), tiles of 128 and of 256, parts of the contracted axis, incomplete blocks
SIZES = [(1, 20, 128), (1, 64, 300), (9, 33, 20001), (20, 130, 700), (40, 8200, 300), (48, 100, 384), (64, 40, 5000), (130, 140, 500), (300, 300, 2100),
         (200, 129, 128)]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("codes", [(0, 0), (1, 0), (0, 1), (1, 1)])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_largest_codes_at_the_largest_scales(A, m, n, k, codes, out):
    """One block in two at 2^113 to 2^120, the others at 1; the other operand's scale brings every product to 2^20 of the codes'."""
    rng = np.random.default_rng(m + n + k)
    blocks = -(-k // 128)
    e = np.where(np.arange(blocks) % 2 == 0, rng.integers(113, 121, size=blocks), 0)[:, None]
    far_a, far_b = np.tile(e, (1, m)), np.tile(e, (1, n))
    ones_a, ones_b = (rng.integers(-1, 2, size=(rows, k)).astype(np.float64) for rows in (m, n))
    for a, ea, b in ((large(rng, m, k, codes[0]), far_a, ones_b), (ones_a, 20 - far_a, large(rng, n, k, codes[1]))):
        eb = np.tile(20 - ea[:, :1], (1, n))
        y = product(A, a, ea, b, eb, out, codes)
        assert torch_mod().equal(y.cpu(), rounded(a @ b.T * 2.0 ** 20, out))


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("codes", [(0, 0), (1, 1)])
@pytest.mark.parametrize("m,n", [(3, 40), (50, 70), (150, 200)])
def test_rows_at_both_ends(A, m, n, codes, out):
    """Rows of both operands at 2^120 and at 2^-100 in turn: finite where they meet each other, next to nothing where both are small, and
    not finite where the result is beyond float32 (there a part of the sum may have passed the other infinity, so any that is not finite
    will do, and where the terms alone are, anything)."""
    torch = torch_mod()
    rng = np.random.default_rng(m)
    a, b = large(rng, m, 128, codes[0]), rng.integers(-1, 2, size=(n, 128)).astype(np.float64)
    ea = np.where(np.arange(m) % 2 == 0, 120, -100)[None]
    eb = np.where(np.arange(n) % 2 == 0, 120, -100)[None]
    want, terms = (v @ w.T * 2.0 ** (ea.T + eb) for v, w in ((a, b), (np.abs(a), np.abs(b))))
    y, ref = product(A, a, ea, b, eb, out, codes).cpu(), rounded(want, out)
    beyond, near = (torch.from_numpy(mask) for mask in (terms >= 2.0 ** 128, terms > 2.0 ** -126))
    mid = near & ~beyond
    assert mid.any() and torch.equal(y[mid], ref[mid])
    assert torch.all(y[~near].abs() <= 2.0 ** -126)
    assert not torch.isfinite(y[beyond & torch.isinf(ref)]).any()


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m", [2, 33, 140])
def test_largest_floats_quantized_and_multiplied(A, m, out):
    """What the quantizer makes of values next to the largest float32: E4M3 codes of 256 at 2^120, against a weight of 2^-90."""
    torch = torch_mod()
    x = torch.full((m, 256), torch.finfo(torch.float32).max, device="cuda")
    x[:, 1::2] = 0
    w = torch.full((70, 256), 2.0 ** -90, device="cuda")
    a, sa, _, _ = A.accept_block_quantize(A.make_block_desc(m, 256), x)
    b, sb, _, _ = A.accept_block_quantize(A.make_block_desc(70, 256, group=128), w)
    assert int(sa.view(torch.uint8).max()) == 247
    y = A.accept_block_matmul(A.make_matmul_desc(m, 70, 256, out_dtype=A.F32 if out == "f32" else A.BF16), a, sa, b, sb)
    assert torch.all(y == 128 * 2.0 ** (128 - 90))


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m", [2, 33, 140])
def test_a_far_row_leaves_the_others_as_they_were(A, m, out):
    """A row beyond float32 by itself, whatever form its results then take, changes no bit of another row's."""
    rng = np.random.default_rng(m)
    k, n = 428, 60
    a, ea = orc.quantize(rng.standard_normal((m, k)), 1, 0)
    b, eb = orc.quantize(rng.standard_normal((n, k)), 1, 0)
    before = product(A, a, ea, b, eb, out, (0, 0))
    a[1, 128:256], ea[1, 1], eb[1] = 448.0, 120, -100
    alone = product(A, a[1:2], ea[:, 1:2], b, eb, out, (0, 0))
    a[1, 128:256], ea[1, 1] = 0.0, 0
    without = product(A, a, ea, b, eb, out, (0, 0))
    a[1, 128:256], ea[1, 1] = 448.0, 120
    y = product(A, a, ea, b, eb, out, (0, 0))
    torch = torch_mod()
    others = torch.arange(m, device="cuda") != 1
    assert torch.isfinite(y).all() and not torch.equal(before[others], y[others])      # (eb is another one now)
    assert torch.equal(y[others], without[others])
    v, w = a[1:2] * orc.spread(ea[:, 1:2], 1, k, 1), b * orc.spread(eb, n, k, 1)
    bound = (k * 2.0 ** -24 + (2.0 ** -10 if out == "bf16" else 0)) * (np.abs(v) @ np.abs(w).T)
    want = v @ w.T
    bound = bound + (2.0 ** -8 if out == "bf16" else 2.0 ** -24) * (np.abs(want) + bound)
    for got in (y[1:2], alone):
        assert np.all(np.abs(got.double().cpu().numpy() - want) <= bound)
