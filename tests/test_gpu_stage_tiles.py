"""Products through the tiles of 128 x 128 and 256 x 256 (and of few rows), at every number of blocks that their loops tell apart.

Exact: codes are -1, 0 and 1 and scales 2^-1 .. 2^1 an operand, so every sum is a multiple of 2^-2 below 2^24 of them: the 8-bit instruction
cuts nothing off, float32 rounds nothing, and a bfloat16 result is the exact sum rounded once.  A dropped or doubled column, a wrong scale
or a result in a wrong place shows.  Random operands: the bound of the products' other tests.
"""
import numpy as np
import pytest

from oracle import stage_oracle as orc
from stage_util import HALF_BF16, U, torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def types():
    torch = torch_mod()
    return torch.float8_e4m3fn, torch.float8_e5m2


def small(rng, rows, k, group, code, stride=0):
    """(codes, scales, float32 values of -1, 0 and 1 times 2^-1 .. 2^1); NaN behind column k."""
    torch = torch_mod()
    v = rng.integers(-1, 2, size=(rows, k), dtype=np.int8).astype(np.float32)
    e = rng.integers(-1, 2, size=(-(-k // 128), -(-rows // group)))
    stride = stride or -(-k // 16) * 16 + 32
    held = torch.empty(rows * stride, dtype=types()[code], device="cuda").view(rows, stride)
    if stride < 1 << 16:
        held.copy_(torch.full((rows, stride), float("nan"), device="cuda").to(held.dtype))
    held[:, :k] = torch.from_numpy(v).cuda().to(held.dtype)
    scales = torch.from_numpy(np.ascontiguousarray(e + 127).astype(np.uint8)).cuda().view(torch.float8_e8m0fnu)
    return held[:, :k], scales, v * orc.spread(e, rows, k, group).astype(np.float32)


def check_exact(A, seed, m, n, k, out, codes=(0, 0), groups=(1, 128), y_pad=0, a_stride=0):
    torch = torch_mod()
    rng = np.random.default_rng(seed)
    a, sa, va = small(rng, m, k, groups[0], codes[0], a_stride)
    b, sb, vb = small(rng, n, k, groups[1], codes[1])
    d = A.make_matmul_desc(m, n, k, out_dtype=A.F32 if out == "f32" else A.BF16, a_code=codes[0], b_code=codes[1], a_group=groups[0],
                           b_group=groups[1], a_stride=a.stride(0), b_stride=b.stride(0), y_stride=n + y_pad if y_pad else 0)
    held = torch.full((m, n + y_pad), 7.0, dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    y = A.accept_block_matmul(d, a, sa, b, sb, y=held[:, :n])
    want = torch.from_numpy(va) @ torch.from_numpy(vb).t()      # exact in float32, in any order
    assert torch.equal(y.cpu(), want.to(y.dtype))
    assert torch.all(held[:, n:] == 7)


# one block alone, two, odd and even numbers of whole blocks, each with and without an incomplete one behind
LENGTHS = [128, 256, 384, 512, 640, 768, 1024, 130, 257, 400, 1100, 60, 2048, 2047]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("k", LENGTHS)
@pytest.mark.parametrize("m,n", [(1, 50), (30, 70), (64, 200), (130, 150), (300, 257)])
def test_every_number_of_blocks(A, m, n, k, out):
    check_exact(A, m + k, m, n, k, out, y_pad=k % 3)


@pytest.mark.parametrize("k", LENGTHS)
def test_every_number_of_blocks_in_large_tiles(A, k):
    check_exact(A, k, 3600, 3500, k, "bf16", y_pad=k % 3)


@pytest.mark.parametrize("codes", [(0, 0), (1, 0), (0, 1), (1, 1)])
@pytest.mark.parametrize("groups", [(1, 1), (1, 128), (128, 1), (128, 128)])
def test_types_and_groups_in_large_tiles(A, groups, codes):
    check_exact(A, 5, 3587, 3590, 640, "bf16", codes, groups, y_pad=5)


@pytest.mark.parametrize("k,codes,b_group", [(384, (1, 0), 128), (2304, (1, 1), 1), (1030, (0, 0), 128)])
def test_random_operands_in_large_tiles(A, k, codes, b_group):
    """Bound: k U and 2^-10 of the terms' magnitudes, then bfloat16's rounding."""
    torch = torch_mod()
    rng = np.random.default_rng(k)
    m, n = 3600, 3500
    parts = []
    for rows, group, code in ((m, 1, codes[0]), (n, b_group, codes[1])):
        x = torch.from_numpy(rng.standard_normal((rows, k)).astype(np.float32)).cuda()
        c, s, _, _ = A.accept_block_quantize(A.make_block_desc(rows, k, group=group, code=code), x)
        each = s.float().t().repeat_interleave(group, 0)[:rows].repeat_interleave(128, 1)[:, :k]
        parts.append((c, s, (c.float() * each).cpu().double()))
    (a, sa, va), (b, sb, vb) = parts
    d = A.make_matmul_desc(m, n, k, out_dtype=A.BF16, a_code=codes[0], b_code=codes[1], b_group=b_group)
    y = A.accept_block_matmul(d, a, sa, b, sb).cpu().double()
    want, terms = va @ vb.t(), va.abs() @ vb.abs().t()
    bound = (k * U + 2.0 ** -10) * terms
    assert torch.all((y - want).abs() <= bound + HALF_BF16 * (want.abs() + bound))


@pytest.mark.parametrize("m,n,out", [(1100, 130, "f32"), (1100, 130, "bf16"), (3600, 3500, "bf16")])
def test_tiles_of_rows_beyond_32_bits(A, m, n, out):
    """Rows 2^22 bytes apart, the furthest that the tiles take: the last of them lie beyond 4 GiB."""
    torch_mod().cuda.empty_cache()
    check_exact(A, m, m, n, 300, out, a_stride=1 << 22)
