"""Sizes with more workgroups than one launch takes in a dimension (2^32 threads; 65535 in the others): the calls take them, and what lies
behind the border is right.  Values are chosen so that every result is exact and can be compared on the GPU."""
import pytest

from stage_util import torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    yield pkg
    torch.cuda.empty_cache()


def parts(length, each=1 << 25):
    return [slice(i, min(i + each, length)) for i in range(0, length, each)]


def few_bits(shape, dtype, seed):
    """Values of four significant bits, 8 .. 15 times 2^-3 .. 2^4, either sign: codes of E4M3 that hold them exactly, alone in a block."""
    torch = torch_mod()
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.empty(shape, dtype=dtype, device="cuda")
    flat = v.view(-1)
    for p in parts(flat.numel()):
        n = p.stop - p.start
        r = torch.randint(0, 128, (n,), generator=g, device="cuda", dtype=torch.int32)
        flat[p] = ((8 + (r & 7)).float() * torch.exp2(((r >> 3) & 7).float() - 3) * (1 - 2 * (r >> 6)).float()).to(dtype)
    return v


@pytest.mark.parametrize("rows,dtype", [((1 << 27) + 3, "f32"), ((1 << 28) + 5, "bf16")])
def test_quantize_many_rows(A, rows, dtype):
    torch = torch_mod()
    torch.cuda.empty_cache()
    x = few_bits((rows, 1), torch.float32 if dtype == "f32" else torch.bfloat16, 1)
    d = A.make_block_desc(rows, 1, in_dtype=A.F32 if dtype == "f32" else A.BF16)
    codes, scales, _, _ = A.accept_block_quantize(d, x)
    for p in parts(rows):
        assert torch.equal(codes[p, 0].float() * scales[0, p].float(), x[p, 0].float())


@pytest.mark.parametrize("group", [1, 128])
@pytest.mark.parametrize("along_rows", [True, False])
def test_quantize_many_squares(A, along_rows, group):
    """A row, and a column, of 2^31 - 1 values (a scale for each, along the row, takes the other kernel)."""
    torch = torch_mod()
    torch.cuda.empty_cache()
    length = (1 << 31) - 1
    x = torch.empty(length, dtype=torch.bfloat16, device="cuda")
    unit = few_bits((128,), torch.bfloat16, 2)
    unit[0] = 240.0
    blocks = -(-length // 128)
    x[:length // 128 * 128].view(-1, 128).copy_(unit.expand(length // 128, 128))
    x[length // 128 * 128:] = unit[:length % 128]
    x[::1 << 20] = 120.0                              # here and there another largest value
    rows, cols = (1, length) if along_rows else (length, 1)
    d = A.make_block_desc(rows, cols, group=group, in_dtype=A.BF16)
    got = A.accept_block_quantize(d, x.view(rows, cols), rowwise=along_rows, colwise=not along_rows)
    codes, scales = got[:2] if along_rows else got[2:]
    assert codes.shape == (1, length) and scales.shape == (blocks, 1)
    for p in parts(blocks, 1 << 18):
        c = slice(p.start * 128, min(p.stop * 128, length))
        each = scales[p, 0].float().repeat_interleave(128)[:c.stop - c.start]
        assert torch.equal(codes[0, c].float() * each, x[c].float())


def test_gradients_of_many_columns(A):
    """One row: dweight is dy * h and dbias dy, each a single product."""
    torch = torch_mod()
    torch.cuda.empty_cache()
    cols = (1 << 28) + 100
    x, dy = torch.randn(1, cols, device="cuda"), torch.randn(1, cols, device="cuda")
    stats = torch.tensor([[0.25], [1.5]], device="cuda")
    _, dweight, dbias = A.accept_layer_norm_backward(A.make_norm_desc(1, cols), dy, x, None, stats)
    assert torch.equal(dbias, dy[0])
    for p in parts(cols):
        assert torch.equal(dweight[p], dy[0, p] * ((x[0, p] - 0.25) * 1.5))


@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_product_with_many_columns(A, out):
    """Codes of -1, 0 and 1, a scale of its own for each 128 columns."""
    torch = torch_mod()
    torch.cuda.empty_cache()
    n, k = (1 << 27) + 77, 16
    f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    a = torch.tensor([[1.0, -1, 0, 1, 1, -1, 1, 0, 1, 1, -1, 1, 0, 1, -1, 1]], device="cuda")
    table = torch.tensor([0x38, 0xB8, 0, 0x38], dtype=torch.uint8, device="cuda")       # 1, -1, 0, 1
    b = torch.empty(n, k, dtype=torch.uint8, device="cuda")
    for p in parts(n):
        b[p] = table[torch.randint(0, 4, (p.stop - p.start, k), device="cuda")]
    b = b.view(f8)
    blocks = -(-n // 128)
    sb = torch.randint(125, 130, (1, blocks), device="cuda").to(torch.uint8)
    sa = torch.full((1, 1), 127, dtype=torch.uint8, device="cuda").view(e8)
    d = A.make_matmul_desc(1, n, k, out_dtype=A.F32 if out == "f32" else A.BF16, a_stride=16, b_stride=16)
    y = A.accept_block_matmul(d, a.to(f8), sa, b, sb.view(e8))
    for p in parts(n):
        scale = torch.exp2(sb[0, p.start // 128:-(-p.stop // 128)].float() - 127).repeat_interleave(128)[:p.stop - p.start]
        assert torch.equal(y[0, p].float(), (b[p].float() * a).sum(1) * scale)


def test_product_with_many_rows_of_the_first_by_long_rows_of_the_second(A):
    """Rows of b further apart than the tiles take: 64 rows of a a workgroup, more than 65535 of these."""
    torch = torch_mod()
    torch.cuda.empty_cache()
    m, n, k, stride = (1 << 22) + 70, 2, 16, (1 << 22) + 16
    f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    table = torch.tensor([0x38, 0xB8, 0, 0x38], dtype=torch.uint8, device="cuda")
    a = table[torch.randint(0, 4, (m, k), device="cuda")].view(f8)
    b = torch.as_strided(torch.empty(stride + k, dtype=f8, device="cuda"), (n, k), (stride, 1))
    b.view(torch.uint8).copy_(table[torch.randint(0, 4, (n, k), device="cuda")])
    sa = torch.randint(125, 130, (1, m), device="cuda").to(torch.uint8)
    sb = torch.full((1, n), 126, dtype=torch.uint8, device="cuda").view(e8)
    d = A.make_matmul_desc(m, n, k, b_group=1, a_stride=16, b_stride=stride)
    y = A.accept_block_matmul(d, a, sa.view(e8), b, sb)
    want = torch.stack([(a.float() * b[j].float()).sum(1) for j in range(n)], 1) * torch.exp2(sa[0].float() - 128)[:, None]
    assert torch.equal(y, want)
