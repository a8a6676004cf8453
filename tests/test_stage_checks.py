"""What the stage operators refuse, and their sizes: host code, no GPU."""
import ctypes

import pytest

V = ctypes.c_void_p
INVALID = 1


@pytest.fixture(scope="module")
def A():
    import paper_2311_05827_amd as pkg
    return pkg


@pytest.fixture(scope="module")
def lib(A):
    return A.stage_binding.lib


def test_descriptor_layouts(A):
    S = A.stage_binding
    assert ctypes.sizeof(S.NormDesc) == 64 and S.NormDesc.rows.offset == 16 and S.NormDesc.eps.offset == 56
    assert ctypes.sizeof(S.BlockDesc) == 40 and S.BlockDesc.rows.offset == 16
    assert ctypes.sizeof(S.MatmulDesc) == 72 and S.MatmulDesc.m.offset == 24 and S.MatmulDesc.y_stride.offset == 64


def test_block_stride(A):
    assert [A.accept_block_stride(v) for v in (0, 1, 128, 129, 768)] == [0, 128, 128, 256, 768]
    assert A.accept_block_stride(-1) == -1 and A.accept_block_stride((1 << 40) + 1) == -1


BAD_NORM = [dict(rows=-1), dict(cols=0), dict(cols=-3), dict(x_dtype=2), dict(y_dtype=-1), dict(param_dtype=9), dict(code=2),
            dict(x_stride=7), dict(y_stride=1), dict(dx_stride=-8), dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")),
            dict(rows=1 << 31), dict(rows=1 << 30, cols=1 << 30), dict(rows=1 << 30, x_stride=1 << 20)]


@pytest.mark.parametrize("bad", BAD_NORM)
def test_norm_refuses(A, lib, bad):
    d = A.make_norm_desc(**{"rows": 4, "cols": 8, **bad})
    n = ctypes.c_size_t(7)
    p = [V(0x1000)] * 8
    assert lib.accept_norm_workspace_size(ctypes.byref(d), ctypes.byref(n)) == INVALID and n.value == 7
    assert lib.accept_layer_norm(ctypes.byref(d), *p[:5], None) == INVALID
    assert lib.accept_layer_norm_quantize(ctypes.byref(d), *p[:6], None) == INVALID
    assert lib.accept_layer_norm_backward(ctypes.byref(d), *p[:8], None) == INVALID
    with pytest.raises(A.AcceptError):
        A.accept_norm_workspace_size(d)


def test_norm_refuses_pointers(A, lib):
    d = ctypes.byref(A.make_norm_desc(4, 8, y_dtype=A.BF16))
    at, odd = V(0x1000), V(0x1002)
    assert lib.accept_layer_norm(None, at, at, at, at, at, None) == INVALID
    for args in ((None, at, at, at, at), (at, at, at, None, at), (odd, at, at, at, at), (at, odd, at, at, at), (at, at, odd, at, at),
                 (at, at, at, V(0x1001), at), (at, at, at, at, odd)):
        assert lib.accept_layer_norm(d, *args, None) == INVALID
    for args in ((None, at, at, at, at, at), (at, at, at, None, at, at), (at, at, at, at, None, at), (at, at, at, V(0x1004), at, at)):
        assert lib.accept_layer_norm_quantize(d, *args, None) == INVALID
    good = [at] * 8   # dy, x, weight, stats, dx, dweight, dbias, workspace
    for i, v in ((0, None), (1, None), (3, None), (4, None), (7, None), (1, odd), (2, odd), (3, odd), (4, odd), (5, odd), (6, odd),
                 (0, V(0x1001)), (7, V(0x1008))):
        args = list(good)
        args[i] = v
        assert lib.accept_layer_norm_backward(d, *args, None) == INVALID, i


BAD_BLOCK = [dict(rows=-1), dict(cols=-1), dict(group=0), dict(group=64), dict(in_dtype=2), dict(code=-1), dict(x_stride=5),
             dict(rows=1 << 31), dict(rows=1 << 30, cols=1 << 20)]


@pytest.mark.parametrize("bad", BAD_BLOCK)
def test_quantize_refuses(A, lib, bad):
    d = A.make_block_desc(**{"rows": 4, "cols": 8, **bad})
    at = V(0x1000)
    assert lib.accept_block_quantize(ctypes.byref(d), at, at, at, at, at, None) == INVALID


def test_quantize_refuses_pointers(A, lib):
    d = A.make_block_desc(4, 8)
    at = V(0x1000)
    for args in ((None, at, at, at, at), (at, None, None, None, None), (at, at, None, at, at), (at, None, at, at, at), (at, at, at, at, None),
                 (at, at, at, None, at), (V(0x1002), at, at, at, at), (at, V(0x1008), at, at, at), (at, at, at, V(0x1008), at)):
        assert lib.accept_block_quantize(ctypes.byref(d), *args, None) == INVALID
    assert lib.accept_block_quantize(None, at, at, at, at, at, None) == INVALID
    d.reserved = 1
    assert lib.accept_block_quantize(ctypes.byref(d), at, at, at, at, at, None) == INVALID


BAD_MATMUL = [dict(m=-1), dict(n=-1), dict(k=-1), dict(out_dtype=2), dict(a_code=2), dict(b_code=-1), dict(a_group=2), dict(b_group=0),
              dict(a_stride=8), dict(a_stride=40), dict(b_stride=16), dict(b_stride=100), dict(y_stride=3), dict(m=1 << 31),
              dict(n=(1 << 31) - 1), dict(k=1 << 31), dict(m=1 << 21, n=1 << 20), dict(m=1 << 30, a_stride=1 << 11)]


@pytest.mark.parametrize("bad", BAD_MATMUL)
def test_matmul_refuses(A, lib, bad):
    d = A.make_matmul_desc(**{"m": 4, "n": 8, "k": 32, **bad})
    n = ctypes.c_size_t(7)
    at = V(0x1000)
    assert lib.accept_matmul_workspace_size(ctypes.byref(d), ctypes.byref(n)) == INVALID and n.value == 7
    assert lib.accept_block_matmul(ctypes.byref(d), at, at, at, at, at, at, None) == INVALID


def test_matmul_refuses_pointers(A, lib):
    d = A.make_matmul_desc(4, 8, 32)
    at = V(0x1000)
    for i in range(5):
        args = [at] * 6
        args[i] = None
        assert lib.accept_block_matmul(ctypes.byref(d), *args, None) == INVALID, i
    for i, v in ((0, V(0x1008)), (2, V(0x1008)), (4, V(0x1002))):
        args = [at] * 6
        args[i] = v
        assert lib.accept_block_matmul(ctypes.byref(d), *args, None) == INVALID, i
    assert lib.accept_matmul_workspace_size(None, None) == INVALID
    split = A.make_matmul_desc(100, 100, 8192)   # parts of the contracted axis: needs a workspace
    assert A.accept_matmul_workspace_size(split) > 0
    assert lib.accept_block_matmul(ctypes.byref(split), at, at, at, at, at, None, None) == INVALID
    assert lib.accept_block_matmul(ctypes.byref(split), at, at, at, at, at, V(0x1008), None) == INVALID


def test_workspaces_are_small(A):
    for rows, cols in ((0, 1), (1, 1), (16384, 8192), (8144, 768), (100, 100000)):
        b = A.accept_norm_workspace_size(A.make_norm_desc(rows, cols))
        assert b % 256 == 0 and 8 * cols <= b <= 512 * 8 * cols + 256
    for m, n, k in ((1, 4096, 4096), (48, 8192, 2048), (8192, 8192, 8192), (2048, 768, 8144), (0, 5, 5), (5, 5, 0)):
        assert A.accept_matmul_workspace_size(A.make_matmul_desc(m, n, k)) <= 64 * 4 * m * n + 256


def test_tensors_on_the_host_are_refused(A):
    import torch
    x = torch.zeros(4, 8)
    s = torch.zeros(2, 4)
    nd, bd, md = A.make_norm_desc(4, 8), A.make_block_desc(4, 8), A.make_matmul_desc(4, 4, 8)
    c, e = x.to(torch.float8_e4m3fn), torch.zeros(1, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    for call in (lambda: A.accept_layer_norm(nd, x), lambda: A.accept_layer_norm_quantize(nd, x),
                 lambda: A.accept_layer_norm_backward(nd, x, x, None, s), lambda: A.accept_block_quantize(bd, x),
                 lambda: A.accept_block_matmul(md, c, e, c, e), lambda: A.accept_layer_norm(nd, None),
                 lambda: A.accept_layer_norm(bd, x), lambda: A.accept_block_quantize(nd, x), lambda: A.accept_block_matmul(nd, c, e, c, e)):
        with pytest.raises(A.AcceptError) as err:
            call()
        assert err.value.status == INVALID
