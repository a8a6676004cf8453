"""What the attention operators refuse, their sizes, and what a cache's table means: host code, no GPU."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import attention_oracle as orc

V = ctypes.c_void_p
INVALID, UNSUPPORTED = 1, 2
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_05827_amd", "csrc")


@pytest.fixture(scope="module")
def A():
    import paper_2311_05827_amd as pkg
    return pkg


@pytest.fixture(scope="module")
def lib(A):
    return A.attention_binding.lib


def test_descriptor_layouts(A):
    assert ctypes.sizeof(A.RotateDesc) == 64 and A.RotateDesc.sequences.offset == 32
    assert ctypes.sizeof(A.AttentionDesc) == 112 and A.AttentionDesc.sequences.offset == 24 and A.AttentionDesc.scale.offset == 104
    assert ctypes.sizeof(A.CacheDesc) == 120 and A.CacheDesc.sequences.offset == 40 and A.CacheDesc.scale.offset == 112


def test_pages_on_the_host(tmp_path):
    """The kernels' own rule for places, pages and rows, compiled for the host, against the oracle's."""
    source = tmp_path / "pages.cpp"
    source.write_text('''
#include <cstdio>
#include <initializer_list>
#include "pages.hpp"
int main() {
  for (int shift : {4, 6, 10}) for (int count : {0, 3, 1 << 20}) for (int wide : {0, 2, 5}) {
    const accept::Pages p{count, wide, shift, 3};
    for (long long j : {-1LL, 0LL, 15LL, 16LL, 31LL, 1023LL, 1024LL, 5119LL, 5120LL, (1LL << 31) + 5})
      for (int page : {-2147483647 - 1, -1, 0, 2, 3, (1 << 20) - 1, 1 << 20, 2147483647})
        std::printf("%d %d %d %lld %d %d %lld\\n", shift, count, wide, j, page, int(accept::has_place(p, j) && accept::is_page(p, page)),
                    (long long)accept::cache_row(p, page, j, 2));
  }
}
''')
    program = tmp_path / "pages"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(source), "-o", str(program)], check=True)
    lines = subprocess.run([str(program)], check=True, capture_output=True, text=True).stdout.splitlines()
    assert len(lines) == 3 * 3 * 3 * 10 * 8
    for line in lines:
        shift, count, wide, j, page, there, row = map(int, line.split())
        size = 1 << shift
        p, at = orc.place([page] * wide, size, j)
        exists = p >= 0 and p < count and j // size < wide
        assert there == exists
        if exists:
            assert row == (page * 3 + 2) * size + at and 0 <= row < count * 3 * size


def test_places_up_to_the_last_that_32_bits_hold(tmp_path):
    """The kernels' own arithmetic of places, compiled for the host with every overflow an error: tables of up to 2^31 - 16 places."""
    source = tmp_path / "places.cpp"
    source.write_text('''
#include <cstdio>
#include <initializer_list>
#include "pages.hpp"
int main() {
  for (int keys : {1, 15, 16, 31, 32, 33, 2147483520, 2147483521, 2147483584, 2147483631, 2147483632})
    for (int unit : {32, 64, 128}) {
      const int units = int((keys + 0LL + unit - 1) / unit);
      for (int unit1 : {1, units > 1 ? units - 1 : 1, units})
        for (int some : {0, keys - 1, keys}) std::printf("end %d %d %d %d\\n", unit1, unit, some, accept::units_end(unit1, unit, some));
      for (int by : {0, 1, 15, 16, 31}) for (int key0 : {0, (units - 1) * unit, (keys - 1) / 32 * 32}) std::printf("at %d %d %d %d\\n", key0, by, keys, accept::place_at(key0, by, keys));
    }
}
''')
    program = tmp_path / "places"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC, str(source), "-o", str(program)],
                   check=True)
    lines = subprocess.run([str(program)], check=True, capture_output=True, text=True).stdout.splitlines()
    assert len(lines) == 11 * 3 * (9 + 15)
    for line in lines:
        what, (a, b, c, got) = line.split()[0], map(int, line.split()[1:])
        assert got == (min(a * b, c) if what == "end" else min(a + b, c - 1)), line


BAD_ROTATE = [dict(tokens=-1), dict(heads=0), dict(heads=65536), dict(head_size=0), dict(head_size=12), dict(head_size=264), dict(rotated=-2),
              dict(rotated=3), dict(rotated=66), dict(dtype=2), dict(pairs=2), dict(inverse=2), dict(rest=3), dict(sequences=-1),
              dict(x_stride=120), dict(x_stride=130), dict(y_stride=126), dict(x_stride=(1 << 22) + 8), dict(tokens=1 << 31),
              dict(tokens=1 << 30, x_stride=1 << 20), dict(sequences=7)]


@pytest.mark.parametrize("bad", BAD_ROTATE)
def test_rotate_refuses(A, lib, bad):
    d = A.make_rotate_desc(**{"tokens": 5, "heads": 2, "head_size": 64, **bad})
    at = V(0x1000)
    assert lib.accept_rotate(ctypes.byref(d), at, at, None, None, at, None) == INVALID


def test_rotate_refuses_pointers(A, lib):
    d = A.make_rotate_desc(5, 2, 64)
    at = V(0x1000)
    for args in ((None, at, None, None, at), (at, None, None, None, at), (at, at, None, None, None), (V(0x1008), at, None, None, at),
                 (at, V(0x1002), None, None, at), (at, at, V(0x1002), None, at), (at, at, None, V(0x1002), at), (at, at, None, None, V(0x1004))):
        assert lib.accept_rotate(ctypes.byref(d), *args, None) == INVALID
    assert lib.accept_rotate(None, at, at, None, None, at, None) == INVALID
    d.y_stride = 256   # in place with another stride
    assert lib.accept_rotate(ctypes.byref(d), at, at, None, None, at, None) == INVALID
    d.reserved, d.y_stride = 1, 0
    assert lib.accept_rotate(ctypes.byref(d), at, at, None, None, V(0x9000), None) == INVALID


BAD_ATTENTION = [dict(q_tokens=-1), dict(k_tokens=-1), dict(heads=3), dict(kv_heads=0), dict(heads=1), dict(head_size=20), dict(head_size=512),
                 dict(dtype=5), dict(causal=2), dict(rest=2), dict(sequences=-2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                 dict(scale=float("inf")), dict(q_stride=4), dict(q_stride=258), dict(k_stride=100), dict(v_stride=124), dict(o_stride=255),
                 dict(dq_stride=8), dict(dk_stride=129), dict(dv_stride=(1 << 22) + 8), dict(q_tokens=1 << 31)]


@pytest.mark.parametrize("bad", BAD_ATTENTION)
def test_attention_refuses(A, lib, bad):
    d = A.make_attention_desc(**{"q_tokens": 6, "k_tokens": 6, "heads": 4, "kv_heads": 2, "head_size": 64, **bad})
    n, at = ctypes.c_size_t(7), V(0x1000)
    for size in (lib.accept_attention_workspace_size, lib.accept_attention_backward_workspace_size):
        assert size(ctypes.byref(d), ctypes.byref(n)) == INVALID and n.value == 7
    assert lib.accept_attention(ctypes.byref(d), at, at, at, None, None, at, at, at, None) == INVALID
    assert lib.accept_attention_backward(ctypes.byref(d), at, at, at, at, at, at, None, None, at, at, at, at, None) == INVALID
    with pytest.raises(A.AcceptError):
        A.accept_attention_workspace_size(d)


def test_attention_refuses_pointers(A, lib):
    d = A.make_attention_desc(6, 6, 4, 2, 64)
    at = V(0x1000)
    good = [at, at, at, None, None, at, at, at]   # q, k, v, offsets, o, lse, workspace
    for i, v in ((0, None), (1, None), (2, None), (5, None), (0, V(0x1008)), (1, V(0x1004)), (2, V(0x1008)), (3, V(0x1002)), (4, V(0x1001)),
                 (5, V(0x1008)), (6, V(0x1002))):
        args = list(good)
        args[i] = v
        assert lib.accept_attention(ctypes.byref(d), *args, None) == INVALID, i
    good = [at] * 6 + [None, None] + [at] * 4     # do, q, k, v, o, lse, offsets, dq, dk, dv, workspace
    for i, v in [(i, None) for i in (0, 1, 2, 3, 4, 5, 8, 9, 10, 11)] + [(i, V(0x1008)) for i in (0, 1, 2, 3, 4, 8, 9, 10, 11)] + [(5, V(0x1002))]:
        args = list(good)
        args[i] = v
        assert lib.accept_attention_backward(ctypes.byref(d), *args, None) == INVALID, i
    assert lib.accept_attention(None, *[at] * 8, None) == INVALID
    uneven = A.make_attention_desc(6, 6, 4, 2, 64, sequences=4)
    assert lib.accept_attention(ctypes.byref(uneven), at, at, at, None, None, at, at, at, None) == INVALID
    assert lib.accept_attention(ctypes.byref(uneven), at, at, at, at, None, at, at, at, None) == INVALID
    huge = A.make_attention_desc((1 << 31) - 1, 6, 64, 1, 8)
    assert lib.accept_attention(ctypes.byref(huge), at, at, at, None, None, at, at, at, None) == UNSUPPORTED


BAD_CACHE = [dict(tokens=-1), dict(sequences=-1), dict(heads=3), dict(kv_heads=0), dict(head_size=4), dict(page_size=8), dict(page_size=48),
             dict(page_size=1 << 17), dict(pages=-1), dict(table_pages=-1), dict(table_pages=1 << 27), dict(pages=1 << 31), dict(rotated=5),
             dict(rotated=128), dict(pairs=2), dict(tree_words=-1), dict(tree_words=65), dict(scale=0.0), dict(rest=2), dict(dtype=2),
             dict(q_stride=8), dict(k_stride=130), dict(v_stride=1), dict(o_stride=100), dict(qo_stride=1 << 23), dict(pages=1 << 30)]


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_cache_refuses(A, lib, bad):
    d = A.make_cache_desc(**{"tokens": 6, "sequences": 3, "heads": 4, "kv_heads": 2, "head_size": 64, "page_size": 16, "pages": 10,
                             "table_pages": 4, **bad})
    n, at = ctypes.c_size_t(7), V(0x1000)
    assert lib.accept_cache_workspace_size(ctypes.byref(d), ctypes.byref(n)) == INVALID and n.value == 7
    assert lib.accept_cache_append(ctypes.byref(d), *[at] * 11, None) == INVALID
    assert lib.accept_cache_attention(ctypes.byref(d), *[at] * 9, None) == INVALID


def test_cache_refuses_pointers(A, lib):
    d = A.make_cache_desc(6, 3, 4, 2, 64, 16, 10, 4, rotated=64)
    at = V(0x1000)
    good = [at] * 4 + [None, at, None, at, V(0x9000), at, at]  # q, k, v, frequencies, offsets, lengths, positions, table, qo, caches
    for i, v in [(i, None) for i in (0, 1, 2, 3, 5, 7, 8, 9, 10)] + [(i, V(0x1008)) for i in (0, 1, 2, 8, 9, 10)] + [(i, V(0x1002)) for i in (3, 4, 5, 6, 7)]:
        args = list(good)
        args[i] = v
        assert lib.accept_cache_append(ctypes.byref(d), *args, None) == INVALID, (i, v)
    d.qo_stride = 512   # in place with another stride
    assert lib.accept_cache_append(ctypes.byref(d), *[at] * 4, None, at, None, at, at, at, at, None) == INVALID
    d = A.make_cache_desc(6, 3, 4, 2, 64, 16, 10, 4, tree_words=1)
    good = [at] * 3 + [None] + [at] * 5                        # q, caches, offsets, lengths, table, tree, o, workspace
    for i, v in [(i, None) for i in (0, 1, 2, 4, 5, 6, 7, 8)] + [(i, V(0x1008)) for i in (0, 1, 2, 7, 8)] + [(6, V(0x1004)), (4, V(0x1002))]:
        args = list(good)
        args[i] = v
        assert lib.accept_cache_attention(ctypes.byref(d), *args, None) == INVALID, (i, v)
    d.sequences = 4
    assert lib.accept_cache_attention(ctypes.byref(d), *good, None) == INVALID
    d.sequences, d.reserved = 3, 1
    assert lib.accept_cache_attention(ctypes.byref(d), *good, None) == INVALID


def test_nothing_to_do_is_done(A, lib):
    """No tokens: no pointer is needed, and nothing is launched (there is no GPU here)."""
    assert lib.accept_rotate(ctypes.byref(A.make_rotate_desc(0, 2, 64)), *[None] * 6) == 0
    assert lib.accept_attention(ctypes.byref(A.make_attention_desc(0, 6, 4, 2, 64)), *[None] * 9) == 0
    assert lib.accept_attention_backward(ctypes.byref(A.make_attention_desc(0, 0, 4, 2, 64)), *[None] * 13) == 0
    d = A.make_cache_desc(0, 0, 4, 2, 64, 16, 10, 4)
    assert lib.accept_cache_append(ctypes.byref(d), *[None] * 12) == 0 and lib.accept_cache_attention(ctypes.byref(d), *[None] * 10) == 0


def test_workspaces_are_bounded(A):
    """The cache's does not grow with contexts or tokens, the backward pass's is some floats a query and head."""
    for heads, kv in ((1, 1), (32, 8), (128, 128)):
        small = A.accept_cache_workspace_size(A.make_cache_desc(1, 1, heads, kv, 128, 16, 10, 4))
        large = A.accept_cache_workspace_size(A.make_cache_desc(4096, 64, heads, kv, 128, 16, 1 << 20, 1 << 16))
        assert small <= large <= 1 << 26
    d = A.make_attention_desc(5000, 5000, 32, 8, 128)
    assert 4 * 5000 * 32 <= A.accept_attention_backward_workspace_size(d) <= 1 << 28


def test_tensors_on_the_host_are_refused(A):
    import torch
    x, f = torch.zeros(6, 2, 64), torch.zeros(32)
    i, t = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32)
    cache = torch.zeros(2, 2, 16, 64)
    ad, cd, rd = A.make_attention_desc(6, 6, 2, 2, 64), A.make_cache_desc(6, 1, 2, 2, 64, 16, 2, 1), A.make_rotate_desc(6, 2, 64)
    lse = torch.zeros(2, 6)
    for call in (lambda: A.accept_rotate(rd, x, f), lambda: A.accept_rotate(ad, x, f), lambda: A.accept_attention(ad, x, x, x),
                 lambda: A.accept_attention(rd, x, x, x), lambda: A.accept_attention_backward(ad, x, x, x, x, x, lse), lambda: A.accept_attention(ad, None, x, x),
                 lambda: A.accept_cache_append(cd, x, x, x, cache, cache, t, i), lambda: A.accept_cache_attention(cd, x, cache, cache, t, i),
                 lambda: A.accept_cache_attention(ad, x, cache, cache, t, i)):
        with pytest.raises(A.AcceptError) as err:
            call()
        assert err.value.status == INVALID


@pytest.mark.parametrize("scale", [2.0 ** -101, 1e-300, 2.0 ** 101, 1e300])
def test_scales_that_float32_does_not_carry(A, lib, scale):
    n = ctypes.c_size_t(7)
    a, c = A.make_attention_desc(6, 6, 4, 2, 64, scale=scale), A.make_cache_desc(6, 3, 4, 2, 64, 16, 10, 4, scale=scale)
    assert lib.accept_attention_workspace_size(ctypes.byref(a), ctypes.byref(n)) == INVALID
    assert lib.accept_cache_workspace_size(ctypes.byref(c), ctypes.byref(n)) == INVALID and n.value == 7
    a.scale, c.scale = 2.0 ** -100, 2.0 ** 100
    assert lib.accept_attention_workspace_size(ctypes.byref(a), ctypes.byref(n)) == 0
    assert lib.accept_cache_workspace_size(ctypes.byref(c), ctypes.byref(n)) == 0


def test_shapes_that_a_stage_refuses(A):
    """Each of these would otherwise be taken for something else: a head for a token, a batch for another one."""
    import torch
    x = torch.zeros
    f = x(32)
    for bad in (lambda: A.stage.rotate(x(6, 64), f), lambda: A.stage.rotate(x(1, 2, 3, 2, 64), f),
                lambda: A.stage.attention(x(6, 64), x(6, 64), x(6, 64)),
                lambda: A.stage.attention(x(2, 6, 2, 64), x(4, 6, 2, 64), x(4, 6, 2, 64)),
                lambda: A.stage.attention(x(2, 6, 2, 64), x(12, 2, 64), x(12, 2, 64)),
                lambda: A.stage.attention(x(2, 6, 2, 64), x(2, 6, 2, 64), x(3, 4, 2, 64)),
                lambda: A.stage.Cache(4, 16, 2, 64, device="cpu", dtype=torch.float32).step(x(2, 2, 2, 64), x(2, 2, 2, 64), x(2, 2, 2, 64)),
                lambda: A.stage.Cache(2, 16, 2, 64, device="cpu", dtype=torch.float32).step(x(2, 2, 2, 64), x(4, 2, 64), x(4, 2, 64))):
        with pytest.raises(ValueError):
            bad()


def test_frequencies_have_no_gradients(A):
    import torch
    x, f = torch.zeros(6, 2, 64, requires_grad=True), torch.zeros(32, requires_grad=True)
    with pytest.raises(ValueError, match="gradients"):
        A.stage.rotate(x, f)
    with torch.no_grad(), pytest.raises(A.AcceptError):   # (they are on the host)
        A.stage.rotate(x, f)


def test_a_cache_has_no_gradients(A):
    """A step whose tensors ask for gradients is refused, as a block with a cache is: what it returned would have none."""
    import torch
    cache, x, f = A.stage.Cache(1, 16, 2, 64, device="cpu", dtype=torch.float32), torch.zeros(3, 2, 64), torch.zeros(32)
    for i in range(4):
        ask = [t.clone().requires_grad_(True) if j == i else t for j, t in enumerate((x, x, x, f))]
        with pytest.raises(ValueError, match="gradients"):
            cache.step(*ask[:3], frequencies=ask[3])
        with torch.no_grad(), pytest.raises(A.AcceptError):   # (these tensors are on the host)
            cache.step(*ask[:3], frequencies=ask[3])


def test_frequencies_stay_float32(A):
    """Casting a block casts its weights; the frequencies keep their type and every bit, there and back."""
    import torch
    layer = A.stage.SelfAttention(64, 2, 1, 32, device="cpu")
    want = layer.frequencies.clone()
    assert want.dtype == torch.float32 and want.numel() == 16
    for cast in (lambda m: m.bfloat16(), lambda m: m.float(), lambda m: m.half(), lambda m: m.to(torch.float64), lambda m: m.to("cpu", torch.bfloat16)):
        assert cast(layer) is layer and layer.frequencies.dtype == torch.float32 and torch.equal(layer.frequencies, want)
    assert layer.out.weight.dtype == torch.bfloat16 and "frequencies" in dict(layer.named_buffers()) and "frequencies" not in layer.state_dict()
    away = A.stage.SelfAttention(64, 2, 1, 32, device="meta")
    assert away.frequencies.is_meta and torch.equal(away.to_empty(device="cpu").frequencies, want)
    layer.frequencies = want / 8    # somebody's own
    assert torch.equal(layer.float().frequencies, want / 8)


def test_oracle_against_sums_by_hand():
    """Three keys, two queries, one channel."""
    q, k, v = np.array([[1.0], [2.0]]), np.array([[0.5], [-1.0], [3.0]]), np.array([[1.0], [10.0], [100.0]])
    o, lse, _ = orc.attention(q, k, v, orc.causal(2, 3), 1.0)
    e = np.exp
    assert np.allclose(o[0, 0], (e(0.5) + 10 * e(-1.0)) / (e(0.5) + e(-1.0))) and np.allclose(lse[0], np.log(e(0.5) + e(-1.0)))
    assert np.allclose(o[1, 0], (e(1.0) + 10 * e(-2.0) + 100 * e(6.0)) / (e(1.0) + e(-2.0) + e(6.0)))
    o, lse, _ = orc.attention(q, k[:1], v[:1], orc.causal(2, 1), 1.0)
    assert o[0, 0] == 0 and lse[0] == -np.inf and o[1, 0] == 1.0
    x = np.array([[[1.0, 0.0, 5.0, 7.0]]])
    assert np.allclose(orc.rotate(x, np.array([1]), np.array([np.pi / 2]), True), [[[0, 1, 5, 7]]])
    assert np.allclose(orc.rotate(x, np.array([1]), np.array([np.pi / 2, 0.0]), False), [[[-5, 0, 1, 7]]])


def test_oracle_where_all_scores_are_minus_infinity():
    """Such a score has no weight beside another, and no weight of its own: exp(-inf - -inf)."""
    q, k, v = np.array([[1.0], [2.0]]), np.array([[-np.inf], [2.0]]), np.array([[1.0], [10.0]])
    seen = orc.causal(2, 2)
    o, lse, p = orc.attention(q, k, v, seen, 1.0)
    assert np.isnan(o[0, 0]) and lse[0] == -np.inf and np.isnan(p[0, 0]) and p[0, 1] == 0 and o[1, 0] == 10.0 and lse[1] == 4.0
    _, dk, dv, p, ds = orc.gradients(np.ones((2, 1)), q, k, v, o, lse, seen, 1.0)
    assert np.isnan(dk[0, 0]) and np.isnan(dv[0, 0]) and np.isnan(ds[0, 0]) and ds[0, 1] == 0 and dk[1, 0] == 0 and dv[1, 0] == 1
