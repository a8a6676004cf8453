"""Rotation by position against the oracle in 64 bits."""
import numpy as np
import pytest

from attention_util import ends_of, ints, orc, tokens_of
from stage_util import U, f64, rounding, torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def frequencies(rotated, base=10000.0):
    torch = torch_mod()
    f = (base ** (-np.arange(0, rotated, 2) / max(rotated, 1))).astype(np.float32)
    return torch.tensor(f, device="cuda"), f.astype(np.float64)


def check(name, got, x, positions, f, neighbours, inverse):
    """cos and sin are off by at most 4 U (the part of a turn that is left, rounded, times pi: pi U; the functions: a step of 2 U), the two
    products and their sum by 3 U of |a| + |b| more, and the result is rounded."""
    want = orc.rotate(x, positions, f, neighbours, inverse)
    terms = orc.rotate(np.abs(x), np.zeros(len(x)), f, neighbours)
    half = len(f)
    if neighbours:
        both = np.repeat(terms[..., 0:2 * half:2] + terms[..., 1:2 * half:2], 2, axis=-1)
    else:
        both = np.concatenate([terms[..., :half] + terms[..., half:2 * half]] * 2, axis=-1)
    bound = np.zeros_like(x)
    bound[..., :2 * half] = (5 + 3) * U * both
    bound[..., :2 * half] += rounding(name, np.abs(want[..., :2 * half]) + bound[..., :2 * half])
    assert np.all(np.abs(got - want) <= bound)


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("tokens,heads,head,rotated", [(1, 1, 8, 8), (1, 40, 128, 128), (37, 3, 64, 32), (300, 5, 96, 20), (9, 2, 256, 254),
                                                       (130, 2, 40, 0), (1000, 7, 80, 80), (5, 6, 72, 2)])
def test_sizes(A, name, neighbours, tokens, heads, head, rotated):
    torch = torch_mod()
    rng = np.random.default_rng(1)
    x, values = tokens_of(rng.standard_normal((tokens, heads, head)), name)
    f, f64s = frequencies(rotated)
    for inverse in (False, True):
        d = A.make_rotate_desc(tokens, heads, head, rotated, dtype=A.F32 if name == "f32" else A.BF16, pairs=int(neighbours), inverse=inverse)
        y = A.accept_rotate(d, x, f if rotated else None)
        check(name, f64(y), values, np.arange(tokens), f64s, neighbours, inverse)
        place = x.clone()
        assert A.accept_rotate(d, place, f, y=place) is place and torch.equal(place, y)


@pytest.mark.parametrize("neighbours", [False, True])
def test_far_positions(A, neighbours):
    """Positions up to 2^31 - 1: the angle is what 64 bits make of position and frequency (2^31 * 2^-52 is still 2 U)."""
    torch = torch_mod()
    rng = np.random.default_rng(2)
    positions = np.concatenate([rng.integers(0, 1 << 31, 60), [(1 << 31) - 1, 1 << 24, (1 << 24) + 1, 0]])
    x, values = tokens_of(rng.standard_normal((len(positions), 2, 64)), "f32", pad=12)
    f, f64s = frequencies(64)
    d = A.make_rotate_desc(len(positions), 2, 64, dtype=A.F32, pairs=int(neighbours), x_stride=2 * 64 + 12, sequences=5)
    y = A.accept_rotate(d, x, f, positions=ints(positions))
    check("f32", f64(y), values, positions, f64s, neighbours, False)


@pytest.mark.parametrize("times", [1.0, 300.0, 1e6])
def test_far_angles(A, times):
    """The farthest positions, with frequencies from `times` / 2 to `times`: as near as near ones.  The oracle's angles come from whole numbers, by
    1 / (2 pi) with 80 digits: 64 bits would lose the last ones that count."""
    torch = torch_mod()
    from fractions import Fraction
    turn = Fraction(15915494309189533576888376337251436203445964574046, 10 ** 50)   # 1 / (2 pi)
    rng = np.random.default_rng(5)
    n, pairs = 64, 32
    positions = (1 << 31) - 1 - rng.integers(0, 1 << 20, n)
    f = (times * (1 + np.arange(pairs)) / (2 * pairs) + times / 2).astype(np.float32)
    left = np.empty((n, pairs))
    for i, p in enumerate(positions):
        for j, freq in enumerate(f):
            turns = int(p) * Fraction(float(freq)) * turn
            left[i, j] = float(turns - round(turns)) * 2 * np.pi
    x, values = tokens_of(rng.standard_normal((n, 2, 2 * pairs)), "f32")
    y = A.accept_rotate(A.make_rotate_desc(n, 2, 2 * pairs, dtype=A.F32), x, torch.tensor(f, device="cuda"), positions=ints(positions))
    a, b = values[..., :pairs], values[..., pairs:]
    c, s = np.cos(left)[:, None], np.sin(left)[:, None]
    want, terms = np.concatenate([a * c - b * s, a * s + b * c], -1), np.concatenate([np.abs(a) + np.abs(b)] * 2, -1)
    bound = (4 + 3) * U * terms      # (see check)
    assert np.all(np.abs(f64(y) - want) <= bound + rounding("f32", np.abs(want) + bound))


@pytest.mark.parametrize("given", [False, True])
def test_sequences_and_the_tokens_behind_them(A, given):
    torch = torch_mod()
    rng = np.random.default_rng(3)
    lengths = [5, 0, 70, 1, 0] + [3] * 90
    ends = ends_of(lengths)
    n = ends[-1] + 11
    x, values = tokens_of(rng.standard_normal((n, 3, 32)), "f32")
    f, f64s = frequencies(16)
    places = np.concatenate([np.arange(m) for m in lengths])
    positions = rng.integers(0, 5000, n) if given else None
    kw = dict(offsets=ints(ends), positions=ints(positions) if given else None)
    d = A.make_rotate_desc(n, 3, 32, 16, dtype=A.F32, sequences=len(lengths))
    y = torch.full_like(x, 7.0)
    A.accept_rotate(d, x, f, y=y, **kw)
    check("f32", f64(y)[:ends[-1]], values[:ends[-1]], positions[:ends[-1]] if given else places, f64s, False, False)
    assert torch.all(y[ends[-1]:] == 7)
    made = A.accept_rotate(d, x, f, **kw)
    assert torch.equal(made[:ends[-1]], y[:ends[-1]]) and torch.all(made[ends[-1]:] == 0)
    each = A.accept_rotate(A.make_rotate_desc(12, 3, 32, 16, dtype=A.F32, sequences=3), x[:12], f)
    check("f32", f64(each), values[:12], np.arange(12) % 4, f64s, False, False)


def test_the_way_back(A):
    """By the angle and by its negative: the value again, to twice the bound of one way."""
    torch = torch_mod()
    x = torch.randn(200, 4, 64, device="cuda")
    f, _ = frequencies(64)
    there = A.accept_rotate(A.make_rotate_desc(200, 4, 64), x, f)
    back = A.accept_rotate(A.make_rotate_desc(200, 4, 64, inverse=True), there, f)
    assert float((back - x).abs().max()) <= 2 * (2 * 8 + 1) * U * float(x.abs().max()) * 2


def test_what_does_not_turn_is_copied(A):
    """NaN payloads aside, the bits."""
    torch = torch_mod()
    x = torch.randn(30, 2, 64, device="cuda").bfloat16()
    x[3, 1, 40] = float("inf")
    f, _ = frequencies(16)
    y = A.accept_rotate(A.make_rotate_desc(30, 2, 64, 16, dtype=A.BF16), x, f)
    assert torch.equal(y[..., 16:], x[..., 16:])


def test_refusals(A):
    torch = torch_mod()
    x = torch.randn(6, 2, 64, device="cuda")
    f, _ = frequencies(64)
    d = A.make_rotate_desc(6, 2, 64)
    for call in (lambda: A.accept_rotate(d, x.bfloat16(), f), lambda: A.accept_rotate(d, x[:5], f), lambda: A.accept_rotate(d, x, f[:31]),
                 lambda: A.accept_rotate(d, x, None), lambda: A.accept_rotate(d, x, f, positions=ints(range(5))),
                 lambda: A.accept_rotate(A.make_rotate_desc(6, 2, 64, sequences=4), x, f), lambda: A.accept_rotate(d, x, f, offsets=ints([0, 3, 6])),
                 lambda: A.accept_rotate(d, x, f.cpu())):
        with pytest.raises(A.AcceptError):
            call()
