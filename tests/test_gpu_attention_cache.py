"""The cache of pages, and attention over it, against the oracle in 64 bits."""
from fractions import Fraction

import numpy as np
import pytest

from attention_util import U, check_forward, ends_of, ints, orc, tokens_of
from stage_util import f64, rounding, torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def words_of(rng, n, words):
    """Trees of n nodes: a token sees itself and what it continues."""
    masks = []
    for j in range(n):
        parent = int(rng.integers(-1, j)) if j else -1
        masks.append((masks[parent] if parent >= 0 else 0) | 1 << j)
    return np.array([[m >> (64 * w) & ((1 << 64) - 1) for w in range(words)] for m in masks], dtype=np.uint64).reshape(n, words)


class Cache:
    """A cache in use: contexts, new tokens, pages in no order, and what is in no token's place NaN."""

    def __init__(self, A, seed, name, contexts, new, heads, kv_heads, head, page, rotated=0, neighbours=False, words=0, scale=None, behind=0,
                 spare=2, pad=0, bad=()):
        rng = np.random.default_rng(seed)
        torch = torch_mod()
        self.A, self.name, self.heads, self.kv, self.head, self.page = A, name, heads, kv_heads, head, page
        self.contexts, self.new, self.ends = contexts, new, ends_of(new)
        self.rotated, self.neighbours, self.words = rotated, neighbours, words
        self.scale = head ** -0.5 if scale is None else scale
        n = self.ends[-1] + behind
        each = [-(-(c + m) // page) for c, m in zip(contexts, new)]
        self.pages, self.width = sum(each) + spare, max(each + [1]) + 1
        free = list(rng.permutation(self.pages))
        self.table = np.full((len(new), self.width), 1 << 30, dtype=np.int64)   # behind the last page: no page, and not read
        for s, m in enumerate(each):
            for i in range(m):
                self.table[s, i] = free.pop()
        for s, i, page_number in bad:
            self.table[s, i] = page_number
        size = (self.pages, kv_heads, page, head)
        k, v = np.full(size, np.nan), np.full(size, np.nan)
        self.keys = [rng.standard_normal((c, kv_heads, head)) for c in contexts]
        self.values = [rng.standard_normal((c, kv_heads, head)) for c in contexts]
        for s, c in enumerate(contexts):
            for j in range(c):
                p, at = orc.place(self.table[s], page, j)
                if 0 <= p < self.pages:
                    k[p, :, at], v[p, :, at] = self.keys[s][j], self.values[s][j]
        dtype = torch.float32 if name == "f32" else torch.bfloat16
        self.k_cache, self.v_cache = torch.tensor(k, dtype=dtype, device="cuda"), torch.tensor(v, dtype=dtype, device="cuda")
        self.q, self.xq = tokens_of(rng.standard_normal((n, heads, head)), name, pad)
        self.k, self.xk = tokens_of(rng.standard_normal((n, kv_heads, head)), name, pad)
        self.v, self.xv = tokens_of(rng.standard_normal((n, kv_heads, head)), name, pad)
        self.offsets, self.lengths, self.table_dev = ints(self.ends), ints(contexts), ints(self.table.reshape(-1)).view(self.table.shape)
        self.frequencies = torch.tensor(10000.0 ** (-np.arange(0, rotated, 2) / max(rotated, 1)), dtype=torch.float32, device="cuda") if rotated else None
        self.tree_words = np.concatenate([words_of(rng, m, words) for m in new]) if words else None
        self.tree = torch.tensor(np.concatenate([self.tree_words, np.zeros((behind, words), np.uint64)]).view(np.int64), device="cuda") if words else None
        self.desc = A.make_cache_desc(n, len(new), heads, kv_heads, head, page, self.pages, self.width,
                                      dtype=A.F32 if name == "f32" else A.BF16, rotated=rotated, pairs=int(neighbours), tree_words=words,
                                      scale=scale, q_stride=heads * head + pad, k_stride=kv_heads * head + pad, v_stride=kv_heads * head + pad)

    def append(self, positions=None, **kw):
        return self.A.accept_cache_append(self.desc, self.q, self.k, self.v, self.k_cache, self.v_cache, self.table_dev, self.lengths,
                                          offsets=self.offsets, positions=positions, frequencies=self.frequencies, **kw)

    def attend(self, q=None, **kw):
        desc = self.desc
        if q is not None:
            desc = type(desc).from_buffer_copy(desc)
            desc.q_stride = 0
        self.o = self.A.accept_cache_attention(desc, self.q if q is None else q, self.k_cache, self.v_cache, self.table_dev, self.lengths,
                                               offsets=self.offsets, tree=self.tree, **kw)
        return self.o

    def held(self, s):
        """(keys, values, exists) of a sequence's places as the caches hold them, 64 bits."""
        kc, vc = f64(self.k_cache), f64(self.v_cache)
        n = self.contexts[s] + self.new[s]
        k, v, there = np.zeros((n, self.kv, self.head)), np.zeros((n, self.kv, self.head)), np.zeros(n, dtype=bool)
        for j in range(n):
            p, at = orc.place(self.table[s], self.page, j)
            if 0 <= p < self.pages:
                k[j], v[j], there[j] = kc[p, :, at], vc[p, :, at], True
        return k, v, there

    def check_attention(self, q=None):
        o, xq = f64(self.o), self.xq if q is None else f64(q)
        for s, (a, b) in enumerate(orc.spans(self.ends)):
            if a == b:
                continue
            k, v, there = self.held(s)
            c, n = self.contexts[s], self.new[s]
            seen = orc.tree_seen(self.tree_words[a:b], c, n, c + n) if self.words else orc.causal(n, c + n)
            seen = seen & there[None, :]
            for h in range(self.heads):
                kv = h // (self.heads // self.kv)
                check_forward(self.name, xq[a:b, h], k[:, kv], v[:, kv], seen, self.scale, o[a:b, h], None, "sequence %d head %d" % (s, h))


# contexts, new tokens, heads, key heads, head size, page size
CASES = [
    ([0], [1], 1, 1, 8, 16),
    ([1], [1], 4, 1, 64, 16),
    ([700], [1], 8, 2, 128, 16),
    ([31, 32, 33, 500], [1, 1, 1, 1], 4, 4, 64, 32),
    ([15, 0, 129, 300], [1, 3, 0, 40], 6, 2, 80, 16),
    ([2000, 3], [1, 1], 3, 1, 256, 64),
    ([64, 200], [70, 33], 4, 1, 32, 128),
    ([100] * 70, [1] * 70, 2, 1, 64, 16),
    ([40, 5000], [2, 1], 32, 1, 96, 1024),
]


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("contexts,new,heads,kv_heads,head,page", CASES)
def test_append_and_attend(A, name, contexts, new, heads, kv_heads, head, page):
    torch = torch_mod()
    rotated, neighbours = head // 2 // 2 * 2, head % 16 == 0
    c = Cache(A, 1, name, contexts, new, heads, kv_heads, head, page, rotated, neighbours, pad=16)
    before = [t.clone() for t in (c.k_cache, c.v_cache)]
    q = c.append()
    f = f64(c.frequencies)
    written = torch.zeros(c.k_cache.shape[:1] + c.k_cache.shape[2:3], dtype=torch.bool)
    for s, (a, b) in enumerate(orc.spans(c.ends)):
        position = contexts[s] + np.arange(b - a)
        k, v, there = c.held(s)
        assert there.all()
        for got, x in ((f64(q)[a:b], c.xq[a:b]), (k[contexts[s]:], c.xk[a:b])):
            want = orc.rotate(x, position, f, neighbours)
            assert np.all(np.abs(got - want) <= 8 * U * 2 * np.abs(x).max(initial=0) + rounding(name, np.abs(want) + 1e-5 * U))
        assert np.array_equal(v[contexts[s]:], c.xv[a:b])
        for j in position:
            written[orc.place(c.table[s], page, j)] = True
    for t, old in zip((c.k_cache, c.v_cache), before):   # nothing else was written
        kept = ~written[:, None, :, None].cuda().expand_as(t)
        assert torch.equal(t[kept].nan_to_num(9.0), old[kept].nan_to_num(9.0))
    c.attend(q)
    c.check_attention(q)


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("contexts,new,words,page", [([500, 0, 31], [40, 17, 64], 1, 16), ([100, 33], [100, 128], 2, 64), ([45], [70], 1, 32),
                                                     ([300], [1], 3, 16)])
def test_trees(A, name, contexts, new, words, page):
    """Also one with more nodes than its words have bits: those are seen by nobody."""
    c = Cache(A, 2, name, contexts, new, 4, 2, 64, page, words=words)
    depth = np.concatenate([contexts[s] + np.array([bin(int(w[0])).count("1") for w in c.tree_words[a:b]]) for s, (a, b) in enumerate(orc.spans(c.ends))])
    q = c.append(positions=ints(depth))
    assert np.array_equal(f64(q), c.xq)   # nothing turns
    c.attend()
    c.check_attention()


def test_positions_are_those_given(A):
    c = Cache(A, 3, "f32", [20], [9], 2, 1, 64, 16, rotated=64)
    positions = np.array([5, 5, 7, 1 << 20, 0, 3, 3, 3, 100])
    q = c.append(positions=ints(positions))
    want = orc.rotate(c.xk, positions, f64(c.frequencies), False)
    k, _, _ = c.held(0)
    assert np.all(np.abs(k[20:] - want) <= (8 * 2 + 1) * U * np.abs(c.xk).max())
    assert np.all(np.abs(f64(q) - orc.rotate(c.xq, positions, f64(c.frequencies), False)) <= (8 * 2 + 1) * U * np.abs(c.xq).max())


def test_queries_of_places_beyond_32_bits(A):
    """A sequence of 2^31 - 2 tokens goes on: its new keys have no place, but their queries turn by where they would be."""
    c = Cache(A, 20, "f32", [20], [5], 2, 1, 64, 16, rotated=64)
    before = c.k_cache.clone()
    c.lengths = ints([(1 << 31) - 2])
    q = f64(c.append())
    # what is left of a turn, from whole numbers: 64 bits would lose the last ones that count
    f, positions = f64(c.frequencies), (1 << 31) - 2 + np.arange(5)
    turn = Fraction(15915494309189533576888376337251436203445964574046, 10 ** 50)
    left = np.array([[float(t - round(t)) for t in (int(p) * Fraction(float(x)) * turn for x in f)] for p in positions]) * 2 * np.pi
    a, b = c.xq[..., :32], c.xq[..., 32:]
    cos, sin = np.cos(left)[:, None], np.sin(left)[:, None]
    want, terms = np.concatenate([a * cos - b * sin, a * sin + b * cos], -1), np.concatenate([np.abs(a) + np.abs(b)] * 2, -1)
    assert np.all(np.abs(q - want) <= (4 + 3) * U * terms + U * (np.abs(want) + 7 * U * terms))
    assert np.array_equal(f64(c.k_cache), f64(before), equal_nan=True)


def test_in_place_and_without_queries(A):
    torch = torch_mod()
    c, d, e = (Cache(A, 4, "bf16", [20, 3], [9, 2], 2, 1, 64, 16, rotated=64) for _ in range(3))
    q = c.append()
    d.append(q_out=d.q)
    assert torch.equal(d.q, q)
    d.q = None
    e.q = None
    assert e.append() is None
    assert torch.equal(c.k_cache.nan_to_num(9.0), e.k_cache.nan_to_num(9.0)) and torch.equal(c.v_cache.nan_to_num(9.0), d.v_cache.nan_to_num(9.0))


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 64])
def test_pages_that_do_not_exist(A, name, page):
    """What would go there is dropped, and nobody sees it; a sequence with no page at all has zeros."""
    torch = torch_mod()
    c = Cache(A, 5, name, [300, 0, 90], [3, 2, 1], 4, 1, 64, page, bad=[(0, 1, -1), (0, 300 // page, 1 << 20), (1, 0, -7)])
    rows = [t.clone() for t in (c.k_cache, c.v_cache)]
    c.append()
    c.attend()
    c.check_attention()
    assert torch.all(c.o[3:5] == 0)
    spare = sorted(set(range(c.pages)) - {int(p) for p in c.table.reshape(-1) if 0 <= p < c.pages})
    for t, old in zip((c.k_cache, c.v_cache), rows):
        assert torch.equal(t[spare].nan_to_num(9.0), old[spare].nan_to_num(9.0))


def test_lengths_beyond_the_table(A):
    """A length that the table has no pages for, or a negative one: device data that no host check sees."""
    torch = torch_mod()
    c = Cache(A, 6, "bf16", [100, 20], [1, 1], 2, 1, 64, 16)
    c.lengths = ints([(1 << 31) - 1, -5])
    c.append()
    o = c.attend()
    torch.cuda.synchronize()
    k, v, _ = c.held(1)
    assert np.array_equal(f64(o)[1], np.repeat(v[:1, 0], 2, axis=0)) and np.array_equal(v[0], c.xv[1])   # its first place, alone


def test_no_pages(A):
    torch = torch_mod()
    desc = A.make_cache_desc(3, 3, 2, 1, 64, 16, 0, 0)
    q, k = torch.randn(3, 2, 64, device="cuda"), torch.randn(3, 1, 64, device="cuda")
    empty, table, lengths = torch.empty(0, 1, 16, 64, device="cuda"), torch.empty(3, 0, dtype=torch.int32, device="cuda"), ints([0, 4, 9])
    assert torch.equal(A.accept_cache_append(desc, q, k, k, empty, empty, table, lengths), q)
    assert torch.all(A.accept_cache_attention(desc, q, empty, empty, table, lengths) == 0)


def test_rows_behind_the_last_sequence(A):
    torch = torch_mod()
    c = Cache(A, 7, "bf16", [50, 20], [3, 40], 4, 2, 64, 16, rotated=64, behind=50)
    q = c.append()
    assert torch.all(q[43:] == 0)
    o = c.attend(q).clone()
    assert torch.all(o[43:] == 0)
    given = torch.full_like(o, 7.0)
    c.attend(q, o=given)
    assert torch.all(given[43:] == 7) and torch.equal(given[:43], o[:43])
    again = torch.full_like(q, 7.0)
    c.append(q_out=again)
    assert torch.all(again[43:] == 7) and torch.equal(again[:43], q[:43])
    c.desc.rest = A.REST_ZEROS
    c.attend(q, o=given)
    assert torch.equal(given, o)


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_a_cache_that_holds_nan(A, name):
    """NaN in places that some new tokens see and others do not: only the ones that see it are NaN."""
    c = Cache(A, 8, name, [200], [40], 2, 1, 64, 16)
    c.append()
    p, at = orc.place(c.table[0], 16, 215)
    c.v_cache[p, 0, at, 3] = float("nan")
    o = f64(c.attend())
    assert np.isfinite(o[:15]).all() and np.isnan(o[15:, :, 3]).all() and np.isfinite(np.delete(o, 3, axis=2)).all()
    c.check_attention()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("head", [16, 80, 256])
@pytest.mark.parametrize("new", [9, 40])   # wavefronts with keys of their own, and with keys that they share
def test_a_cache_that_holds_nan_at_every_width(A, name, head, new):
    c = Cache(A, 18, name, [300], [new], 2, 1, head, 16)
    c.append()
    p, at = orc.place(c.table[0], 16, 305)
    c.v_cache[p, 0, at, head - 3] = float("nan")
    o = f64(c.attend())
    assert np.isfinite(o[:5]).all() and np.isnan(o[5:, :, head - 3]).all() and np.isfinite(np.delete(o, head - 3, axis=2)).all()
    c.check_attention()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("head", [16, 80, 128, 256])
@pytest.mark.parametrize("new", [1, 9, 40])   # wavefronts with keys of their own, and with keys that they share
def test_scores_of_minus_infinity(A, name, head, new):
    """Rows that see nothing else are NaN: of a context in one part, and of one in many.  Beside another score those keys are as if they were not there;
    and rows that see no place (there are pages for none) are zeros."""
    contexts = [20, 900, 700, 0]
    c = Cache(A, 21, name, contexts, [new] * 4, 2, 1, head, 16, bad=[(3, i, -1) for i in range(-(-new // 16))])
    c.q[:, :, 0], c.xq[:, :, 0] = 1.0, 1.0
    c.k[:2 * new, :, 0], c.xk[:2 * new, :, 0] = -float("inf"), -np.inf
    for s, many in ((0, 20), (1, 900), (2, 600)):
        for j in range(many):
            p, at = orc.place(c.table[s], 16, j)
            c.k_cache[p, :, at, 0] = -float("inf")
    c.append()
    o = f64(c.attend())
    assert np.isnan(o[:2 * new]).all() and np.isfinite(o[2 * new:]).all() and np.all(o[3 * new:] == 0)
    k, v, _ = c.held(2)
    seen = orc.causal(new, 700 + new)[:, 600:]
    for h in range(2):
        check_forward(name, c.xq[2 * new:3 * new, h], k[600:, 0], v[600:, 0], seen, c.scale, o[2 * new:3 * new, h])


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_scores_that_are_not_finite(A, name, new, bad):
    """A context's key whose score is NaN or plus infinity, in one of many parts and in the only one; the third sequence has none."""
    c = Cache(A, 22, name, [900, 20, 300], [new] * 3, 2, 1, 64, 16)
    c.q[:, :, 0], c.xq[:, :, 0] = 1.0, 1.0
    for s, j in ((0, 400), (1, 3)):
        p, at = orc.place(c.table[s], 16, j)
        c.k_cache[p, :, at, 0] = bad
    c.append()
    o = f64(c.attend())
    assert np.isnan(o[:2 * new]).all() and np.isfinite(o[2 * new:]).all()
    k, v, _ = c.held(2)
    for h in range(2):
        check_forward(name, c.xq[2 * new:, h], k[:, 0], v[:, 0], orc.causal(new, 300 + new), c.scale, o[2 * new:, h])


def test_steps_of_a_server(A):
    """A prompt, then token after token: the same attention as over the whole sequence at once, to the bounds of both (the cache holds the
    same bfloat16 keys, so the scores agree; weights and results are rounded in two orders)."""
    torch = torch_mod()
    n, prompt, heads, kv, head, page = 75, 50, 4, 2, 64, 16
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(n, heads + 2 * kv, head, device="cuda", generator=g).bfloat16()
    f = torch.tensor(10000.0 ** (-np.arange(0, head, 2) / head), dtype=torch.float32, device="cuda")
    turned = A.accept_rotate(A.make_rotate_desc(n, heads + kv, head, dtype=A.BF16, x_stride=(heads + 2 * kv) * head), x[:, :heads + kv], f)
    desc = A.make_attention_desc(n, n, heads, kv, head, dtype=A.BF16, q_stride=(heads + kv) * head, k_stride=(heads + kv) * head,
                                 v_stride=(heads + 2 * kv) * head)
    want, _ = A.accept_attention(desc, turned[:, :heads], turned[:, heads:], x[:, heads + kv:])
    pages = -(-n // page)
    k_cache = torch.full((pages, kv, page, head), float("nan"), dtype=torch.bfloat16, device="cuda")
    v_cache = k_cache.clone()
    table, lengths = torch.randperm(pages, device="cuda", generator=g).int().view(1, -1), ints([0])
    got = []
    stride = (heads + 2 * kv) * head
    for at, to in [(0, prompt)] + [(i, i + 1) for i in range(prompt, n)]:
        d = A.make_cache_desc(to - at, 1, heads, kv, head, page, pages, pages, dtype=A.BF16, rotated=head, q_stride=stride, k_stride=stride,
                              v_stride=stride, qo_stride=stride)
        piece = x[at:to].clone()
        q = A.accept_cache_append(d, piece[:, :heads], piece[:, heads:heads + kv], piece[:, heads + kv:], k_cache, v_cache, table, lengths,
                                  frequencies=f, q_out=piece[:, :heads])
        got.append(A.accept_cache_attention(d, q, k_cache, v_cache, table, lengths))
        lengths += to - at
    got = torch.cat(got)
    tokens = torch.arange(n, device="cuda")
    flat = k_cache[table[0].long()].transpose(1, 2).reshape(-1, kv, head)[:n]
    assert torch.equal(flat, turned[:, heads:])   # bit for bit: the same rotation
    seen = orc.causal(n, n)
    for h in range(heads):
        q64, k64, v64 = f64(turned[:, h]), f64(turned[:, heads + h // 2]), f64(x[:, heads + kv + h // 2])
        check_forward("bf16", q64, k64, v64, seen, head ** -0.5, f64(got[:, h]))
        check_forward("bf16", q64, k64, v64, seen, head ** -0.5, f64(want[:, h]))


def test_a_long_cache(A):
    """Rows of the caches beyond 2^31 elements, and a long context in many parts."""
    torch = torch_mod()
    heads, kv, head, page, context = 4, 1, 128, 64, 40000
    each = -(-(context + 1) // page)
    pages = (1 << 31) // (kv * page * head) + each + 5
    k_cache = torch.zeros(pages, kv, page, head, dtype=torch.bfloat16, device="cuda")
    v_cache = torch.zeros_like(k_cache)
    g = torch.Generator(device="cuda").manual_seed(10)
    where = torch.arange(pages - each, pages, device="cuda")
    k_cache[where] = torch.randn(each, kv, page, head, device="cuda", generator=g).bfloat16()
    v_cache[where] = torch.randn(each, kv, page, head, device="cuda", generator=g).bfloat16()
    q, k, v = (torch.randn(1, h, head, device="cuda", generator=g).bfloat16() for h in (heads, kv, kv))
    desc = A.make_cache_desc(1, 1, heads, kv, head, page, pages, each, dtype=A.BF16)
    table, lengths = where.int().view(1, -1), ints([context])
    A.accept_cache_append(desc, None, k, v, k_cache, v_cache, table, lengths)
    o = f64(A.accept_cache_attention(desc, q, k_cache, v_cache, table, lengths))
    k64 = f64(k_cache[where].reshape(-1, head)[:context + 1])
    v64 = f64(v_cache[where].reshape(-1, head)[:context + 1])
    assert np.array_equal(k64[-1], f64(k)[0, 0])
    for h in range(heads):
        check_forward("bf16", f64(q)[:, h], k64, v64, np.ones((1, context + 1), bool), head ** -0.5, o[:, h])


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 40])   # wavefronts with keys of their own, and with keys that they share
def test_a_context_as_long_as_a_table_can_be(A, name, new):
    """2^31 - 64 places, all but the last page's the same page of zeros, whose weights are e^-80 of the others': the last tokens are among what is
    seen.  (2^31 e^-60 is below 2^-55: what the zeros add is far inside the bounds.)"""
    torch = torch_mod()
    head, page, width = 8, 64, (1 << 25) - 1
    assert A.make_cache_desc(new, 1, 1, 1, head, page, 2, width).table_pages * page == (1 << 31) - 64
    g = torch.Generator(device="cuda").manual_seed(19)
    dtype = torch.float32 if name == "f32" else torch.bfloat16
    k_cache = torch.zeros(2, 1, page, head, dtype=dtype, device="cuda")
    v_cache = torch.ones_like(k_cache)
    k_cache[1] = 10 + torch.randn(1, page, head, device="cuda", generator=g)
    v_cache[1] = 5 + torch.randn(1, page, head, device="cuda", generator=g)
    q, k, v = (torch.randn(new, 1, head, device="cuda", generator=g) for _ in range(3))
    q, k, v = (1 + 0.1 * q).to(dtype), (10 + k).to(dtype), v.to(dtype)
    table = torch.zeros(1, width, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    lengths = ints([width * page - new])
    desc = A.make_cache_desc(new, 1, 1, 1, head, page, 2, width, dtype=A.F32 if name == "f32" else A.BF16, scale=1.0)
    A.accept_cache_append(desc, None, k, v, k_cache, v_cache, table, lengths)
    o = A.accept_cache_attention(desc, q, k_cache, v_cache, table, lengths)
    assert torch.equal(k_cache[1, 0, -new:], k[:, 0]) and torch.equal(v_cache[1, 0, -new:], v[:, 0])
    check_forward(name, f64(q)[:, 0], f64(k_cache)[1, 0], f64(v_cache)[1, 0], orc.causal(new, page), 1.0, f64(o)[:, 0])


def test_captured_steps_that_share_a_workspace(A):
    """A graph of one step's append and attention, replayed while lengths and inputs change in place, beside a second graph with the same
    workspace: every replay is what the eager calls give."""
    torch = torch_mod()
    a, b = (Cache(A, s, "bf16", [300, 41, 0], [1, 1, 1], 8, 2, 64, 16, rotated=64, spare=40) for s in (11, 12))
    for c in (a, b):
        c.table_dev = torch.arange(3 * c.width, device="cuda", dtype=torch.int32).view(3, c.width).contiguous() % c.pages
    ws = torch.empty(A.accept_cache_workspace_size(a.desc), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for c in (a, b):
        c.k_cache.nan_to_num_(0.5), c.v_cache.nan_to_num_(0.25)
        c.attend(c.append(), workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(c.attend(c.append(), workspace=ws))
        graphs.append(graph)
    for turn in range(4):
        for c in (a, b):
            c.lengths += 1
            c.k.normal_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for c, got in zip((a, b), outs):
            got = got.clone()
            assert torch.equal(c.attend(c.append()), got), turn


def test_the_same_call_gives_the_same_bits(A):
    torch = torch_mod()
    c = Cache(A, 13, "bf16", [3000, 10, 777], [1, 5, 33], 8, 2, 128, 32)
    c.append()
    first = c.attend().clone()
    assert all(torch.equal(c.attend(), first) for _ in range(4))


def test_refusals(A):
    torch = torch_mod()
    c = Cache(A, 14, "bf16", [20], [4], 2, 1, 64, 16, rotated=64)
    call = lambda **kw: A.accept_cache_attention(c.desc, **{**dict(q=c.q, k_cache=c.k_cache, v_cache=c.v_cache, table=c.table_dev,
                                                                    lengths=c.lengths, offsets=c.offsets), **kw})
    for kw in (dict(q=c.q[:3]), dict(k_cache=c.k_cache[:1]), dict(v_cache=c.v_cache.transpose(1, 2)), dict(table=c.table_dev.long()),
               dict(table=c.table_dev[:, :1]), dict(lengths=ints([1, 2])), dict(offsets=ints([0])), dict(tree=torch.zeros(4, 1, dtype=torch.int64, device="cuda")),
               dict(q=c.q.float()), dict(k_cache=c.k_cache.float()), dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(A.AcceptError):
            call(**kw)
    with pytest.raises(A.AcceptError):
        c.frequencies = None
        c.append()
