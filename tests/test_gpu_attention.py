"""Attention over sequences and its gradients against the oracle in 64 bits."""
import numpy as np
import pytest

from attention_util import check_forward, check_gradients, ends_of, ints, orc, tokens_of
from stage_util import f64, torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def code(A, name):
    return A.F32 if name == "f32" else A.BF16


class Case:
    """Inputs of sequences, on the device and in 64 bits, and one call's outputs."""

    def __init__(self, A, seed, name, q_lengths, k_lengths, heads, kv_heads, head, causal=True, scale=None, pad=0, behind=0, packed=True,
                 size=1.0, change=None):
        rng = np.random.default_rng(seed)
        self.A, self.name, self.heads, self.kv_heads, self.head, self.causal = A, name, heads, kv_heads, head, causal
        self.q_ends, self.k_ends = ends_of(q_lengths), ends_of(k_lengths)
        self.nq, self.nk, self.behind = self.q_ends[-1] + behind, self.k_ends[-1] + behind, behind
        self.scale = head ** -0.5 if scale is None else scale
        values = {"q": size * rng.standard_normal((self.nq, heads, head)), "k": size * rng.standard_normal((self.nk, kv_heads, head)),
                  "v": rng.standard_normal((self.nk, kv_heads, head)), "do": rng.standard_normal((self.nq, heads, head))}
        if change:
            change(values)
        self.pad = pad
        self.t, self.x = {}, {}
        for what, v in values.items():
            self.t[what], self.x[what] = tokens_of(v, name, 0 if what == "do" else pad)
        self.q_off, self.k_off = (ints(self.q_ends), ints(self.k_ends)) if packed else (None, None)
        whole, kv_whole = heads * head + pad, kv_heads * head + pad
        self.desc = A.make_attention_desc(self.nq, self.nk, heads, kv_heads, head, sequences=len(q_lengths), dtype=code(A, name),
                                          causal=causal, scale=scale, q_stride=whole, k_stride=kv_whole, v_stride=kv_whole)

    def forward(self, **kw):
        self.o, self.lse = self.A.accept_attention(self.desc, self.t["q"], self.t["k"], self.t["v"], self.q_off, self.k_off, **kw)
        return self.o, self.lse

    def backward(self, **kw):
        return self.A.accept_attention_backward(self.desc, self.t["do"], self.t["q"], self.t["k"], self.t["v"], self.o, self.lse,
                                                self.q_off, self.k_off, **kw)

    def seen(self, s):
        rows, keys = self.q_ends[s + 1] - self.q_ends[s], self.k_ends[s + 1] - self.k_ends[s]
        return orc.causal(rows, keys) if self.causal else np.ones((rows, keys), dtype=bool)

    def pieces(self):
        for s, ((a, b), (c, d)) in enumerate(zip(orc.spans(self.q_ends), orc.spans(self.k_ends))):
            yield s, slice(a, b), slice(c, d)

    def check_forward(self):
        o, lse = f64(self.o), f64(self.lse)
        for s, rows, keys in self.pieces():
            for h in range(self.heads):
                kv = h // (self.heads // self.kv_heads)
                check_forward(self.name, self.x["q"][rows, h], self.x["k"][keys, kv], self.x["v"][keys, kv], self.seen(s), self.scale,
                              o[rows, h], lse[h, rows], "sequence %d head %d" % (s, h))

    def check_backward(self, grads):
        dq, dk, dv = (f64(g) for g in grads)
        o, lse = f64(self.o), f64(self.lse)
        group = self.heads // self.kv_heads
        for s, rows, keys in self.pieces():
            for kv in range(self.kv_heads):
                hs = range(kv * group, kv * group + group)
                heads = [(self.x["do"][rows, h], self.x["q"][rows, h], self.x["k"][keys, kv], self.x["v"][keys, kv], o[rows, h], lse[h, rows])
                         for h in hs]
                check_gradients(self.name, heads, self.scale, self.seen(s), ([dq[rows, h] for h in hs], dk[keys, kv], dv[keys, kv]),
                                "sequence %d key head %d" % (s, kv))


# lengths of queries and keys, heads, key heads, head size
SIZES = [
    ([1], [1], 1, 1, 8),
    ([1], [300], 2, 1, 64),
    ([33], [33], 2, 2, 64),
    ([130], [130], 3, 1, 128),
    ([257], [257], 2, 1, 80),
    ([70], [200], 2, 2, 96),
    ([200], [70], 2, 1, 64),        # the first 130 queries see nothing
    ([64, 0, 1, 128, 31], [64, 0, 1, 128, 31], 4, 2, 32),
    ([5, 300, 129], [70, 300, 0], 2, 1, 128),
    ([100, 40], [100, 90], 2, 1, 256),
    ([200], [200], 1, 1, 248),
    ([65] * 70, [65] * 70, 1, 1, 40),  # more sequences than lanes
]


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("q_lengths,k_lengths,heads,kv_heads,head", SIZES)
def test_both_passes(A, name, causal, q_lengths, k_lengths, heads, kv_heads, head):
    c = Case(A, 1, name, q_lengths, k_lengths, heads, kv_heads, head, causal)
    c.forward()
    c.check_forward()
    c.check_backward(c.backward())


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("sequences", [65, 600, 5000])
def test_many_short_sequences(A, name, sequences):
    """More than a workgroup looks at: a few longer than its rows among them, empty ones, and tokens behind the last."""
    lengths = [0 if s % 11 == 0 else 260 if s % 400 == 33 else 129 if s % 300 == 64 else 1 + s * s % 7 for s in range(sequences)]
    keys = [n + 3 * (s % 2) if s % 13 else 0 for s, n in enumerate(lengths)]
    c = Case(A, 26, name, lengths, keys, 2, 1, 16, behind=150)
    o, lse = c.forward()
    grads = c.backward()
    c.check_forward()
    c.check_backward(grads)
    for t, n in ((o, c.q_ends[-1]), (grads[0], c.q_ends[-1]), (grads[1], c.k_ends[-1]), (grads[2], c.k_ends[-1])):
        assert n + 150 == t.shape[0] and (t[n:] == 0).all()
    assert (lse[:, c.q_ends[-1]:] == -np.inf).all()


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_equal_sequences_without_offsets(A, name):
    c = Case(A, 2, name, [45] * 3, [45] * 3, 4, 2, 64, packed=False)
    c.forward()
    c.check_forward()
    c.check_backward(c.backward())


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_strides_and_a_scale(A, name):
    c = Case(A, 3, name, [50, 83], [50, 83], 4, 2, 64, scale=0.3, pad=24)
    c.forward()
    c.check_forward()
    c.check_backward(c.backward())


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_queries_keys_and_values_side_by_side(A, name):
    """Views of one product's result, and their gradients into one buffer of the same form."""
    torch = torch_mod()
    rng = np.random.default_rng(4)
    heads, kv, head, n = 4, 2, 32, 150
    both, xs = tokens_of(rng.standard_normal((n, heads + 2 * kv, head)), name)
    do, xdo = tokens_of(rng.standard_normal((n, heads, head)), name)
    stride = (heads + 2 * kv) * head
    desc = A.make_attention_desc(n, n, heads, kv, head, dtype=code(A, name), q_stride=stride, k_stride=stride, v_stride=stride,
                                 dq_stride=stride, dk_stride=stride, dv_stride=stride)
    q, k, v = both[:, :heads], both[:, heads:heads + kv], both[:, heads + kv:]
    o, lse = A.accept_attention(desc, q, k, v)
    d = torch.full_like(both, float("nan"))
    dq, dk, dv = A.accept_attention_backward(desc, do, q, k, v, o, lse, dq=d[:, :heads], dk=d[:, heads:heads + kv], dv=d[:, heads + kv:])
    assert torch.isfinite(d).all() and dq.data_ptr() == d.data_ptr()
    apart = A.accept_attention(A.make_attention_desc(n, n, heads, kv, head, dtype=code(A, name)), q.contiguous(), k.contiguous(), v.contiguous())
    assert torch.equal(o, apart[0]) and torch.equal(lse, apart[1])
    again = A.accept_attention_backward(A.make_attention_desc(n, n, heads, kv, head, dtype=code(A, name)), do, q.contiguous(),
                                        k.contiguous(), v.contiguous(), o, lse)
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), again))


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_scores_of_hundreds(A, name):
    """Scores up to several hundred: weights are one, or nothing, and no sum overflows."""
    c = Case(A, 5, name, [150], [150], 2, 1, 64, size=7.0)
    c.forward()
    c.check_forward()
    c.check_backward(c.backward())


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_scores_that_grow_along_the_keys(A, name):
    """Every tile has a new maximum: by little (results stay relative to an old one) and by much."""
    def rise(values):
        n = values["k"].shape[0]
        values["k"][:] = np.linspace(0, 1, n)[:, None, None] ** 3 * np.abs(values["k"])
        values["q"][:] = np.abs(values["q"])
    c = Case(A, 6, name, [40], [700], 2, 1, 64, size=1.5, change=rise)
    c.forward()
    c.check_forward()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("causal", [True, False])
def test_what_is_not_seen_has_no_effect(A, name, bad, causal):
    """Keys and values that only some rows see, and queries and gradients that only some keys are seen by, are not finite; so are the
    tokens of the next sequence and those behind the last one."""
    def spoil(values):
        for what in ("k", "v", "q", "do"):
            values[what][140:, :, 3] = bad if what != "k" else np.nan   # another sequence, and behind it
        values["v"][100, 0, 5] = bad      # rows before the 100th do not see it
        values["do"][20, 0, 7] = bad      # keys behind the 20th are not seen by it
    c = Case(A, 7, name, [140, 30], [140, 30], 2, 1, 64, causal, behind=9, change=spoil)
    c.forward()
    grads = c.backward()
    o, lse = f64(c.o), f64(c.lse)
    rows = slice(0, 140)
    seen = c.seen(0)
    for h in range(2):
        check_forward(name, c.x["q"][rows, h], c.x["k"][rows, 0], c.x["v"][rows, 0], seen, c.scale, o[rows, h], lse[h, rows])
    # What the formula makes finite is, and within its bounds.  (The rows that see value 100 have sums of do * o that are not finite, and
    # with them everything that the keys they see get from them.)
    heads = [(c.x["do"][rows, h], c.x["q"][rows, h], c.x["k"][rows, 0], c.x["v"][rows, 0], o[rows, h], lse[h, rows]) for h in range(2)]
    dq, dk, dv = (f64(g)[rows] for g in grads)
    check_gradients(name, heads, c.scale, seen, ([dq[:, h] for h in range(2)], dk[:, 0], dv[:, 0]), kinds=False)
    assert not np.isfinite(dv[:21, 0, 7]).any()
    if causal:
        assert np.isfinite(o[:100]).all() and not np.isfinite(o[100:140, :, 5]).any()
        assert np.isfinite(dv[21:, 0]).all() and np.isfinite(np.delete(dq[:100], 20, axis=0)).all()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("head", [16, 80, 128, 256])
def test_what_is_not_seen_at_every_width(A, name, head):
    """NaN in one value that a causal row's later keys hold, and in one row's do: results that the formula makes finite are, within their bounds."""
    def spoil(values):
        values["v"][100, 0, head - 3] = np.nan
        values["do"][20, 0, head - 1] = np.nan
    c = Case(A, 17, name, [140], [140], 2, 1, head, True, change=spoil)
    c.forward()
    grads = c.backward()
    o, lse, seen = f64(c.o), f64(c.lse), c.seen(0)
    for h in range(2):
        check_forward(name, c.x["q"][:, h], c.x["k"][:, 0], c.x["v"][:, 0], seen, c.scale, o[:, h], lse[h])
    heads = [(c.x["do"][:, h], c.x["q"][:, h], c.x["k"][:, 0], c.x["v"][:, 0], o[:, h], lse[h]) for h in range(2)]
    dq, dk, dv = (f64(g) for g in grads)
    check_gradients(name, heads, c.scale, seen, ([dq[:, h] for h in range(2)], dk[:, 0], dv[:, 0]), kinds=False)
    assert np.isfinite(o[:100]).all() and np.isfinite(np.delete(o, head - 3, axis=2)).all() and not np.isfinite(o[100:, :, head - 3]).any()
    assert np.isfinite(dv[21:, 0]).all() and np.isfinite(np.delete(dq[:100], 20, axis=0)).all()


SPOILED = {"v": (300, 5), "k": (200, 2), "q": (150, 1), "do": (250, 7)}


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("head", [16, 64, 80, 128, 256])
@pytest.mark.parametrize("what", ["v", "k", "q", "do"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_one_value_in_the_middle_of_many(A, name, head, what, bad):
    """Rows and keys next to the one that holds it have tiles that they see all of, before and behind: what does not see it is within its bounds."""
    token, value = SPOILED[what]

    def spoil(values):
        values[what][token, -1, value] = bad
    c = Case(A, 22, name, [401, 70], [401, 70], 4, 2, head, change=spoil)
    c.forward()
    o, lse = f64(c.o), f64(c.lse)
    dq, dk, dv = (f64(g) for g in c.backward())
    with np.errstate(invalid="ignore"):
        for s, rows, keys in c.pieces():
            for kv in range(2):
                heads = [(c.x["do"][rows, h], c.x["q"][rows, h], c.x["k"][keys, kv], c.x["v"][keys, kv], o[rows, h], lse[h, rows]) for h in (2 * kv, 2 * kv + 1)]
                if what != "k" or kv == 0 or s:   # (scores of infinity: see below)
                    for h, (_, q, k, v, *_) in zip((2 * kv, 2 * kv + 1), heads):
                        check = slice(0, rows.stop - rows.start) if what != "q" or h != 3 or s else slice(0, token)
                        check_forward(name, q[check], k, v, c.seen(s)[check], c.scale, o[rows, h][check], lse[h, rows][check], "sequence %d head %d" % (s, h))
                check_gradients(name, heads, c.scale, c.seen(s), ([dq[rows, 2 * kv], dq[rows, 2 * kv + 1]], dk[keys, kv], dv[keys, kv]),
                                "sequence %d key head %d" % (s, kv), kinds=False)
    if what == "v":
        assert np.isfinite(np.delete(o, value, axis=2)).all() and np.isfinite(o[:token]).all() and not np.isfinite(o[token:401, 2:, value]).any()
    if what == "k":
        assert np.isfinite(o[:token]).all() and np.isfinite(dq[:token]).all()
    if what == "q":
        assert np.isfinite(np.delete(o, token, axis=0)).all() and np.isfinite(dv[token + 1:]).all() and np.isfinite(dk[token + 1:]).all()
    if what == "do":
        assert np.isfinite(np.delete(dq, token, axis=0)).all() and np.isfinite(dv[token + 1:]).all() and np.isfinite(dk[token + 1:]).all()


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_the_last_value_of_rows_that_see_all(A, name):
    """Its row stands in for the rest of the last tile, where it has weight zero: infinities stay infinities."""
    def spoil(values):
        values["v"][129, 0, 5], values["do"][149, 0, 7] = np.inf, -np.inf
    c = Case(A, 23, name, [150], [130], 1, 1, 64, False, change=spoil)
    c.forward()
    c.check_forward()
    o = f64(c.o)
    assert np.all(o[:, 0, 5] == np.inf)
    c.t["v"][129, 0, 5], c.x["v"][129, 0, 5] = 1.0, 1.0
    c.forward()
    dv = f64(c.backward()[2])
    assert np.all(dv[:, 0, 7] == -np.inf) and np.isfinite(np.delete(dv, 7, axis=2)).all()


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_one_value_at_the_start_of_many(A, name):
    """Thousands of rows see it: they are NaN in that value, at no more than a look at their last tiles."""
    def spoil(values):
        values["v"][0, 0, 3], values["do"][6000, 0, 9] = np.nan, np.nan
    c = Case(A, 24, name, [6001], [6001], 1, 1, 64, change=spoil)
    o = f64(c.forward()[0])
    assert np.isnan(o[:, 0, 3]).all() and np.isfinite(np.delete(o, 3, axis=2)).all()
    dv = f64(c.backward()[2])
    assert np.isnan(dv[:, 0, 9]).all() and np.isfinite(np.delete(dv, 9, axis=2)).all()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("head", [16, 64, 128, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_scores_of_minus_infinity(A, name, head, causal):
    """A sequence's first 70 keys have no score but minus infinity.  Rows that see nothing else are NaN, and so is what keys get from them; for the
    others it is as if those keys were not there.  Rows that see no key are zeros beside them."""
    def spoil(values):
        values["q"][:, :, 0] = 1.0
        values["k"][:70, :, 0] = -np.inf
        values["k"][150:180, :, 0] = -np.inf    # all of the second sequence
    c = Case(A, 21, name, [150, 30, 40], [150, 30, 20], 2, 1, head, causal, change=spoil)
    c.forward()
    o, lse = f64(c.o), f64(c.lse)
    grads = [f64(g) for g in c.backward()]
    for s, rows, keys in c.pieces():
        seen = c.seen(s)
        for h in range(2):
            q, k, v = c.x["q"][rows, h], c.x["k"][keys, 0], c.x["v"][keys, 0]
            with np.errstate(invalid="ignore"):
                check_forward(name, q, k, v, seen, c.scale, o[rows, h], lse[h, rows], "sequence %d head %d" % (s, h))
            if s == 0:   # to the bounds of the keys that count
                behind = slice(70, 150) if causal else slice(0, 150)
                check_forward(name, q[behind], k[70:], v[70:], seen[behind, 70:], c.scale, o[behind, h], lse[h, behind], "head %d" % h)
        heads = [(c.x["do"][rows, h], c.x["q"][rows, h], c.x["k"][keys, 0], c.x["v"][keys, 0], o[rows, h], lse[h, rows]) for h in range(2)]
        with np.errstate(invalid="ignore"):
            check_gradients(name, heads, c.scale, seen, ([grads[0][rows, h] for h in range(2)], grads[1][keys, 0], grads[2][keys, 0]),
                            "sequence %d" % s, kinds=False)
    if causal:
        assert np.isnan(o[:70]).all() and np.isfinite(o[70:150]).all() and np.all(o[180:200] == 0)
        assert np.isnan(grads[2][:70]).all() and np.isfinite(grads[2][70:150]).all()
    assert np.isnan(o[150:180]).all() and np.all(lse[:, 150:180] == -np.inf) and np.isnan(grads[1][150:180]).all() and np.isnan(grads[0][150:180]).all()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("n", [150, 1500])   # one share, and some
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_scores_that_are_not_finite(A, name, n, bad):
    """Rows that see a score of NaN or plus infinity are NaN, and the logarithm of their sum is; the others are as without that key."""
    def spoil(values):
        values["q"][:, :, 0] = 1.0
        values["k"][n - 50, :, 0] = bad
    c = Case(A, 28, name, [n], [n], 1, 1, 64, change=spoil)
    assert (A.accept_attention_workspace_size(c.desc) > 0) == (n == 1500)
    o, lse = (f64(t) for t in c.forward())
    assert np.isnan(o[n - 50:]).all() and np.isnan(lse[:, n - 50:]).all()
    first = slice(0, n - 50)
    check_forward(name, c.x["q"][first, 0], c.x["k"][first, 0], c.x["v"][first, 0], c.seen(0)[first, first], c.scale, o[first, 0], lse[0, first])
    dq, dk, dv = (f64(g) for g in c.backward())
    assert np.isfinite(dq[first]).all() and np.isnan(dq[n - 50:]).all() and np.isnan(dk).all() and np.isnan(dv).all()


def test_rows_behind_the_last_sequence(A):
    """Left as they were in what the caller gives, zeros in what the call makes or where the descriptor says so."""
    torch = torch_mod()
    c = Case(A, 8, "bf16", [50, 20], [50, 20], 2, 1, 64, behind=300)
    c.forward()
    made = c.backward()
    assert torch.all(c.o[70:] == 0) and torch.all(c.lse[:, 70:] == -float("inf")) and all(torch.all(g[70:] == 0) for g in made)
    o, lse = torch.full_like(c.o, 7.0), torch.full_like(c.lse, 7.0)
    grads = [torch.full_like(g, 7.0) for g in made]
    first = c.o.clone()
    c.forward(o=o, lse=lse)
    c.backward(dq=grads[0], dk=grads[1], dv=grads[2])
    assert torch.all(o[70:] == 7) and torch.all(lse[:, 70:] == 7) and all(torch.all(g[70:] == 7) for g in grads)
    assert torch.equal(o[:70], first[:70]) and all(torch.equal(g[:70], m[:70]) for g, m in zip(grads, made))
    one = c.backward(dq=grads[0])
    assert torch.all(one[0][70:] == 7) and torch.all(one[1][70:] == 0) and torch.all(one[2][70:] == 0)
    c.desc.rest = A.REST_ZEROS
    c.forward(o=o, lse=lse)
    assert torch.all(o[70:] == 0) and torch.all(lse[:, 70:] == -float("inf"))
    c.backward(dq=grads[0], dk=grads[1], dv=grads[2])
    assert all(torch.equal(g, m) for g, m in zip(grads, made))


def test_one_output_given_and_one_made(A):
    """Each has its own rest: kept in what is given, zeros or minus infinity in what is made."""
    torch = torch_mod()
    c = Case(A, 25, "bf16", [50, 20], [50, 20], 2, 1, 64, behind=300)
    o, lse = (t.clone() for t in c.forward())
    torch.full((2, 370), 9.0, device="cuda"), torch.full((370, 2, 64), 9.0, device="cuda").bfloat16()   # (what an allocation may find)
    given = torch.full_like(lse, 7.0)
    made, same = c.forward(lse=given)
    assert same is given and torch.all(given[:, 70:] == 7) and torch.equal(given[:, :70], lse[:, :70]) and torch.equal(made, o)
    given = torch.full_like(o, 7.0)
    same, made = c.forward(o=given)
    assert same is given and torch.all(given[70:] == 7) and torch.equal(given[:70], o[:70]) and torch.equal(made, lse)
    c.desc.rest = A.REST_ZEROS
    assert torch.equal(c.forward(lse=torch.full_like(lse, 7.0))[1], lse) and torch.equal(c.forward(o=torch.full_like(o, 7.0))[0], o)


def test_offsets_beyond_the_tokens_stay_inside(A):
    """Offsets are device data that no host check sees: whatever they hold, nothing outside the tensors is read or written.  (The kernels
    bring them inside first; what such a call computes is not specified.)"""
    torch = torch_mod()
    c = Case(A, 9, "bf16", [50, 20], [50, 20], 2, 1, 64)
    c.q_off, c.k_off = ints([0, 1 << 30, 70]), ints([0, -5, 1 << 30])
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    assert c.o.shape == (70, 2, 64)


def test_offsets_of_many_sequences_beyond_the_tokens_stay_inside(A):
    """The same with more sequences than a workgroup looks at: offsets that rise, fall and go outside."""
    torch = torch_mod()
    rng = np.random.default_rng(27)
    c = Case(A, 27, "bf16", [2] * 300, [2] * 300, 2, 1, 64)
    want, _ = c.forward()
    want = want.clone()
    good = c.q_off, c.k_off
    c.q_off, c.k_off = (ints(rng.integers(-(1 << 31), 1 << 31, 301)) for _ in range(2))
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    assert c.o.shape == (600, 2, 64)
    c.q_off, c.k_off = good
    assert torch.equal(c.forward()[0], want)


def test_no_tokens(A):
    torch = torch_mod()
    for name in ("bf16", "f32"):
        c = Case(A, 10, name, [0], [0], 2, 1, 64)
        assert c.forward()[0].shape == (0, 2, 64) and c.backward()[1].shape == (0, 1, 64)
        c = Case(A, 10, name, [5], [0], 2, 1, 64)
        o, lse = c.forward()
        assert torch.all(o == 0) and torch.all(lse == -float("inf")) and torch.all(c.backward()[0] == 0)
        c = Case(A, 10, name, [0], [5], 2, 1, 64)
        c.forward()
        assert all(torch.all(g == 0) for g in c.backward()[1:])


@pytest.mark.parametrize("causal", [True, False])
def test_gradients_are_differences(A, causal):
    """The float32 gradients against central differences, in 64 bits, of a weighted sum of the definition's outputs, along random directions.
    (The differences' own error, h^2 times the third derivative, is below 1e-7 of them for h = 1e-4 and scores of size 1.)"""
    rng = np.random.default_rng(11)
    c = Case(A, 11, "f32", [37], [37], 2, 1, 40, causal)
    c.forward()
    grads = [f64(g) for g in c.backward()]
    seen = c.seen(0)

    def loss(q, k, v):
        return sum((orc.attention(q[:, h], k[:, 0], v[:, 0], seen, c.scale)[0] * c.x["do"][:, h]).sum() for h in range(2))

    x = [c.x["q"], c.x["k"], c.x["v"]]
    for i in range(3):
        for _ in range(4):
            direction = rng.standard_normal(x[i].shape)
            there = [v + (1e-4 * direction if j == i else 0) for j, v in enumerate(x)]
            back = [v - (1e-4 * direction if j == i else 0) for j, v in enumerate(x)]
            slope = (loss(*there) - loss(*back)) / 2e-4
            terms = np.abs(grads[i] * direction).sum()
            assert abs((grads[i] * direction).sum() - slope) <= 1e-5 * terms


def test_the_same_call_gives_the_same_bits(A):
    torch = torch_mod()
    c = Case(A, 12, "bf16", [300, 41, 512], [300, 41, 512], 4, 1, 128)
    first = [*c.forward(), *c.backward()]
    for _ in range(3):
        again = [*c.forward(), *c.backward()]
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_on_another_stream_and_captured(A):
    """Both passes on a stream of their own, and as a graph that is replayed on other inputs in the same buffers."""
    torch = torch_mod()
    c = Case(A, 13, "bf16", [90, 200], [90, 200], 4, 2, 64)
    want = [t.clone() for t in (*c.forward(), *c.backward())]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [*c.forward(), *c.backward()]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = [*c.forward(), *c.backward()]
    q = c.t["q"].clone()
    for turn in range(3):
        c.t["q"].copy_(q * (1 + turn))
        graph.replay()
        torch.cuda.synchronize()
        eager = [*c.forward(), *c.backward()]
        assert all(torch.equal(a, b) for a, b in zip(eager, held)), turn


def test_long_rows_of_a_wide_tensor(A):
    """Offsets beyond 32 bits: tokens 2^22 - 64 elements apart."""
    torch = torch_mod()
    stride, n = (1 << 22) - 64, 600
    held = torch.empty(n, stride, dtype=torch.bfloat16, device="cuda")
    q = held[:, :128].unflatten(1, (2, 64)).normal_()
    k, v = held[:, 128:192].unflatten(1, (1, 64)).normal_(), held[:, -64:].unflatten(1, (1, 64)).normal_()
    desc = A.make_attention_desc(n, n, 2, 1, 64, dtype=A.BF16, q_stride=stride, k_stride=stride, v_stride=stride)
    near = A.make_attention_desc(n, n, 2, 1, 64, dtype=A.BF16)
    o, lse = A.accept_attention(desc, q, k, v)
    o2, lse2 = A.accept_attention(near, q.contiguous(), k.contiguous(), v.contiguous())
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    do = torch.randn_like(o)
    for a, b in zip(A.accept_attention_backward(desc, do, q, k, v, o, lse),
                    A.accept_attention_backward(near, do, q.contiguous(), k.contiguous(), v.contiguous(), o, lse)):
        assert torch.equal(a, b)


def test_refusals(A):
    torch = torch_mod()
    c = Case(A, 14, "bf16", [20], [20], 2, 1, 64)
    q, k, v = c.t["q"], c.t["k"], c.t["v"]
    c.forward()
    bad = [lambda: A.accept_attention(c.desc, q.float(), k, v), lambda: A.accept_attention(c.desc, q[:19], k, v),
           lambda: A.accept_attention(c.desc, q.cpu(), k, v), lambda: A.accept_attention(c.desc, q.transpose(0, 1).contiguous().transpose(0, 1), k, v),
           lambda: A.accept_attention(c.desc, q, k, v, q_offsets=ints([0, 10, 20])), lambda: A.accept_attention(c.desc, q, k, v, q_offsets=c.q_off.long()),
           lambda: A.accept_attention(c.desc, q, k, v, lse=torch.zeros(20, 2, device="cuda")),
           lambda: A.accept_attention_backward(c.desc, c.t["do"], q, k, v, c.o, c.lse, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda")),
           lambda: A.accept_attention_backward(c.desc, c.t["do"], q, k, v, c.o, c.lse.t().contiguous())]
    for call in bad:
        with pytest.raises(A.AcceptError):
            call()
    held = torch.zeros(20 * 128 + 1, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(A.AcceptError):
        A.accept_attention(c.desc, held[1:].view(20, 2, 64), k, v)   # not 16-byte aligned
