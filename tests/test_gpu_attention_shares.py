"""Attention whose keys, or whose keys' queries, are shared out among workgroups because there are few: against the oracle in 64 bits, and what a
share does not see or has none of."""
import numpy as np
import pytest

from attention_util import check_forward, check_gradients, ints
from stage_util import f64, torch_mod
from test_gpu_attention import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


# lengths of queries and keys, heads, key heads, head size, shares expected at least (forward, backward)
SIZES = [
    ([1], [5000], 1, 1, 64, 4, 1),
    ([3, 1], [1100, 3000], 2, 1, 128, 2, 1),
    ([1500], [1500], 2, 1, 128, 2, 4),
    ([2100, 0, 40], [2100, 7, 40], 2, 2, 80, 1, 2),
    ([2000], [300], 4, 1, 64, 1, 8),            # most rows see no key
    ([1200], [1200], 1, 1, 256, 2, 2),
]


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("q_lengths,k_lengths,heads,kv_heads,head,forward,backward", SIZES)
def test_both_passes(A, name, causal, q_lengths, k_lengths, heads, kv_heads, head, forward, backward):
    c = Case(A, 1, name, q_lengths, k_lengths, heads, kv_heads, head, causal)
    one = 4 * heads * c.nq * head
    assert A.accept_attention_workspace_size(c.desc) >= (forward * one if forward > 1 else 0)
    assert A.accept_attention_backward_workspace_size(c.desc) >= (8 * backward * c.nk * kv_heads * head if backward > 1 else 0)
    c.forward()
    c.check_forward()
    c.check_backward(c.backward())


def test_rows_behind_the_last_sequence(A):
    torch = torch_mod()
    c = Case(A, 2, "bf16", [1100, 900], [1100, 900], 2, 1, 64, behind=70)
    assert A.accept_attention_backward_workspace_size(c.desc) > 8 * 2 * c.nq + 256
    c.forward()
    made = c.backward()
    assert torch.all(c.o[2000:] == 0) and torch.all(c.lse[:, 2000:] == -float("inf")) and all(torch.all(g[2000:] == 0) for g in made)
    o, lse, grads = torch.full_like(c.o, 7.0), torch.full_like(c.lse, 7.0), [torch.full_like(g, 7.0) for g in made]
    first = c.o.clone()
    c.forward(o=o, lse=lse)
    c.backward(dq=grads[0], dk=grads[1], dv=grads[2])
    assert torch.all(o[2000:] == 7) and torch.all(lse[:, 2000:] == 7) and all(torch.all(g[2000:] == 7) for g in grads)
    assert torch.equal(o[:2000], first[:2000]) and all(torch.equal(g[:2000], m[:2000]) for g, m in zip(grads, made))


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_what_is_not_seen_has_no_effect(A, name):
    """A value that is NaN is seen by the rows from its own on, in one share only."""
    def spoil(values):
        values["v"][1300, 0, 5] = np.nan
    c = Case(A, 3, name, [1500], [1500], 1, 1, 64, change=spoil)
    assert A.accept_attention_workspace_size(c.desc) > 0
    o = f64(c.forward()[0])
    assert np.isfinite(o[:1300]).all() and np.isnan(o[1300:, 0, 5]).all() and np.isfinite(np.delete(o, 5, axis=2)).all()
    c.check_forward()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("token", [40, 780, 1490])
def test_gradients_of_what_is_not_seen(A, name, token):
    """A gradient that is NaN, in one share of the queries, and a key, in one of the keys."""
    def spoil_do(values):
        values["do"][token, 1, 5] = np.nan

    def spoil_k(values):
        values["k"][token, 0, 5] = np.nan
    for spoil in (spoil_do, spoil_k):
        c = Case(A, 7, name, [1500], [1500], 2, 1, 128, change=spoil)
        assert A.accept_attention_backward_workspace_size(c.desc) > 8 * 2 * c.nq + 256
        c.forward()
        o, lse = f64(c.o), f64(c.lse)
        dq, dk, dv = (f64(g) for g in c.backward())
        heads = [(c.x["do"][:, h], c.x["q"][:, h], c.x["k"][:, 0], c.x["v"][:, 0], o[:, h], lse[h]) for h in range(2)]
        with np.errstate(invalid="ignore"):
            check_gradients(name, heads, c.scale, c.seen(0), ([dq[:, 0], dq[:, 1]], dk[:, 0], dv[:, 0]), kinds=False)
        if spoil is spoil_do:
            assert np.isfinite(dv[token + 1:]).all() and np.isfinite(dk[token + 1:]).all() and np.isfinite(np.delete(dq, token, axis=0)).all()
        else:
            assert np.isfinite(o[:token]).all() and np.isfinite(dq[:token]).all()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("minus", [2500, 3000])
def test_scores_of_minus_infinity(A, name, minus):
    """Of all keys: the row is NaN; of all but the last share's: it is as if those were not there.  (The second sequence's row sees no key.)"""
    def spoil(values):
        values["q"][:, :, 0] = 1.0
        values["k"][:minus, :, 0] = -np.inf
    c = Case(A, 6, name, [1, 3], [3000, 0], 2, 1, 64, False, change=spoil)
    assert A.accept_attention_workspace_size(c.desc) > 0
    o, lse = (f64(t) for t in c.forward())
    assert np.all(o[1:] == 0) and np.all(lse[:, 1:] == -np.inf)
    for h in range(2):
        if minus == 3000:
            assert np.isnan(o[0, h]).all() and lse[h, 0] == -np.inf
        else:
            check_forward(name, c.x["q"][:1, h], c.x["k"][minus:, 0], c.x["v"][minus:, 0], np.ones((1, 3000 - minus), bool), c.scale, o[:1, h], lse[h, :1])


def test_the_same_bits_and_workspaces(A):
    """Again, with a workspace that holds NaN, on another stream and captured."""
    torch = torch_mod()
    c = Case(A, 4, "bf16", [1600], [1600], 2, 1, 64)
    fw = torch.full((A.accept_attention_workspace_size(c.desc) // 4,), float("nan"), device="cuda")
    bw = torch.full((A.accept_attention_backward_workspace_size(c.desc) // 4,), float("nan"), device="cuda")
    want = [*c.forward(), *c.backward()]
    assert fw.numel() > 0
    for _ in range(2):
        got = [*c.forward(workspace=fw.view(torch.uint8)), *c.backward(workspace=bw.view(torch.uint8))]
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = [*c.forward(), *c.backward()]
    for _ in range(3):
        c.t["q"].normal_()
        graph.replay()
        torch.cuda.synchronize()
        eager = [*c.forward(), *c.backward()]
        assert all(torch.equal(a, b) for a, b in zip(held, eager))
    with pytest.raises(A.AcceptError):
        c.forward(workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))


def test_without_offsets(A):
    c = Case(A, 5, "bf16", [1100, 1100], [1100, 1100], 1, 1, 128, packed=False)
    assert A.accept_attention_workspace_size(c.desc) > 0
    c.forward()
    c.check_forward()
    c.check_backward(c.backward())
