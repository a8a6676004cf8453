"""Helpers of the attention operators' tests: inputs, the oracle over sequences, and bounds of the errors.

Bounds.  U = 2^-24 and H = 2^-8 (bfloat16's rounding; 0 for float32) are relative to the value.  A score is a sum of `head` products in
float32, scaled, and put relative to the row's maximum: off by at most d_i = (head + 8) U scale max_j sum |q_i||k_j| + 4 U |lse_i|.  A weight
relative to its sum is then off by 2 d_i and by the sums' and the exponentials' (n + 16) U of itself, and its rounding to bfloat16 by
H; so o is off by at most (H + 2 d_i + (n + 16) U) sum p|v|, and its own rounding.  ds_ij = p_ij (do_i v_j - e_i) scale has p's error, that of
its difference, (head + 8) U scale p_ij (sum |do_i||v_j| + sum |do_i||o_i|), and H; the sums over n of them n U more.
An exponential below float32's smallest normal value, 2^-126, is zero: a weight that the formula has is then off by all of itself, so by up to
TINY = 2^-126 (forward, where weights are relative to a maximum that may be 2^8 behind the row's true one, their sum at least 2^-8 of the largest: 2^-118), times what it is multiplied by.
"""
import numpy as np

from oracle import attention_oracle as orc
from stage_util import HALF_BF16, U, dtype_of, f64, rounding, torch_mod


TINY = 2.0 ** -126


def tokens_of(values, name, pad=0):
    """(device tensor (tokens, heads, head) of that type, its tokens `pad` elements further apart; the values it holds).  What lies
    between the tokens is NaN."""
    torch = torch_mod()
    n, heads, head = values.shape
    held = torch.full((n, heads * head + pad), float("nan"), dtype=dtype_of(name))
    t = held[:, :heads * head].unflatten(1, (heads, head))
    t.copy_(torch.from_numpy(np.ascontiguousarray(values)))
    t = held.cuda()[:, :heads * head].unflatten(1, (heads, head))
    return t, t.cpu().double().numpy()


def ints(values):
    torch = torch_mod()
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def ends_of(lengths):
    return [0] + list(np.cumsum(lengths))


def score_error(q, k, seen, scale, lse):
    """d_i of every row."""
    with np.errstate(invalid="ignore"):
        terms = np.where(seen, np.abs(q) @ np.abs(k).T, 0.0).max(axis=1, initial=0.0)
    return (q.shape[1] + 8) * U * scale * terms + 4 * U * np.abs(np.where(np.isfinite(lse), lse, 0))


def half(name):
    return HALF_BF16 if name == "bf16" else 0.0


def check_forward(name, q, k, v, seen, scale, got_o, got_lse=None, what=""):
    """One head against the oracle."""
    o, lse, p = orc.attention(q, k, v, seen, scale)
    d, n = score_error(q, k, seen, scale, lse), k.shape[0]
    bound = (half(name) + 2 * d + (n + 16) * U)[:, None] * orc.weighted(p, np.abs(v), seen)
    bound = bound + 2.0 ** 8 * TINY * orc.weighted(seen.astype(float), np.abs(v), seen)
    bound = bound + rounding(name, np.abs(o) + bound)
    same(got_o, o, bound, what + " o")
    if got_lse is not None:
        same(got_lse, lse, d + (n + 16) * U + 2 * U * np.abs(np.where(np.isfinite(lse), lse, 0)), what + " lse")


def same(got, want, bound, what, kinds=True):
    """Within the bound; where the oracle's value is not finite, the same one (kinds false: one that is not finite either)."""
    finite = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), finite), what + ": not finite elsewhere"
    if kinds:
        assert np.array_equal(np.isnan(got), np.isnan(want)), what + ": NaN elsewhere"
        assert np.array_equal(got[~finite & ~np.isnan(want)], want[~finite & ~np.isnan(want)]), what + ": infinities elsewhere"
    off = np.abs(got[finite] - want[finite])
    over = off > np.broadcast_to(bound, want.shape)[finite]
    assert not over.any(), "%s: off by %g where %g is allowed (%d of %d values)" % (
        what, off[over].max(), np.broadcast_to(bound, want.shape)[finite][over][off[over].argmax()], over.sum(), over.size)


def check_gradients(name, heads, scale, seen, got, what="", kinds=True):
    """The heads that share a key head: `heads` is a list of (do, q, k, v, o, lse); got = ([dq of each], dk, dv)."""
    dqs, dk, dv = got
    want_k, want_v, bound_k, bound_v = 0.0, 0.0, 0.0, 0.0
    h = half(name)
    m = len(heads) * seen.shape[0]
    for (do, q, k, v, o, lse), dq in zip(heads, dqs):
        n, size = k.shape
        wq, wk, wv, p, ds = orc.gradients(do, q, k, v, o, lse, seen, scale)
        d = score_error(q, k, seen, scale, lse)[:, None] + 16 * U
        with np.errstate(invalid="ignore"):
            terms = np.abs(do) @ np.abs(v).T + (np.abs(do) * np.abs(o)).sum(1, keepdims=True)
            difference = np.where(seen, scale * (p * (size + 8) * U + TINY) * terms, 0.0)
        e_ds = np.abs(ds) * (h + d) + difference
        bound = orc.weighted(e_ds + n * U * np.abs(ds), np.abs(k), seen)
        same(dq, wq, bound + rounding(name, np.abs(wq) + bound), what + " dq", kinds)
        want_k, want_v = want_k + wk, want_v + wv
        bound_k = bound_k + orc.weighted((e_ds + m * U * np.abs(ds)).T, np.abs(q), seen.T)
        bound_v = bound_v + orc.weighted((p * (h + d + m * U) + TINY).T, np.abs(do), seen.T)
    same(dk, want_k, bound_k + rounding(name, np.abs(want_k) + bound_k), what + " dk", kinds)
    same(dv, want_v, bound_v + rounding(name, np.abs(want_v) + bound_v), what + " dv", kinds)
