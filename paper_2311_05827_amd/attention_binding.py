"""Binding of libaccept's attention operators (include/accept_attention.h): rotation by position, attention over sequences and its
gradients, a cache of pages and the attention over it.

Argument marshalling only, as in stage_binding.py: tensors are checked on the host against the descriptor, outputs that are not
given are allocated, and the kernels run on the current stream of the current device, where the tensors have to be.  Queries, keys, values and
outputs are (tokens, heads, head_size), their tokens `stride` elements apart, or (tokens, heads * head_size).  What a call allocates
holds zeros (lse: minus infinity) for tokens behind the last sequence, whatever the descriptor's `rest` says; what it is given follows the descriptor.
csrc/native.cpp makes the same checks and calls without the interpreter; whatever it does not take comes to the code here, which says
what is wrong.
"""
from __future__ import annotations

import ctypes

from . import binding as B
from . import stage_binding as S
import torch  # after the binding, which decides the order in which the runtimes are loaded

REST_KEPT, REST_ZEROS = 0, 1
ROTATE_HALVES, ROTATE_NEIGHBOURS = 0, 1
MAX_TOKEN_STRIDE = 1 << 22


class RotateDesc(ctypes.Structure):
    """Mirror of accept_rotate_desc."""
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "heads", "head_size", "rotated", "pairs", "inverse", "rest", "reserved")] + \
               [(n, ctypes.c_int64) for n in ("sequences", "tokens", "x_stride", "y_stride")]


class AttentionDesc(ctypes.Structure):
    """Mirror of accept_attention_desc."""
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "heads", "kv_heads", "head_size", "causal", "rest")] + \
               [(n, ctypes.c_int64) for n in ("sequences", "q_tokens", "k_tokens", "q_stride", "k_stride", "v_stride", "o_stride",
                                              "dq_stride", "dk_stride", "dv_stride")] + [("scale", ctypes.c_double)]


class CacheDesc(ctypes.Structure):
    """Mirror of accept_cache_desc."""
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "heads", "kv_heads", "head_size", "page_size", "rotated", "pairs", "tree_words",
                                              "rest", "reserved")] + \
               [(n, ctypes.c_int64) for n in ("sequences", "tokens", "pages", "table_pages", "q_stride", "k_stride", "v_stride", "o_stride",
                                              "qo_stride")] + [("scale", ctypes.c_double)]


def _declare(lib):
    P, V = ctypes.POINTER, ctypes.c_void_p
    sz = P(ctypes.c_size_t)
    for name, args in (("accept_rotate", [P(RotateDesc)] + [V] * 6),
                       ("accept_attention_workspace_size", [P(AttentionDesc), sz]),
                       ("accept_attention", [P(AttentionDesc)] + [V] * 9),
                       ("accept_attention_backward_workspace_size", [P(AttentionDesc), sz]),
                       ("accept_attention_backward", [P(AttentionDesc)] + [V] * 13),
                       ("accept_cache_append", [P(CacheDesc)] + [V] * 12),
                       ("accept_cache_workspace_size", [P(CacheDesc), sz]),
                       ("accept_cache_attention", [P(CacheDesc)] + [V] * 10)):
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = ctypes.c_int
    return lib


lib = _declare(B.lib)
_native = B._native


# ------------------------------------------------------------------------------- descriptors
def make_rotate_desc(tokens, heads, head_size, rotated=None, dtype=B.F32, pairs=ROTATE_HALVES, inverse=False, sequences=1, x_stride=0,
                     y_stride=0, rest=REST_KEPT):
    """rotated None: all of a head."""
    return RotateDesc(int(dtype), int(heads), int(head_size), int(head_size if rotated is None else rotated), int(pairs), int(inverse),
                      int(rest), 0, int(sequences), int(tokens), int(x_stride), int(y_stride))


def make_attention_desc(q_tokens, k_tokens, heads, kv_heads, head_size, sequences=1, dtype=B.F32, causal=True, scale=None, q_stride=0,
                        k_stride=0, v_stride=0, o_stride=0, dq_stride=0, dk_stride=0, dv_stride=0, rest=REST_KEPT):
    """scale None: 1 / sqrt(head_size)."""
    return AttentionDesc(int(dtype), int(heads), int(kv_heads), int(head_size), int(causal), int(rest), int(sequences), int(q_tokens),
                         int(k_tokens), int(q_stride), int(k_stride), int(v_stride), int(o_stride), int(dq_stride), int(dk_stride),
                         int(dv_stride), _scale(scale, head_size))


def make_cache_desc(tokens, sequences, heads, kv_heads, head_size, page_size, pages, table_pages, dtype=B.F32, rotated=0,
                    pairs=ROTATE_HALVES, tree_words=0, scale=None, q_stride=0, k_stride=0, v_stride=0, o_stride=0, qo_stride=0,
                    rest=REST_KEPT):
    """scale None: 1 / sqrt(head_size)."""
    return CacheDesc(int(dtype), int(heads), int(kv_heads), int(head_size), int(page_size), int(rotated), int(pairs), int(tree_words),
                     int(rest), 0, int(sequences), int(tokens), int(pages), int(table_pages), int(q_stride), int(k_stride),
                     int(v_stride), int(o_stride), int(qo_stride), _scale(scale, head_size))


def _scale(scale, head_size):
    return float(scale) if scale is not None else float(head_size) ** -0.5 if head_size > 0 else 1.0


def accept_attention_workspace_size(desc):
    return S._size_of(lib.accept_attention_workspace_size, desc, "accept_attention_workspace_size")


def accept_attention_backward_workspace_size(desc):
    return S._size_of(lib.accept_attention_backward_workspace_size, desc, "accept_attention_backward_workspace_size")


def accept_cache_workspace_size(desc):
    return S._size_of(lib.accept_cache_workspace_size, desc, "accept_cache_workspace_size")


# ------------------------------------------------------------------------------------ checks
def _check_tokens(t, where, what, dtype, tokens, heads, head, stride):
    """(tokens, heads, head) or (tokens, heads * head), tokens `stride` apart, 16-byte aligned."""
    S._check_place(t, where, what, dtype)
    whole = heads * head
    if tuple(t.shape) not in ((tokens, heads, head), (tokens, whole)):
        S._refuse(where, what, "is %s, the descriptor says %s" % (tuple(t.shape), (tokens, heads, head)))
    if tokens == 0:
        return
    near = t.stride(-1) == 1 and (t.dim() == 2 or heads == 1 or t.stride(1) == head)
    if not near or (tokens > 1 and t.stride(0) != (stride or whole)):
        S._refuse(where, what, "has strides %s, the descriptor says %d from a token to the next" % (tuple(t.stride()), stride or whole))
    if t.data_ptr() % 16:
        S._refuse(where, what, "is not 16-byte aligned")


def _make_tokens(like, tokens, heads, head, stride, zeros=False):
    make = torch.zeros if zeros else torch.empty
    whole = heads * head
    if stride in (0, whole):
        return make((tokens, heads, head), dtype=like.dtype, device=like.device)
    if stride < whole:
        raise B.AcceptError(B.INVALID_ARG, "tokens of %d values are %d apart" % (whole, stride))
    return make((tokens, stride), dtype=like.dtype, device=like.device)[:, :whole].unflatten(1, (heads, head))


def _check_ints(t, where, what, size):
    S._check_flat(t, where, what, torch.int32, size)


def _check_offsets(t, where, what, desc, tokens, otherwise=False):
    if t is not None:
        _check_ints(t, where, what, desc.sequences + 1)
    elif not otherwise and (tokens % desc.sequences if desc.sequences else tokens):
        S._refuse(where, what, "are missing, and %d sequences have %d tokens" % (desc.sequences, tokens))


def _rest_desc(desc, zeros):
    """The descriptor, or, for an output that the call allocates, one with zeros for tokens of no sequence."""
    if not zeros or desc.rest == REST_ZEROS:
        return desc
    other = type(desc).from_buffer_copy(desc)
    other.rest = REST_ZEROS
    return other


# ----------------------------------------------------------------------------------- operators
def accept_rotate(desc, x, frequencies, offsets=None, positions=None, y=None):
    """Enqueue the rotation of x (tokens, heads, head_size) by its tokens' positions on the current stream; returns y, which may be
    given as x.  frequencies (rotated / 2) float32; positions (tokens) int32, or None: a token's place in its sequence."""
    if type(desc) is RotateDesc:
        got = _native.rotate(desc, x, frequencies, offsets, positions, y)
        if type(got) is tuple:
            return got[0]
        if got > 0:
            raise B.AcceptError(got, "accept_rotate")
    where = "accept_rotate"
    S._check_desc(desc, RotateDesc, where)
    if desc.dtype not in (B.F32, B.BF16):
        raise B.AcceptError(B.INVALID_ARG, where + ": bad descriptor")
    dtype = B._DTYPES[desc.dtype]
    sizes = (desc.tokens, desc.heads, desc.head_size)
    _check_tokens(x, where, "x", dtype, *sizes, desc.x_stride)
    if desc.rotated or frequencies is not None:
        S._check_flat(frequencies, where, "frequencies", torch.float32, desc.rotated // 2)
    if positions is not None:
        _check_ints(positions, where, "positions", desc.tokens)
    _check_offsets(offsets, where, "offsets", desc, desc.tokens, positions is not None)
    made = y is None
    if made:
        y = _make_tokens(x, *sizes, desc.y_stride)
    _check_tokens(y, where, "y", dtype, *sizes, desc.y_stride)
    use = _rest_desc(desc, made and offsets is not None)
    B._check(lib.accept_rotate(ctypes.byref(use), B._ptr(x), B._ptr(frequencies), B._ptr(offsets), B._ptr(positions), B._ptr(y),
                               B._stream_handle()), where)
    return y


def _check_attention(where, desc, q, k, v, q_offsets, k_offsets):
    S._check_desc(desc, AttentionDesc, where)
    accept_attention_workspace_size(desc)  # raises on a bad descriptor
    dtype = B._DTYPES[desc.dtype]
    _check_tokens(q, where, "q", dtype, desc.q_tokens, desc.heads, desc.head_size, desc.q_stride)
    _check_tokens(k, where, "k", dtype, desc.k_tokens, desc.kv_heads, desc.head_size, desc.k_stride)
    _check_tokens(v, where, "v", dtype, desc.k_tokens, desc.kv_heads, desc.head_size, desc.v_stride)
    _check_offsets(q_offsets, where, "q_offsets", desc, desc.q_tokens)
    _check_offsets(k_offsets, where, "k_offsets", desc, desc.k_tokens)


def _workspace(where, workspace, nbytes, device):
    if not nbytes:
        return None
    if workspace is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    S._check_workspace(workspace, where, nbytes)
    return workspace


def accept_attention(desc, q, k, v, q_offsets=None, k_offsets=None, o=None, lse=None, workspace=None):
    """Enqueue attention of q (q_tokens, heads, head_size) over k and v (k_tokens, kv_heads, head_size) on the current stream; returns
    (o, lse), lse (heads, q_tokens) float32 as the backward pass takes it."""
    if type(desc) is AttentionDesc:
        got = _native.attention(desc, q, k, v, q_offsets, k_offsets, o, lse, workspace)
        if type(got) is tuple:
            return got
        if got > 0:
            raise B.AcceptError(got, "accept_attention")
    where = "accept_attention"
    _check_attention(where, desc, q, k, v, q_offsets, k_offsets)
    sizes = (desc.q_tokens, desc.heads, desc.head_size)
    made = o is None and lse is None
    one = not made and q_offsets is not None  # one of the two: what is made here has its rest from here
    if lse is None:
        lse = torch.full((desc.heads, desc.q_tokens), float("-inf"), dtype=torch.float32, device=q.device) if one else \
            torch.empty((desc.heads, desc.q_tokens), dtype=torch.float32, device=q.device)
    if o is None:
        o = _make_tokens(q, *sizes, desc.o_stride, one)
    _check_tokens(o, where, "o", q.dtype, *sizes, desc.o_stride)
    S._check_table(lse, where, "lse", torch.float32, desc.heads, desc.q_tokens)
    workspace = _workspace(where, workspace, accept_attention_workspace_size(desc), q.device)
    use = _rest_desc(desc, made and q_offsets is not None)
    B._check(lib.accept_attention(ctypes.byref(use), B._ptr(q), B._ptr(k), B._ptr(v), B._ptr(q_offsets), B._ptr(k_offsets), B._ptr(o),
                                  B._ptr(lse), B._ptr(workspace), B._stream_handle()), where)
    return o, lse


def accept_attention_backward(desc, do, q, k, v, o, lse, q_offsets=None, k_offsets=None, dq=None, dk=None, dv=None, workspace=None):
    """Gradients of accept_attention from its outputs and that of o: (dq, dk, dv)."""
    if type(desc) is AttentionDesc:
        got = _native.attention_backward(desc, do, q, k, v, o, lse, q_offsets, k_offsets, dq, dk, dv, workspace)
        if type(got) is tuple:
            return got
        if got > 0:
            raise B.AcceptError(got, "accept_attention_backward")
    where = "accept_attention_backward"
    _check_attention(where, desc, q, k, v, q_offsets, k_offsets)
    of_q, of_k = (desc.q_tokens, desc.heads, desc.head_size), (desc.k_tokens, desc.kv_heads, desc.head_size)
    _check_tokens(do, where, "do", q.dtype, *of_q, desc.o_stride)
    _check_tokens(o, where, "o", q.dtype, *of_q, desc.o_stride)
    S._check_table(lse, where, "lse", torch.float32, desc.heads, desc.q_tokens)
    made = dq is None and dk is None and dv is None
    zeros = not made  # one by one: each that is made here has its zeros from here
    if dq is None:
        dq = _make_tokens(q, *of_q, desc.dq_stride, zeros and q_offsets is not None)
    if dk is None:
        dk = _make_tokens(k, *of_k, desc.dk_stride, zeros and k_offsets is not None)
    if dv is None:
        dv = _make_tokens(v, *of_k, desc.dv_stride, zeros and k_offsets is not None)
    _check_tokens(dq, where, "dq", q.dtype, *of_q, desc.dq_stride)
    _check_tokens(dk, where, "dk", q.dtype, *of_k, desc.dk_stride)
    _check_tokens(dv, where, "dv", q.dtype, *of_k, desc.dv_stride)
    workspace = _workspace(where, workspace, accept_attention_backward_workspace_size(desc), q.device)
    use = _rest_desc(desc, made and (q_offsets is not None or k_offsets is not None))
    B._check(lib.accept_attention_backward(ctypes.byref(use), B._ptr(do), B._ptr(q), B._ptr(k), B._ptr(v), B._ptr(o), B._ptr(lse),
                                           B._ptr(q_offsets), B._ptr(k_offsets), B._ptr(dq), B._ptr(dk), B._ptr(dv), B._ptr(workspace),
                                           B._stream_handle()), where)
    return dq, dk, dv


def _check_cache(where, desc, k_cache, v_cache, table, lengths, offsets):
    S._check_desc(desc, CacheDesc, where)
    accept_cache_workspace_size(desc)  # raises on a bad descriptor
    size = (desc.pages, desc.kv_heads, desc.page_size, desc.head_size)
    for t, what in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        S._check_place(t, where, what, B._DTYPES[desc.dtype])
        if tuple(t.shape) != size or not t.is_contiguous():
            S._refuse(where, what, "is %s, the descriptor says contiguous %s" % (tuple(t.shape), size))
        if t.data_ptr() % 16:
            S._refuse(where, what, "is not 16-byte aligned")
    S._check_table(table, where, "table", torch.int32, desc.sequences, desc.table_pages)
    _check_ints(lengths, where, "lengths", desc.sequences)
    _check_offsets(offsets, where, "offsets", desc, desc.tokens)


def accept_cache_append(desc, q, k, v, k_cache, v_cache, table, lengths, offsets=None, positions=None, frequencies=None, q_out=None):
    """Enqueue the way of k (rotated) and v (tokens, kv_heads, head_size) into the places behind their sequences' lengths on the
    current stream; returns q rotated (q_out, which may be q), or None for q None.  positions (tokens) int32, or None: a token's place."""
    if type(desc) is CacheDesc:
        got = _native.cache_append(desc, q, k, v, k_cache, v_cache, table, lengths, offsets, positions, frequencies, q_out)
        if type(got) is tuple:
            return got[0]
        if got > 0:
            raise B.AcceptError(got, "accept_cache_append")
    where = "accept_cache_append"
    _check_cache(where, desc, k_cache, v_cache, table, lengths, offsets)
    dtype = B._DTYPES[desc.dtype]
    _check_tokens(k, where, "k", dtype, desc.tokens, desc.kv_heads, desc.head_size, desc.k_stride)
    _check_tokens(v, where, "v", dtype, desc.tokens, desc.kv_heads, desc.head_size, desc.v_stride)
    if desc.rotated or frequencies is not None:
        S._check_flat(frequencies, where, "frequencies", torch.float32, desc.rotated // 2)
    if positions is not None:
        _check_ints(positions, where, "positions", desc.tokens)
    made = False
    if q is not None:
        sizes = (desc.tokens, desc.heads, desc.head_size)
        _check_tokens(q, where, "q", dtype, *sizes, desc.q_stride)
        made = q_out is None
        if made:
            q_out = _make_tokens(q, *sizes, desc.qo_stride)
        _check_tokens(q_out, where, "q_out", dtype, *sizes, desc.qo_stride)
    elif q_out is not None:
        S._refuse(where, "q", "is missing")
    use = _rest_desc(desc, made and offsets is not None)
    B._check(lib.accept_cache_append(ctypes.byref(use), B._ptr(q), B._ptr(k), B._ptr(v), B._ptr(frequencies), B._ptr(offsets),
                                     B._ptr(lengths), B._ptr(positions), B._ptr(table), B._ptr(q_out), B._ptr(k_cache), B._ptr(v_cache),
                                     B._stream_handle()), where)
    return q_out


def accept_cache_attention(desc, q, k_cache, v_cache, table, lengths, offsets=None, tree=None, o=None, workspace=None):
    """Enqueue attention of q (tokens, heads, head_size) over its sequences' places on the current stream; lengths are those that the
    append of the same tokens took.  tree (tokens, tree_words) int64, the bits of the new tokens that each sees.  Returns o."""
    if type(desc) is CacheDesc:
        got = _native.cache_attention(desc, q, k_cache, v_cache, table, lengths, offsets, tree, o, workspace)
        if type(got) is tuple:
            return got[0]
        if got > 0:
            raise B.AcceptError(got, "accept_cache_attention")
    where = "accept_cache_attention"
    _check_cache(where, desc, k_cache, v_cache, table, lengths, offsets)
    dtype, sizes = B._DTYPES[desc.dtype], (desc.tokens, desc.heads, desc.head_size)
    _check_tokens(q, where, "q", dtype, *sizes, desc.q_stride)
    if desc.tree_words:
        S._check_table(tree, where, "tree", torch.int64, desc.tokens, desc.tree_words)
    elif tree is not None:
        S._refuse(where, "tree", "is given, the descriptor has no words for it")
    made = o is None
    if made:
        o = _make_tokens(q, *sizes, desc.o_stride)
    _check_tokens(o, where, "o", dtype, *sizes, desc.o_stride)
    workspace = _workspace(where, workspace, accept_cache_workspace_size(desc), q.device)
    use = _rest_desc(desc, made and offsets is not None)
    B._check(lib.accept_cache_attention(ctypes.byref(use), B._ptr(q), B._ptr(k_cache), B._ptr(v_cache), B._ptr(offsets), B._ptr(lengths),
                                        B._ptr(table), B._ptr(tree), B._ptr(o), B._ptr(workspace), B._stream_handle()), where)
    return o
