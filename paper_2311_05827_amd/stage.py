"""What a transformer stage computes right behind the boundary it receives from, wired into PyTorch's autograd.

Nothing here computes: the layer norm, its gradients, the quantization to 8-bit blocks, the products, rotation and attention all run in
libaccept's kernels (include/accept_stage.h, include/accept_attention.h).  This module keeps descriptors from call to call and says which product takes
which operand:

* ``layer_norm(x, weight, bias)``: the statistics are saved for the backward pass.
* ``BlockLinear``: y = x w^T with both operands in E4M3 blocks of 128.  x is quantized once, along its rows for y and along its
  columns for the weight's gradient; the weight once, in squares, for y and for x's gradient; the incoming gradient once, in E5M2,
  along its rows (dx = dy w) and along its columns (dw = dy^T x, in float32).  y and dx have x's type, which also says how they are
  summed: float32 ones in float32, bfloat16 ones by the 8-bit matrix instruction, which cuts products off 13 bits below the largest of
  eight first (about 1e-5 of a result, where its rounding is 2e-3; up to 2^-10 of the sum of the terms' magnitudes, which shows where
  large terms cancel).  For float32's sums of bfloat16 activations pass them as float32.
* ``NormLinear``: the two behind each other; in evaluation mode without gradients the norm writes the product's codes itself.
* ``rotate``, ``attention``: of tokens of a batch, or of sequences packed behind each other; o and the logarithms of the rows' sums
  are saved for the backward pass, the scores never.
* ``SelfAttention``: a block's first half: `NormLinear` to queries, keys and values side by side, rotation, attention and a product; with a
  ``Cache`` its new tokens are appended to the cache's pages and attend to all that is there.
"""
from __future__ import annotations

import functools

from . import attention_binding as T
from . import binding as B
from . import stage_binding as S
import torch  # after the binding, which decides the order in which the runtimes are loaded


def _flat(x):
    """(rows, cols) of x's last axis; contiguous."""
    return x.reshape(-1, x.shape[-1]).contiguous()


# Descriptors by their sizes: making one takes longer than the call it describes.
_norm_desc = functools.lru_cache(maxsize=1024)(S.make_norm_desc)
_block_desc = functools.lru_cache(maxsize=1024)(S.make_block_desc)
_matmul_desc = functools.lru_cache(maxsize=1024)(S.make_matmul_desc)
_rotate_desc = functools.lru_cache(maxsize=1024)(T.make_rotate_desc)
_attention_desc = functools.lru_cache(maxsize=1024)(T.make_attention_desc)
_cache_desc = functools.lru_cache(maxsize=1024)(T.make_cache_desc)


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        flat = _flat(x)
        code = B.dtype_code(flat)
        desc = _norm_desc(flat.shape[0], flat.shape[1], x_dtype=code, y_dtype=code, eps=eps,
                          param_dtype=B.dtype_code(weight if weight is not None else bias if bias is not None else flat))
        y, stats = S.accept_layer_norm(desc, flat, weight, bias)
        ctx.save_for_backward(flat, weight, stats)
        ctx.desc = desc
        ctx.shapes = [None if t is None else t.shape for t in (weight, bias)]
        return y.view(x.shape)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, stats = ctx.saved_tensors
        dx, dweight, dbias = S.accept_layer_norm_backward(ctx.desc, _flat(dy), x, weight, stats,
                                                          need_weight=ctx.needs_input_grad[1], need_bias=ctx.needs_input_grad[2])
        dweight, dbias = (g if g is None else g.view(shape) for g, shape in zip((dweight, dbias), ctx.shapes))
        return dx.view(dy.shape), dweight, dbias, None


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over x's last axis (float32 or bfloat16; weight and bias of one type, either); y has x's type."""
    return _LayerNorm.apply(x, weight, bias, eps)


class _BlockLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight):
        flat = _flat(x)
        (m, k), n = flat.shape, weight.shape[0]
        need_x, need_w = ctx.needs_input_grad[:2]
        codes, scales, x_t, xs_t = S.accept_block_quantize(_block_desc(m, k, in_dtype=B.dtype_code(flat)), flat, colwise=need_w)
        w, ws, w_t, ws_t = quantize_weight(weight, colwise=need_x)
        ctx.save_for_backward(x_t, xs_t, w_t, ws_t)
        ctx.shape, ctx.sizes, ctx.out, ctx.w_dtype = x.shape, (m, n, k), B.dtype_code(flat), weight.dtype
        return S.accept_block_matmul(_matmul_desc(m, n, k, out_dtype=ctx.out), codes, scales, w, ws).view(*x.shape[:-1], n)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x_t, xs_t, w_t, ws_t = ctx.saved_tensors
        (m, n, k), flat = ctx.sizes, _flat(dy)
        need_x, need_w = ctx.needs_input_grad
        codes, scales, codes_t, scales_t = S.accept_block_quantize(
            _block_desc(m, n, in_dtype=B.dtype_code(flat), code=S.E5M2), flat, rowwise=need_x, colwise=need_w)
        dx = dweight = None
        if need_x:
            dx = S.accept_block_matmul(_matmul_desc(m, k, n, out_dtype=ctx.out, a_code=S.E5M2), codes, scales, w_t, ws_t).view(ctx.shape)
        if need_w:
            dweight = S.accept_block_matmul(_matmul_desc(n, k, m, a_code=S.E5M2, b_group=1), codes_t, scales_t, x_t, xs_t).to(ctx.w_dtype)
        return dx, dweight


def quantize_weight(weight, colwise):
    """(codes, scales, codes_t, scales_t) of a weight in squares of 128, the last two None unless asked for."""
    w = weight.detach().contiguous()
    return S.accept_block_quantize(_block_desc(w.shape[0], w.shape[1], group=S.BLOCK, in_dtype=B.dtype_code(w)), w, colwise=colwise)


def _version(t):
    """Counts the changes that PyTorch sees (a tensor made in inference mode has no count)."""
    return None if t.is_inference() else t._version


class BlockLinear(torch.nn.Module):
    """y = x w^T with x and w in 8-bit blocks (see the module's text).  The weight is kept in float32 (or bfloat16) for the
    optimizer and quantized in every call, unless it was laid out for serving: see `freeze`."""

    def __init__(self, in_features, out_features, device="cuda", dtype=torch.float32):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, device=device, dtype=dtype))
        torch.nn.init.normal_(self.weight, std=in_features ** -0.5)
        self._frozen = None

    def freeze(self):
        """Keep the codes of the weight as it is now for the calls without gradients that follow, until the weight changes: by an
        optimizer, `load_state_dict`, `to`, another parameter in its place or any other way that PyTorch counts, or by a call that
        will have a gradient for it.  From then on it is quantized in every call again.  A change behind PyTorch's back (`weight.data`)
        takes another `freeze`, or `unfreeze`."""
        self._frozen = (self.weight, _version(self.weight), quantize_weight(self.weight, colwise=False)[:2])
        return self

    def unfreeze(self):
        self._frozen = None
        return self

    def _apply(self, fn, recurse=True):
        self._frozen = None  # `to` and its like put other data into the parameter without a count
        return super()._apply(fn, recurse)

    def _weight_codes(self):
        frozen = self._frozen
        if frozen is not None:
            weight, version, codes = frozen
            if weight is self.weight and version == _version(weight):
                return codes
            self._frozen = None
        return quantize_weight(self.weight, colwise=False)[:2]

    def serve(self, codes, scales, out_dtype):
        """The product of codes (m, in_features), without gradients."""
        (m, k), n = codes.shape, self.weight.shape[0]
        w, ws = self._weight_codes()
        return S.accept_block_matmul(_matmul_desc(m, n, k, out_dtype=out_dtype), codes, scales, w, ws)

    def forward(self, x):
        if torch.is_grad_enabled():
            if self.weight.requires_grad:
                self._frozen = None  # (an optimizer's fused step is not counted)
            return _BlockLinear.apply(x, self.weight)
        flat = _flat(x)
        codes, scales, _, _ = S.accept_block_quantize(_block_desc(*flat.shape, in_dtype=B.dtype_code(flat)), flat)
        return self.serve(codes, scales, B.dtype_code(flat)).view(*x.shape[:-1], self.weight.shape[0])


class NormLinear(torch.nn.Module):
    """A block's entry: layer norm, then a product.  In evaluation mode (`eval`), where no gradient is asked for, the norm writes its
    output as the product's codes, and no float of it is ever stored.  In training mode the norm's output is rounded to x's type first
    with and without gradients: a pass that is computed again for its gradients, as in activation checkpointing, gives the same bits."""

    def __init__(self, in_features, out_features, eps=1e-5, device="cuda", dtype=torch.float32):
        super().__init__()
        self.norm_weight = torch.nn.Parameter(torch.ones(in_features, device=device, dtype=dtype))
        self.norm_bias = torch.nn.Parameter(torch.zeros(in_features, device=device, dtype=dtype))
        self.linear = BlockLinear(in_features, out_features, device=device, dtype=dtype)
        self.eps = eps

    def forward(self, x):
        if self.training or torch.is_grad_enabled():
            return self.linear(layer_norm(x, self.norm_weight, self.norm_bias, self.eps))
        flat = _flat(x)
        code = B.dtype_code(flat)
        desc = _norm_desc(*flat.shape, x_dtype=code, param_dtype=B.dtype_code(self.norm_weight), eps=self.eps)
        codes, scales, _ = S.accept_layer_norm_quantize(desc, flat, self.norm_weight, self.norm_bias)
        return self.linear.serve(codes, scales, code).view(*x.shape[:-1], self.linear.weight.shape[0])


# ---- attention --------------------------------------------------------------------------------
def _tokens(t):
    """(tokens, heads, head) of (batch, n, heads, head) or (tokens, heads, head), with a stride and an alignment that the operators take."""
    if t.dim() not in (3, 4):
        raise ValueError("%s is neither (batch, n, heads, head) nor (tokens, heads, head)" % (tuple(t.shape),))
    t = t.flatten(0, -3)
    heads, head = t.shape[1:]
    if t.stride(2) == 1 and (heads == 1 or t.stride(1) == head) and heads * head <= t.stride(0) <= T.MAX_TOKEN_STRIDE:
        if t.stride(0) * t.element_size() % 16 == 0 and t.data_ptr() % 16 == 0:
            return t
    t = t.contiguous()
    if t.data_ptr() % 16:
        t = t.clone()
    return t.as_strided(t.shape, (heads * head, head, 1))  # one token has any stride, and is contiguous


def _no_gradients(what, *tensors):
    """Where a tensor's gradient would be lost without a word."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise ValueError("%s has no gradients: call it without them" % what)


def _same_batch(offsets, *tensors):
    """Without offsets the tensors' sequences are those of one batch."""
    if offsets is None and len({t.shape[0] if t.dim() == 4 else None for t in tensors}) > 1:
        raise ValueError("batches of %s" % ", ".join(str(tuple(t.shape)) for t in tensors))


def _sequences(x, offsets):
    """How many: those of the offsets, or the batch's, or one."""
    if offsets is not None:
        return offsets.numel() - 1
    return x.shape[0] if x.dim() == 4 else 1


class _Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, frequencies, offsets, positions, pairs):
        flat = _tokens(x)
        ctx.kind = dict(rotated=2 * frequencies.numel(), dtype=B.dtype_code(flat), pairs=pairs, sequences=_sequences(x, offsets))
        ctx.save_for_backward(frequencies, offsets, positions)
        return T.accept_rotate(_rotate_desc(*flat.shape, x_stride=flat.stride(0), **ctx.kind), flat, frequencies, offsets, positions).view(x.shape)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        flat = _tokens(dy)
        desc = _rotate_desc(*flat.shape, x_stride=flat.stride(0), inverse=True, **ctx.kind)
        return T.accept_rotate(desc, flat, *ctx.saved_tensors).view(dy.shape), None, None, None, None


def rotate(x, frequencies, offsets=None, positions=None, neighbours=False):
    """x (batch, n, heads, head) or (tokens, heads, head) turned by its tokens' positions: their places in their sequences (those of a
    batch; or of `offsets`, sequences + 1 int32 device values), or `positions` (int32, one a token).  frequencies: a float32 for each pair, the angle of a
    step (no gradient: one that asks for it is refused); pairs are a value of the first half of those that turn and one of the second, or two neighbours."""
    _no_gradients("rotation by frequencies", frequencies)
    return _Rotate.apply(x, frequencies, offsets, positions, T.ROTATE_NEIGHBOURS if neighbours else T.ROTATE_HALVES)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, q_offsets, k_offsets, causal, scale):
        fq, fk, fv = _tokens(q), _tokens(k), _tokens(v)
        ctx.desc = _attention_desc(fq.shape[0], fk.shape[0], fq.shape[1], fk.shape[1], fq.shape[2], sequences=_sequences(q, q_offsets),
                                   dtype=B.dtype_code(fq), causal=causal, scale=scale, q_stride=fq.stride(0), k_stride=fk.stride(0),
                                   v_stride=fv.stride(0))
        o, lse = T.accept_attention(ctx.desc, fq, fk, fv, q_offsets, k_offsets)
        ctx.save_for_backward(fq, fk, fv, o, lse, q_offsets, k_offsets)
        ctx.shapes = q.shape, k.shape, v.shape
        return o.view(q.shape)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do):
        q, k, v, o, lse, q_offsets, k_offsets = ctx.saved_tensors
        do = do.reshape(o.shape).contiguous()
        grads = T.accept_attention_backward(ctx.desc, do if do.data_ptr() % 16 == 0 else do.clone(), q, k, v, o, lse, q_offsets, k_offsets)
        return *(g.view(shape) for g, shape in zip(grads, ctx.shapes)), None, None, None, None


def attention(q, k, v, offsets=None, k_offsets=None, causal=True, scale=None):
    """q (batch, n, heads, head) over k and v (batch, m, kv_heads, head), or tokens of packed sequences (tokens, heads, head) with their
    offsets (sequences + 1 int32 device values; k_offsets None: q's).  float32 or bfloat16; heads / kv_heads query heads share a key head.
    With a causal mask a sequence's last query sees its last key.  Tokens behind the last sequence give and get zeros."""
    _same_batch(offsets if k_offsets is None else k_offsets, q, k, v)
    return _Attention.apply(q, k, v, offsets, offsets if k_offsets is None else k_offsets, bool(causal), scale)


class _TurnedAttention(torch.autograd.Function):
    """attention of queries and keys turned by their places, all three side by side in one tensor (tokens, heads + 2 kv_heads, head)."""

    @staticmethod
    def forward(ctx, qkv, frequencies, offsets, sequences, heads, kv, pairs):
        n, both, head = qkv.shape
        wide, code = both * head, B.dtype_code(qkv)
        ctx.kind = dict(rotated=2 * frequencies.numel(), dtype=code, pairs=pairs, sequences=sequences)
        turned = T.accept_rotate(_rotate_desc(n, heads + kv, head, x_stride=wide, **ctx.kind), qkv[:, :heads + kv], frequencies, offsets)
        ctx.desc = _attention_desc(n, n, heads, kv, head, sequences=sequences, dtype=code, q_stride=(heads + kv) * head,
                                   k_stride=(heads + kv) * head, v_stride=wide, dq_stride=wide, dk_stride=wide, dv_stride=wide, rest=T.REST_ZEROS)
        o, lse = T.accept_attention(ctx.desc, turned[:, :heads], turned[:, heads:], qkv[:, heads + kv:], offsets, offsets)
        ctx.save_for_backward(qkv, turned, frequencies, offsets, o, lse)
        return o

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do):
        qkv, turned, frequencies, offsets, o, lse = ctx.saved_tensors
        n, both, head = qkv.shape
        turning, heads, kv = turned.shape[1], ctx.desc.heads, ctx.desc.kv_heads
        do = do.contiguous()
        d = torch.empty_like(qkv)
        T.accept_attention_backward(ctx.desc, do if do.data_ptr() % 16 == 0 else do.clone(), turned[:, :heads], turned[:, heads:], qkv[:, turning:],
                                    o, lse, offsets, offsets, dq=d[:, :heads], dk=d[:, heads:turning], dv=d[:, turning:])
        both_turn = d[:, :turning]
        T.accept_rotate(_rotate_desc(n, turning, head, x_stride=both * head, y_stride=both * head, inverse=True, **ctx.kind), both_turn, frequencies,
                        offsets, y=both_turn)
        return d, None, None, None, None, None, None


class Cache:
    """Keys and values of the sequences that a server is at, in pages of `page_size` tokens, and how many tokens each has (`lengths`).

    Sequences have room for `capacity` tokens each, their pages in order, unless `pages` (how many there are) and `table` (sequences, pages of each;
    int32 on the device) say otherwise; a table may be changed between steps, and sequences may share the pages that none of them writes.  `lengths` are on
    the device, so no call looks whether there is room: a token behind its sequence's last page in the table has no place, its key and value are
    dropped, and nobody sees it, itself included."""

    def __init__(self, sequences, capacity, kv_heads, head_size, page_size=64, dtype=torch.bfloat16, device="cuda", pages=None, table=None):
        each = -(-capacity // page_size)
        if table is None:
            table = torch.arange(sequences * each, dtype=torch.int32, device=device).view(sequences, each)
            pages = sequences * each if pages is None else pages
        elif pages is None:
            raise ValueError("a table needs the number of pages")
        self.k = torch.zeros(pages, kv_heads, page_size, head_size, dtype=dtype, device=device)
        self.v = torch.zeros_like(self.k)
        self.table, self.lengths = table, torch.zeros(sequences, dtype=torch.int32, device=device)

    def step(self, q, k, v, offsets=None, frequencies=None, positions=None, tree=None, neighbours=False, scale=None, advance=None):
        """Append the new tokens' keys (turned, where there are frequencies) and values, and let their queries (turned) attend to all that their
        sequences hold: o (tokens, heads, head), without gradients (tensors that ask for some are refused).  The tokens are those of `offsets`, or as many of each sequence.  tree (tokens, words)
        int64: the new tokens of its sequence that each token sees, as bits, instead of those up to itself; with it a token's position has to be given.
        Then the sequences are longer by their new tokens, unless `advance` says no: a tree's are to be appended again, those that were
        accepted, so `advance` is no for trees if nothing is said."""
        _no_gradients("a cache", q, k, v, frequencies)
        if tree is not None and frequencies is not None and positions is None:
            raise ValueError("tokens of a tree need positions")
        _same_batch(offsets, q, k, v)
        if offsets is None and q.dim() == 4 and q.shape[0] != self.table.shape[0]:
            raise ValueError("a batch of %d for %d sequences" % (q.shape[0], self.table.shape[0]))
        q, k, v = _tokens(q), _tokens(k), _tokens(v)
        n, heads, head = q.shape
        pages, kv, page_size, _ = self.k.shape
        kind = dict(dtype=B.dtype_code(q), rotated=0 if frequencies is None else 2 * frequencies.numel(),
                    pairs=T.ROTATE_NEIGHBOURS if neighbours else T.ROTATE_HALVES, tree_words=0 if tree is None else tree.shape[1], scale=scale)
        sizes = (n, self.table.shape[0], heads, kv, head, page_size, pages, self.table.shape[1])
        turned = frequencies is not None
        out = T.accept_cache_append(_cache_desc(*sizes, q_stride=q.stride(0), k_stride=k.stride(0), v_stride=v.stride(0), **kind),
                                    q if turned else None, k, v, self.k, self.v, self.table, self.lengths, offsets, positions, frequencies)
        q = out if turned else q
        o = T.accept_cache_attention(_cache_desc(*sizes, q_stride=q.stride(0), **kind), q, self.k, self.v, self.table, self.lengths, offsets, tree)
        if tree is None if advance is None else advance:
            self.lengths += n // max(self.table.shape[0], 1) if offsets is None else offsets[1:] - offsets[:-1]
        return o


class SelfAttention(torch.nn.Module):
    """A block's first half, without its residual's addition: layer norm, queries, keys and values by a product in 8-bit blocks, attention of
    tokens turned by their positions, and a product.

    x is (batch, n, features), or (tokens, features) with the `offsets` of packed sequences, or, for serving (no gradients), with a `Cache`: the new
    tokens of its sequences, as many of each or those of `offsets`."""

    def __init__(self, features, heads, kv_heads=None, head_size=None, rotated=None, base=10000.0, neighbours=False, eps=1e-5, device="cuda",
                 dtype=torch.float32):
        super().__init__()
        self.heads, self.kv_heads = heads, heads if kv_heads is None else kv_heads
        self.head_size = features // heads if head_size is None else head_size
        self.pairs = T.ROTATE_NEIGHBOURS if neighbours else T.ROTATE_HALVES
        self.entry = NormLinear(features, (heads + 2 * self.kv_heads) * self.head_size, eps=eps, device=device, dtype=dtype)
        self.out = BlockLinear(heads * self.head_size, features, device=device, dtype=dtype)
        self._rotated = self.head_size if rotated is None else rotated, base
        self.register_buffer("frequencies", self._make_frequencies().to(device), persistent=False)

    def _make_frequencies(self):
        rotated, base = self._rotated
        return (base ** (-torch.arange(0, rotated, 2, dtype=torch.float64) / max(rotated, 1))).float()

    def _apply(self, fn, recurse=True):
        kept = self.frequencies
        super()._apply(fn, recurse)
        # It moves with the module, but in float32 with the values that it has: fewer bits are angles off by radians, and it is in no state to load.
        self.frequencies = (self._make_frequencies() if kept.is_meta else kept).to(self.frequencies.device)
        return self

    def cache(self, sequences, capacity, page_size=64, dtype=torch.bfloat16):
        """A cache of this block's keys and values for so many sequences of up to `capacity` tokens."""
        return Cache(sequences, capacity, self.kv_heads, self.head_size, page_size, dtype, self.frequencies.device)

    def forward(self, x, offsets=None, cache=None, positions=None, tree=None, advance=None):
        sequences = offsets.numel() - 1 if offsets is not None else x.shape[0] if x.dim() == 3 else 1
        qkv = self.entry(x).view(-1, self.heads + 2 * self.kv_heads, self.head_size)
        if cache is None:
            if positions is not None or tree is not None:
                raise ValueError("positions and trees are for calls with a cache")
            o = _TurnedAttention.apply(qkv, self.frequencies, offsets, sequences, self.heads, self.kv_heads, self.pairs)
        else:
            _no_gradients("a cache", qkv)
            if offsets is None and x.dim() == 3 and x.shape[0] != cache.table.shape[0]:
                raise ValueError("a batch of %d for %d sequences" % (x.shape[0], cache.table.shape[0]))
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
            o = cache.step(q, k, v, offsets, self.frequencies, positions, tree, self.pairs == T.ROTATE_NEIGHBOURS, advance=advance)
        return self.out(o.view(*x.shape[:-1], self.heads * self.head_size))
