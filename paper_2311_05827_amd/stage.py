"""What a transformer stage computes right behind the boundary it receives from, wired into PyTorch's autograd.

Nothing here computes: the layer norm, its gradients, the quantization to 8-bit blocks and the products all run in
libaccept's kernels (include/accept_stage.h).  This module keeps descriptors from call to call and says which product takes
which operand:

* ``layer_norm(x, weight, bias)``: the statistics are saved for the backward pass.
* ``BlockLinear``: y = x w^T with both operands in E4M3 blocks of 128.  x is quantized once, along its rows for y and along its
  columns for the weight's gradient; the weight once, in squares, for y and for x's gradient; the incoming gradient once, in E5M2,
  along its rows (dx = dy w) and along its columns (dw = dy^T x, in float32).  y and dx have x's type, which also says how they are
  summed: float32 ones in float32, bfloat16 ones by the 8-bit matrix instruction, which cuts products off 13 bits below the largest of
  eight first (about 1e-5 of a result, where its rounding is 2e-3; up to 2^-10 of the sum of the terms' magnitudes, which shows where
  large terms cancel).  For float32's sums of bfloat16 activations pass them as float32.
* ``NormLinear``: the two behind each other; in evaluation mode without gradients the norm writes the product's codes itself.
"""
from __future__ import annotations

import functools

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
