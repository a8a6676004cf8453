"""Helpers of the stage operators' tests: tensors of a type and stride, values of codes and scales, rounding bounds."""
import numpy as np

from oracle import stage_oracle as orc

U = 2.0 ** -24          # float32: half the distance of neighbouring values, relative
HALF_BF16 = 2.0 ** -8   # bfloat16 (7 fraction bits): the same


def torch_mod():
    import torch
    return torch


def dtype_of(name):
    torch = torch_mod()
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def matrix(values, name, pad=0, offset=0):
    """(device tensor of that type, rows `pad` elements further apart than they are long and the first `offset` in; the
    values it holds, in 64 bits).  What lies between the rows is NaN."""
    torch = torch_mod()
    rows, cols = values.shape
    held = torch.full((offset + rows * (cols + pad),), float("nan"), dtype=dtype_of(name))
    t = held[offset:].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.from_numpy(np.ascontiguousarray(values)))
    held = held.cuda()
    t = held[offset:].view(rows, cols + pad)[:, :cols]
    return t, t.cpu().double().numpy()


def vector(values, name):
    torch = torch_mod()
    t = torch.from_numpy(np.ascontiguousarray(values)).to(dtype_of(name)).cuda()
    return t, t.cpu().double().numpy()


def f64(t):
    return t.detach().cpu().double().numpy()


def code_values(t, code):
    """Values of a tensor of codes, from its bytes."""
    torch = torch_mod()
    return orc.decode(t.contiguous().view(torch.uint8).cpu().numpy(), code)


def exponents(t):
    torch = torch_mod()
    return t.view(torch.uint8).cpu().numpy().astype(np.int64) - 127


def rounding(name, values):
    """Half the distance of neighbouring values of the type."""
    return (U if name == "f32" else HALF_BF16) * np.abs(values)


def hidden(rng, rows, cols):
    return rng.standard_t(3, size=(rows, cols)) * np.exp(0.5 * rng.standard_normal(cols)) + 0.3 * rng.standard_normal(cols)
