"""Outputs that are given are written, whole, by both ways that a call can take: they are filled with another pattern before each."""
import pytest

import test_gpu_stage_binding as binding
from stage_util import torch_mod

pytestmark = pytest.mark.gpu
A = binding.A


def filled(t, byte):
    """t's memory as far as the call may write it (the rows of codes are whole blocks), every byte that."""
    torch = torch_mod()
    wide = torch.as_strided(t, (t.shape[0], t.stride(0)), (t.stride(0), 1)) if t.dim() == 2 else t
    wide.view(torch.uint8).fill_(byte)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("name", binding.NAMES)
def test_given_outputs_are_written(A, name, native, monkeypatch):
    function, good, outs = binding.calls(A)[name]
    want = [t.clone() for t in binding.as_tuple(function(**good))]
    if not native:
        monkeypatch.setattr(A.stage_binding, "_native", binding._Nothing())
    for byte in (0xA5, 0x00):
        for t in outs.values():
            filled(t, byte)
        got = binding.as_tuple(function(**good, **outs))
        for w, g, o in zip(want, got, outs.values()):
            assert g.data_ptr() == o.data_ptr() and binding.same(w, o)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("name", binding.NAMES)
def test_each_output_given_alone(A, name, native, monkeypatch):
    function, good, outs = binding.calls(A)[name]
    want = [t.clone() for t in binding.as_tuple(function(**good))]
    if not native:
        monkeypatch.setattr(A.stage_binding, "_native", binding._Nothing())
    for i, (key, t) in enumerate(outs.items()):
        filled(t, 0xA5)
        got = binding.as_tuple(function(**good, **{key: t}))
        assert got[i].data_ptr() == t.data_ptr()
        for w, g in zip(want, got):
            assert binding.same(w, g)
