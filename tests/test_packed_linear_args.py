"""Refusals of the products with bit-packed weights and of the 8-bit activations: found on the host, before anything is
enqueued (so these run without a GPU; the pointers below are never followed)."""
import ctypes

import pytest
import torch

import paper_2602_04929_b200 as tb
from paper_2602_04929_b200 import binding

ONE = 256
W = dict(d_out=256, d_in=512, bits=4, quant_group=128, packed=ONE, scales=ONE, zeros=ONE)
A = dict(n_adapters=3, rank=16, n_requests=2, A=ONE, B=ONE, scale=ONE, starts=ONE, ids=ONE)


def _w(**kw):
    return ctypes.addressof(_w.__dict__.setdefault("keep", []).append(tb.PackedWeight(**dict(W, **kw))) or _w.keep[-1])


def _a(**kw):
    return ctypes.addressof(_a.__dict__.setdefault("keep", []).append(tb.Adapters(**dict(A, **kw))) or _a.keep[-1])


def forward(w=None, a=None, x=ONE, t=1, n=5, y=ONE, xa=ONE, ws=ONE, nb=1 << 40):
    return tb.load().tb_packed_linear(w or _w(), a, x, t, n, y, xa, ws, nb, None)


def backward(w=None, a=None, dy=ONE, t=1, n=5, x=ONE, codes=None, cs=None, xa=ONE, dx=ONE, dA=ONE, dB=ONE, ws=ONE, nb=1 << 40):
    return tb.load().tb_packed_linear_backward(w or _w(), a, dy, t, n, x, codes, cs, xa, dx, dA, dB, ws, nb, None)


def test_structures_match_the_header():
    assert ctypes.sizeof(tb.PackedWeight) == 16 + 3 * 8
    assert ctypes.sizeof(tb.Adapters) == 16 + 5 * 8


BAD_W = [(dict(d_out=0), 1), (dict(d_in=-32), 1), (dict(bits=1), 1), (dict(bits=9), 1), (dict(quant_group=-1), 1),
         (dict(quant_group=96), 1), (dict(packed=None), 1), (dict(scales=None), 1), (dict(zeros=None), 1), (dict(packed=ONE + 4), 1),
         (dict(d_in=520, quant_group=0), 2), (dict(d_out=252), 2), (dict(quant_group=16), 2), (dict(d_out=1 << 25), 2)]
BAD_A = [(dict(n_adapters=0), 1), (dict(rank=0), 1), (dict(n_requests=0), 1), (dict(A=None), 1), (dict(B=None), 1),
         (dict(scale=None), 1), (dict(starts=None), 1), (dict(ids=None), 1), (dict(A=ONE + 8), 1), (dict(B=ONE + 2), 1),
         (dict(rank=12), 2), (dict(rank=136), 2), (dict(n_adapters=70000), 2)]


@pytest.mark.parametrize("kw,status", BAD_W)
def test_bad_weights(kw, status):
    assert forward(_w(**kw)) == status
    assert backward(_w(**kw), _a()) == status


@pytest.mark.parametrize("kw,status", BAD_A)
def test_bad_adapters(kw, status):
    assert forward(a=_a(**kw)) == status
    assert backward(a=_a(**kw)) == status


def test_bad_calls():
    assert forward(t=2) == 1 and forward(n=-1) == 1 and forward(n=1 << 31) == 2
    for kw in (dict(x=None), dict(y=None), dict(x=ONE + 8), dict(y=ONE + 2), dict(a=_a(), xa=None), dict(a=_a(), xa=ONE + 4)):
        assert forward(**kw) == 1, kw
    assert backward(a=_a(), t=5) == 1 and backward(a=_a(), n=-3) == 1
    for kw in (dict(dy=None), dict(dy=ONE + 8), dict(dx=ONE + 8), dict(dA=None), dict(dB=None), dict(dA=ONE + 4), dict(x=None),
               dict(codes=ONE, cs=ONE), dict(x=None, codes=ONE), dict(x=None, cs=ONE), dict(xa=None), dict(x=ONE + 8),
               dict(dx=None, dA=None, dB=None)):
        assert backward(**dict(dict(a=_a()), **kw)) == 1, kw
    assert backward() == 1                               # gradients of adapters without adapters
    lib = tb.load()
    need = lib.tb_packed_linear_backward_workspace(_w(), _a(), 1, 5)
    assert need > 0 and need % 256 == 0
    for kw in (dict(ws=None), dict(ws=ONE + 8), dict(nb=need - 1)):
        assert backward(a=_a(), **kw) == 3, kw


def test_workspace_queries():
    lib = tb.load()
    for fn in (lib.tb_packed_linear_workspace, lib.tb_packed_linear_backward_workspace):
        assert fn(None, None, 1, 5) == 0 and fn(_w(bits=1), None, 1, 5) == 0 and fn(_w(), None, 1, 0) == 0
        # shapes alone decide: a query needs no pointers
        assert fn(_w(packed=None, scales=None, zeros=None), _a(A=None, B=None), 1, 300) == fn(_w(), _a(), 1, 300)


def test_bad_8_bit_calls():
    lib = tb.load()
    assert lib.tb_checkpoint_pack(ONE, 2, 4, 64, ONE, ONE, None) == 1
    assert lib.tb_checkpoint_pack(ONE, 1, -1, 64, ONE, ONE, None) == 1
    assert lib.tb_checkpoint_pack(ONE, 1, 4, 0, ONE, ONE, None) == 1
    assert lib.tb_checkpoint_pack(ONE, 1, 4, 72, ONE, ONE, None) == 2
    assert lib.tb_checkpoint_pack(None, 1, 4, 64, ONE, ONE, None) == 1
    assert lib.tb_checkpoint_pack(ONE, 1, 4, 64, ONE + 8, ONE, None) == 1
    assert lib.tb_checkpoint_unpack(ONE, None, 4, 64, 1, ONE, None) == 1
    assert lib.tb_checkpoint_unpack(ONE, ONE, 4, 64, 1, ONE + 8, None) == 1
    assert lib.tb_checkpoint_unpack(ONE, ONE, 4, 40, 1, ONE, None) == 2


def test_binding_refuses_host_tensors_and_shapes():
    cpu = torch.zeros((8, 4), dtype=torch.int32)
    with pytest.raises(ValueError):
        tb.packed_weight(cpu, torch.zeros(8, 1), torch.zeros(8, 1, dtype=torch.int32), 32, 4)   # no CUDA tensors
    with pytest.raises(ValueError):
        tb.packed_weight(cpu, torch.zeros(8, 1), torch.zeros(8, 1, dtype=torch.int32), 64, 4)   # width
    with pytest.raises(ValueError):
        tb.packed_weight(cpu, torch.zeros(8, 2), torch.zeros(8, 1, dtype=torch.int32), 32, 4)   # groups
    with pytest.raises(ValueError):
        tb.adapters(torch.zeros(2, 8, 32), torch.zeros(2, 4, 32), torch.zeros(2), cpu[0], cpu[0, 1:])
    with pytest.raises(ValueError):
        tb.adapters(torch.zeros(2, 8, 32), torch.zeros(2, 8, 32), torch.zeros(2), cpu[0], cpu[0])
    assert binding.PackedWeight is tb.PackedWeight
