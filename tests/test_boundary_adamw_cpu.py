"""Numbers at the ends of their types that the calls of the optimizer refuse, on the host."""
import ctypes as C

import pytest
import torch

import paper_2506_21263_amd as dlcx

F = 0x10000  # aligned to 256, never read
TOP = (1 << 63) - 1


def test_lengths_whose_blocks_would_overflow():
    L = dlcx.lib()
    out = dlcx.Table()
    for numel in (TOP, TOP - 4095, 1 << 62, (1 << 31) * 4096):
        t = dlcx.Tensor(grad=F, numel=numel, grad_dtype=dlcx.F32)
        assert L.dlcx_tensor_table(C.addressof(t), 1, F, C.addressof(out), None) == dlcx.EINVAL, numel
        assert L.dlcx_state_decode(0, F, F, numel, F, 0, None) == dlcx.EINVAL, numel


def test_hyperparameters_that_fp32_has_no_room_for():
    t = dlcx.Table(memory=F, blocks=1, count=1, steps=1)

    def adamw(lr=1e-3, eps=1e-8, gs=1.0):
        return dlcx.lib().dlcx_adamw(C.addressof(t), lr, 0.9, 0.95, eps, 1, gs, None, 0.0, None)

    for bad in (dict(eps=1e-46), dict(eps=1e39), dict(gs=1e39), dict(lr=1e39), dict(lr=-1e39)):
        assert adamw(**bad) == dlcx.EINVAL, bad


def test_tensors_of_types_that_have_no_kernel():
    g = torch.zeros(8)
    for bad, says in ((dict(grad=g.half()), "float32 or bfloat16"), (dict(grad=g, param=g.double(), m=g, v=g), "float32 or bfloat16"),
                      (dict(grad=g, param=g), "moments"), (dict(grad=g, param=g, m=g), "moments")):
        with pytest.raises(ValueError, match=says):
            dlcx.tensor(**bad)
