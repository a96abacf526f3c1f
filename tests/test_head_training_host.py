"""Refusals of the operators that the shared head is trained with: nothing here reaches a GPU.  (The pointers are made up; a call
that got past its checks would fail to launch and return another code.)"""
import ctypes as C

import pytest
import torch

import paper_2404_16710_amd as P
from paper_2404_16710_amd import binding as B

ARG, RANGE, CAPACITY = -1, -2, -3
F32, BF16 = B.LS_F32, B.LS_BF16
P0, P1, P2, P3, P4, P5, WS = (C.c_void_p(0x10000 * k) for k in range(1, 8))
BIG = 1 << 40


def changed(args, i, value):
    return [value if k == i else a for k, a in enumerate(args)]


NORM = [P0, F32, 64, P1, BF16, 3, 64, 1e-5, P2, 64, None]
NORM_GRAD = [P0, F32, 64, P1, BF16, P2, 64, 3, 64, 1e-5, P3, 64, P4, WS, BIG, None]
LOSS = [P0, 64, P1, BF16, P2, 3, 64, 100, P3, P4, WS, BIG, None]
GRAD = [P0, 64, P1, BF16, P2, P3, 3, 64, 100, P4, None, P5, 64, P3, WS, BIG, None]


@pytest.mark.parametrize("name, args, i, value, code", [
    ("ls_rms_norm", NORM, 0, None, ARG), ("ls_rms_norm", NORM, 3, None, ARG), ("ls_rms_norm", NORM, 8, None, ARG),
    ("ls_rms_norm", NORM, 0, C.c_void_p(0x10008), ARG), ("ls_rms_norm", NORM, 8, C.c_void_p(0x10002), ARG),
    ("ls_rms_norm", NORM, 1, 2, ARG), ("ls_rms_norm", NORM, 4, -1, ARG), ("ls_rms_norm", NORM, 5, 0, RANGE),
    ("ls_rms_norm", NORM, 5, (1 << 24) + 1, RANGE), ("ls_rms_norm", NORM, 6, 0, RANGE), ("ls_rms_norm", NORM, 6, 40, RANGE),
    ("ls_rms_norm", NORM, 6, 65552, RANGE), ("ls_rms_norm", NORM, 7, 0.0, RANGE), ("ls_rms_norm", NORM, 7, float("nan"), RANGE),
    ("ls_rms_norm", NORM, 2, 63, RANGE), ("ls_rms_norm", NORM, 2, 66, RANGE), ("ls_rms_norm", NORM, 9, 68, RANGE), ("ls_rms_norm", NORM, 9, -64, RANGE),
    ("ls_rms_norm_grad", NORM_GRAD, 5, None, ARG), ("ls_rms_norm_grad", NORM_GRAD, 13, None, ARG), ("ls_rms_norm_grad", NORM_GRAD, 13, C.c_void_p(0x70010), ARG),
    ("ls_rms_norm_grad", NORM_GRAD, 14, 3 * 64 * 4 - 1, CAPACITY), ("ls_rms_norm_grad", NORM_GRAD, 7, -1, RANGE), ("ls_rms_norm_grad", NORM_GRAD, 11, 60, RANGE),
    ("ls_rms_norm_grad", NORM_GRAD, 6, 68, RANGE), ("ls_rms_norm_grad", NORM_GRAD, 12, C.c_void_p(0x10004), ARG),
    ("ls_head_loss", LOSS, 0, None, ARG), ("ls_head_loss", LOSS, 2, C.c_void_p(0x10008), ARG), ("ls_head_loss", LOSS, 3, 5, ARG), ("ls_head_loss", LOSS, 4, None, ARG),
    ("ls_head_loss", LOSS, 8, None, ARG), ("ls_head_loss", LOSS, 9, C.c_void_p(0x10002), ARG), ("ls_head_loss", LOSS, 10, None, ARG),
    ("ls_head_loss", LOSS, 5, 0, RANGE), ("ls_head_loss", LOSS, 5, (1 << 22) + 1, RANGE), ("ls_head_loss", LOSS, 6, 72, RANGE), ("ls_head_loss", LOSS, 7, 0, RANGE),
    ("ls_head_loss", LOSS, 7, (1 << 21) + 1, RANGE), ("ls_head_loss", LOSS, 1, 60, RANGE), ("ls_head_loss", LOSS, 1, 68, RANGE), ("ls_head_loss", LOSS, 11, 16, CAPACITY),
    ("ls_head_loss_grad", GRAD, 5, None, ARG), ("ls_head_loss_grad", GRAD, 11, None, ARG), ("ls_head_loss_grad", GRAD, 13, None, ARG),
    ("ls_head_loss_grad", GRAD, 12, 48, RANGE), ("ls_head_loss_grad", GRAD, 15, 1000, CAPACITY), ("ls_head_loss_grad", GRAD, 14, C.c_void_p(0x70080), ARG),
])
def test_bad_arguments_are_refused(name, args, i, value, code):
    assert getattr(B.lib(), name)(*changed(args, i, value)) == code


def test_norm_gradient_with_nothing_wanted_is_refused():
    assert B.lib().ls_rms_norm_grad(*changed(changed(NORM_GRAD, 10, None), 12, None)) == ARG


def test_workspaces_are_sized_for_supported_arguments_only():
    L = B.lib()
    assert L.ls_rms_norm_grad_workspace(3, 64) >= 3 * 64 * 4 and L.ls_rms_norm_grad_workspace(0, 64) == 0 and L.ls_rms_norm_grad_workspace(3, 65) == 0
    size = L.ls_head_loss_workspace
    assert size(0, 64, 100, BF16, 0) == size(1, 64, 100, 3, 0) == size(1, 64, 100, BF16, 2) == size(1, 60, 100, BF16, 0) == size(1, 64, 0, BF16, 0) == 0
    # many rows of a large vocabulary: at most 64 MB of statistics, or 256 rows
    assert size(1 << 22, 64, 128256, BF16, 0) < 70 << 20 and size(1 << 22, 64, 1 << 21, BF16, 0) < 256 * (1 << 18) + (1 << 20)
    # no logits without gradients; with them at most about 4 GB of logits and p, however many rows
    assert 0 < size(4096, 4096, 32000, BF16, 0) < 16 << 20
    assert 4096 * 32000 * 6 <= size(4096, 4096, 32000, BF16, 1) < 4096 * 32000 * 6 + (64 << 20)
    assert size(1 << 20, 4096, 128256, BF16, 1) < (4 << 30) + 128256 * 4096 * 4 + (1 << 30)


ADAM = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0, grad_scale=1.0, step=1, state_bits=32)


def adam(config=None, n_tensors=1, **tensor):
    t = dict(param=0x10000, grad=0x20000, master=None, m=0x30000, v=0x40000, m_scale=0x50000, v_scale=0x60000, n=100, param_dtype=F32, grad_dtype=F32)
    t.update(tensor)
    table = (B.ls_adam_tensor * 1)(B.ls_adam_tensor(*t.values()))
    c = B.ls_adam_config(*{**ADAM, **(config or {})}.values())
    return B.lib().ls_adamw(table, n_tensors, C.byref(c), None)


@pytest.mark.parametrize("config, tensor, code", [
    ({"step": 0}, {}, RANGE), ({"state_bits": 16}, {}, ARG), ({"beta1": 1.0}, {}, RANGE), ({"beta2": -0.1}, {}, RANGE), ({"eps": 0.0}, {}, RANGE), ({"eps": 1e-40}, {}, RANGE),
    ({"lr": -1.0}, {}, RANGE), ({"lr": float("inf")}, {}, RANGE), ({"weight_decay": float("nan")}, {}, RANGE), ({"grad_scale": float("inf")}, {}, RANGE),
    ({}, {"n": -1}, RANGE), ({}, {"n": (1 << 42) + 1}, RANGE), ({}, {"param": None}, ARG), ({}, {"grad": 0x20008}, ARG), ({}, {"m": None}, ARG), ({}, {"v": 0x40004}, ARG),
    ({}, {"master": 0x80004}, ARG), ({}, {"param_dtype": 2}, ARG), ({}, {"grad_dtype": -1}, ARG),
    ({"state_bits": 8}, {"m_scale": None}, ARG), ({"state_bits": 8}, {"v_scale": 0x60002}, ARG),
])
def test_bad_adamw_arguments_are_refused(config, tensor, code):
    assert adam(config, **tensor) == code


def test_adamw_over_nothing():
    L = B.lib()
    c = B.ls_adam_config(*ADAM.values())
    assert L.ls_adamw(None, 0, C.byref(c), None) == 0 and adam(n=0, param=None) == 0
    assert L.ls_adamw(None, 1, C.byref(c), None) == ARG and L.ls_adamw(None, -1, C.byref(c), None) == RANGE and L.ls_adamw(None, 0, None, None) == ARG


def test_exit_loss_refuses_null_arguments():
    L = B.lib()
    scale = (C.c_float * 4)(1, 1, 1, 1)
    assert L.ls_exit_loss(None, P0, P1, 4, scale, P2, None, None, WS, BIG, None) == ARG
    assert L.ls_exit_loss_workspace(None, 4, scale, 0) == 0


def test_the_binding_refuses_tensors_that_are_not_what_it_needs():
    x, gain = torch.zeros(4, 32), torch.zeros(32)
    with pytest.raises(ValueError, match="GPU"):
        P.rms_norm(x, gain, 1e-5)
    with pytest.raises(ValueError, match="GPU"):
        P.head_loss(x, torch.zeros(9, 32), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="contiguous rows"):
        P.rms_norm(torch.zeros(32, 4).T, gain, 1e-5)
    with pytest.raises(ValueError, match="float32 nor bfloat16"):
        B._dtype_of(x.half(), "x")
    with pytest.raises(ValueError, match="tensor 0"):
        P.AdamW([x], [x])
    with pytest.raises(ValueError, match="one of each"):
        P.AdamW([x], [])
    with pytest.raises(ValueError, match="twice"):
        P.AdamW([x, x], [x, x])
    with pytest.raises(ValueError, match="8 or 32"):
        P.AdamW([x], [x], bits=16)
