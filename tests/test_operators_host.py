"""Refusals of the grouped products, group norm and gradient clipping, which need no GPU: the library checks its arguments
before any HIP call, and the binding its tensors before it calls the library."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2504_04673_amd as sagnn
from paper_2504_04673_amd import binding

P = 1 << 20          # an aligned address that is never used
EINVAL, ECAPACITY = -1, -2


def call(name, good, **change):
    """The call with `good` arguments (a dict in order), some of them changed: its code.  Only for calls that are refused."""
    args = dict(good)
    assert set(change) <= set(args)
    args.update(change)
    return getattr(binding._calls(), name)(*args.values())


GEMM = dict(dtype=0, X=P, ldx=16, W=P, ldw=24, stride_w=384, transW=0, off=P, groups=3, m=100, kdim=16, nout=24, prec=0, act=0, mask=None,
            ldmask=0, Y=P, ldy=24, stream=None)


@pytest.mark.parametrize("change", [
    {"dtype": 2}, {"dtype": -1}, {"dtype": 1, "prec": 1}, {"dtype": 1, "prec": 2}, {"prec": 3}, {"prec": -1}, {"act": 2}, {"act": -1}, {"transW": 2},
    {"groups": 0}, {"groups": -1}, {"groups": 65537}, {"m": -1}, {"m": 1 << 31}, {"kdim": 0}, {"nout": 0}, {"kdim": 65537, "ldx": 65537},
    {"nout": 65537, "ldy": 65537, "ldw": 65537}, {"ldx": 15}, {"ldw": 23}, {"transW": 1, "ldw": 15}, {"ldy": 23}, {"stride_w": -1},
    {"mask": P, "ldmask": 23}, {"X": None}, {"W": None}, {"off": None}, {"Y": None}, {"X": P + 2}, {"W": P + 1}, {"Y": P + 2},
    {"mask": P + 2, "ldmask": 24}, {"dtype": 1, "X": P + 1}, {"off": P + 2},
])
def test_grouped_gemm_act_refuses(change):
    assert call("grouped_gemm_act", GEMM, **change) == EINVAL


def test_grouped_gemm_of_no_rows_is_done():
    assert call("grouped_gemm_act", GEMM, m=0, X=None, W=None, off=None, Y=None) == 0


BWD = dict(dtype=0, X=P, ldx=16, W=P, ldw=24, stride_w=384, off=P, groups=3, m=100, kdim=16, nout=24, prec=0, G=P, ldg=24, mask=None, ldmask=0,
           dX=P, lddx=16, dW=P, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [
    {"dtype": 2}, {"dtype": 1, "prec": 2}, {"prec": 5}, {"groups": 0}, {"m": -1}, {"kdim": 0}, {"nout": -4}, {"ldx": 15}, {"ldg": 23}, {"ldw": 20},
    {"lddx": 15}, {"stride_w": -384}, {"mask": P, "ldmask": 15}, {"X": None}, {"W": None}, {"G": None}, {"off": None}, {"G": P + 2}, {"dX": P + 1},
    {"dW": P + 2}, {"X": P + 3}, {"ws": P + 2}, {"off": P + 1},
])
def test_grouped_gemm_bwd_refuses(change):
    assert call("grouped_gemm_bwd", BWD, **change) == EINVAL


def test_grouped_gemm_bwd_needs_its_workspace():
    b = ctypes.c_size_t(0)
    query = sagnn.lib().grouped_gemm_bwd_workspace_bytes
    assert query(1_000_000, 3, 16, 24, ctypes.byref(b)) == 0 and b.value > 0
    assert call("grouped_gemm_bwd", BWD, m=1_000_000, ws_bytes=b.value - 1) == ECAPACITY
    assert call("grouped_gemm_bwd", BWD, m=1_000_000, ws=None) == EINVAL
    assert query(10, 0, 16, 24, ctypes.byref(b)) == EINVAL and query(10, 3, 16, 24, None) == EINVAL
    assert query(-1, 3, 16, 24, ctypes.byref(b)) == EINVAL and query(10, 3, 16, 70000, ctypes.byref(b)) == EINVAL
    assert call("grouped_gemm_bwd", BWD, m=0, X=None, W=None, G=None, dW=None, ws=None, ws_bytes=0, off=None) == 0


FWD_NORM = dict(dtype=0, X=P, ldx=24, seg=P, n_seg=4, max_rows=0, m=100, C=24, groups=3, gamma=P, beta=P, eps=1e-5, act=1, Y=P, ldy=24, mean=P,
                rstd=P, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [
    {"dtype": 2}, {"n_seg": 0}, {"n_seg": -1}, {"max_rows": -1}, {"m": -1}, {"m": 1 << 31}, {"C": 0}, {"C": 16385, "ldx": 16385, "ldy": 16385, "groups": 1},
    {"groups": 0}, {"groups": 5}, {"groups": 1025, "C": 2050, "ldx": 2050, "ldy": 2050}, {"eps": -1e-5}, {"eps": float("nan")},
    {"eps": float("inf")}, {"act": 3}, {"act": -1}, {"ldx": 23}, {"ldy": 23}, {"X": None}, {"Y": None}, {"mean": None}, {"rstd": None},
    {"m": 500_000, "ws": None}, {"seg": None, "n_seg": 7}, {"X": P + 2}, {"Y": P + 1}, {"gamma": P + 2}, {"beta": P + 1}, {"mean": P + 2}, {"rstd": P + 2},
    {"ws": P + 8}, {"seg": P + 2}, {"n_seg": 1 << 27},
])
def test_group_norm_act_fwd_refuses(change):
    assert call("group_norm_act_fwd", FWD_NORM, **change) == EINVAL


BWD_NORM = dict(dtype=1, X=P, ldx=24, G=P, ldg=24, seg=P, n_seg=4, max_rows=0, m=100, C=24, groups=3, gamma=P, beta=P, act=1, mean=P, rstd=P, dX=P,
                lddx=24, dgamma=P, dbeta=P, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [
    {"dtype": -1}, {"n_seg": 0}, {"max_rows": -5}, {"m": -1}, {"C": 25, "ldx": 25, "ldg": 25, "lddx": 25}, {"groups": 0}, {"act": 9}, {"ldx": 1},
    {"ldg": 23}, {"lddx": 23}, {"X": None}, {"G": None}, {"dX": None}, {"mean": None}, {"rstd": None}, {"ws": None}, {"seg": None, "n_seg": 3},
    {"G": P + 1}, {"dX": P + 1}, {"dgamma": P + 2}, {"dbeta": P + 2}, {"ws": P + 4},
])
def test_group_norm_act_bwd_refuses(change):
    assert call("group_norm_act_bwd", BWD_NORM, **change) == EINVAL


def test_group_norm_needs_its_workspace():
    b = ctypes.c_size_t(0)
    query = sagnn.lib().group_norm_workspace_bytes
    good = dict(dtype=0, m=500_000, n_seg=4, max_rows=0, C=24, groups=3, ld=24, backward=0)

    def size(**change):
        assert query(*{**good, **change}.values(), ctypes.byref(b)) == 0
        return b.value

    assert call("group_norm_act_fwd", FWD_NORM, m=500_000, ws_bytes=size() - 1) == ECAPACITY
    assert call("group_norm_act_fwd", FWD_NORM, m=500_000, ws=None) == EINVAL
    assert size(backward=1) > size() > 0
    assert call("group_norm_act_bwd", BWD_NORM, m=500_000, ws_bytes=size(dtype=1, backward=1) - 1) == ECAPACITY
    # short segments: none forward, gamma's and beta's sums backward; what lies far apart goes the other way
    assert size(max_rows=100) == 0 and size(max_rows=100, backward=1) > 0 and size(max_rows=100, ld=1 << 20) > 0
    assert call("group_norm_act_bwd", BWD_NORM, m=500_000, max_rows=100, ws_bytes=size(dtype=1, backward=1, max_rows=100) - 1) == ECAPACITY
    for bad in ({"m": -1}, {"n_seg": 0}, {"C": 25}, {"groups": 0}, {"C": 0}, {"dtype": 2}, {"max_rows": -1}, {"ld": 23}, {"backward": 2}):
        assert query(*{**good, **bad}.values(), ctypes.byref(b)) == EINVAL, bad
    assert query(*good.values(), None) == EINVAL


def grad_rows(*rows):
    return np.array(rows, dtype=np.int64)


def test_clipping_refuses():
    good = grad_rows([P, P, 100, 0])

    def clip(rows, n=None, max_norm=1.0, norm=P, ws=P, ws_bytes=1 << 30):
        return binding._calls().grad_clip_norm(rows, len(rows) if n is None else n, max_norm, norm, ws, ws_bytes, None)

    for max_norm in (0.0, -1.0, float("nan"), float("inf")):
        assert clip(good, max_norm=max_norm) == EINVAL
        assert binding._calls().grad_scale_to_norm(good, 1, max_norm, P, None) == EINVAL
    assert clip(None, n=1) == EINVAL and clip(good, n=-1) == EINVAL and clip(good, n=65537) == EINVAL
    assert clip(good, norm=None) == EINVAL and clip(good, ws=None) == EINVAL and clip(good, norm=P + 2) == EINVAL and clip(good, ws=P + 4) == EINVAL
    assert clip(good, ws_bytes=8) == ECAPACITY
    assert binding._calls().grad_scale_to_norm(good, 1, 1.0, None, None) == EINVAL
    for row in ([0, P, 9, 0], [P, 0, 9, 0], [P, P, -1, 0], [P, P, 9, 2], [P, P, 9, -1], [P + 2, P, 9, 0], [P, P + 2, 9, 0], [P + 1, P, 9, 1],
                [P, P, 1 << 50, 0]):
        assert clip(grad_rows(row)) == EINVAL, row
    assert clip(grad_rows([1 << 48, 1 << 48, 9, 0])) == EINVAL and clip(grad_rows([P, 1 << 48, 9, 0])) == EINVAL
    # what is written is shared: a tensor twice, one inside another, an output over another's input, over half of its own
    for rows in ([[P, P, 10, 0], [P, P, 10, 0]], [[P, P, 1000, 0], [P + 8, P + 8, 10, 0]], [[P, P, 10, 0], [P + 400, P + 36, 10, 0]],
                 [[P, P + 4, 10, 0]], [[P, P + (1 << 16), 10, 1], [P + 64, P + (1 << 16) + 18, 10, 1]],
                 [[P + 4096 * i, P + 4096 * i, 1000, 0] for i in range(300)] + [[P + 4096 * 7 + 3996, P + (1 << 24), 30, 0]]):
        assert clip(grad_rows(*rows)) == EINVAL, rows[-2:]
    assert binding._calls().grad_global_norm(grad_rows([0, 0, 9, 0]), 1, P, P, 1 << 30, None) == EINVAL
    assert binding._calls().grad_global_norm(good, 1, None, P, 1 << 30, None) == EINVAL
    assert binding._calls().grad_global_norm(good, 1, P, P, 8, None) == ECAPACITY
    b = ctypes.c_size_t(0)
    assert sagnn.lib().grad_norm_workspace_bytes(-1, ctypes.byref(b)) == EINVAL and sagnn.lib().grad_norm_workspace_bytes(5, None) == EINVAL


def test_the_binding_refuses_what_is_not_on_the_gpu():
    x, w, off = torch.zeros(4, 8), torch.zeros(1, 8, 8), torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError):
        sagnn.grouped_gemm_act(x, w, off)
    with pytest.raises(ValueError):
        sagnn.grouped_gemm_bwd(x, w, off, x)
    with pytest.raises(ValueError):
        sagnn.group_norm_act(x, 2)
    with pytest.raises(ValueError):
        sagnn.group_norm_act_bwd(x, x, torch.zeros(1, 2), torch.zeros(1, 2), 2)
    with pytest.raises(ValueError):
        sagnn.grad_clip_norm([x], 1.0)
    with pytest.raises(ValueError):
        sagnn.grad_global_norm([x])


def test_storage_types_and_activations_match_the_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sagnn.h")).read()
    defs = {k: int(v) for k, v in re.findall(r"#define\s+(SAGNN_[A-Z0-9_]+)\s+(\d+)\b", text)}
    assert (defs["SAGNN_F32"], defs["SAGNN_BF16"], defs["SAGNN_ACT_SILU"]) == (binding.F32, binding.BF16, sagnn.ACT_SILU)
