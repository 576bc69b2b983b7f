"""Refusals of the softmax cross entropy, which need no GPU."""
import ctypes

import pytest
import torch

import paper_2504_04673_amd as sagnn
from tests.test_row_operators_host import A, ECAPACITY, EINVAL, P, call

FWD = dict(dtype=0, H=P, ldh=16, W=2 * A, ldw=24, transW=0, bias=P, labels=P, m=100, kdim=16, n=24, prec=0, loss=3 * A, lse=4 * A, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [
    {"dtype": 2}, {"dtype": -1}, {"dtype": 1, "prec": 1}, {"dtype": 1, "prec": 2}, {"prec": 3}, {"prec": -1}, {"transW": 2}, {"transW": -1}, {"m": -1}, {"m": 1 << 31}, {"kdim": 0},
    {"kdim": 65537, "ldh": 65537}, {"n": 0}, {"n": 16777217, "ldw": 16777217}, {"m": 2000000000, "n": 16777216, "ldw": 16777216}, {"ldh": 15}, {"ldw": 23}, {"transW": 1, "ldw": 15},
    {"H": None}, {"W": None}, {"labels": None}, {"loss": None}, {"lse": None}, {"H": P + 2}, {"W": P + 1}, {"bias": P + 2}, {"labels": P + 2}, {"loss": 3 * A + 1}, {"lse": P + 2},
    {"ws": P + 8}, {"loss": 4 * A + 396}, {"lse": P}, {"loss": 2 * A + 1532}, {"n": 40000, "ldw": 40000, "ws": None},
])
def test_softmax_xent_fwd_refuses(change):
    assert call("softmax_xent_fwd", FWD, **change) == EINVAL


BWD = dict(dtype=1, H=P, ldh=16, W=2 * A, ldw=24, transW=0, bias=P, labels=P, lse=P, grad=P, grad_all=1.0, m=100, kdim=16, n=24, prec=0, dH=3 * A, lddh=16, dW=4 * A, dbias=5 * A,
           ws=6 * A, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [
    {"dtype": 2}, {"prec": 1}, {"transW": 3}, {"m": -1}, {"kdim": 0}, {"n": 0}, {"ldh": 15}, {"ldw": 23}, {"lddh": 15}, {"H": None}, {"W": None}, {"labels": None}, {"lse": None},
    {"H": P + 1}, {"dH": 3 * A + 1}, {"dW": 4 * A + 1}, {"dbias": 5 * A + 2}, {"lse": P + 2}, {"grad": P + 1}, {"ws": None}, {"ws": 6 * A + 8}, {"dH": P}, {"dH": 4 * A + 767},
    {"dW": 2 * A}, {"dbias": 4 * A + 764}, {"dbias": P + 92},
])
def test_softmax_xent_bwd_refuses(change):
    assert call("softmax_xent_bwd", BWD, **change) == EINVAL


def test_softmax_xent_needs_its_workspace():
    b = ctypes.c_size_t(0)
    query = sagnn.lib().softmax_xent_workspace_bytes

    def size(*args):
        assert query(*args, ctypes.byref(b)) == 0
        return b.value

    assert size(0, 100, 16, 24, 0, 0) == 0                   # one tile of columns: no join
    need = size(0, 100, 16, 5000, 0, 0)
    assert need > 0 and call("softmax_xent_fwd", FWD, n=5000, ldw=5000, ws_bytes=need - 1) == ECAPACITY
    need = size(1, 100, 16, 24, 0, 1)
    assert call("softmax_xent_bwd", BWD, ws_bytes=need - 1) == ECAPACITY
    # pieces of the classes: P for some of them, however many there are
    assert size(1, 8192, 1024, 1 << 20, 0, 1) < 8192 * (1 << 20)
    for args in ((2, 1, 1, 1, 0, 0), (1, 1, 1, 1, 1, 0), (0, -1, 1, 1, 0, 0), (0, 1, 0, 1, 0, 0), (0, 1, 1, 0, 0, 1), (0, 1, 1, 1, 3, 1), (0, 1, 1, 1, 0, 2)):
        assert query(*args, ctypes.byref(b)) == EINVAL
    assert query(0, 1, 1, 1, 0, 0, None) == EINVAL


def test_no_rows_are_done():
    assert call("softmax_xent_fwd", FWD, m=0, H=None, labels=None, loss=None, lse=None) == 0


def test_binding_refuses():
    h, w, y = torch.zeros(4, 8), torch.zeros(8, 5), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="no CPU path"):
        sagnn.softmax_xent(h, w, y)
    with pytest.raises(ValueError, match="no CPU path"):
        sagnn.softmax_xent_bwd(h, w, y, y.float())
