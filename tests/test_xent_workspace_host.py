"""What the header says of the cross entropy's workspace and of its limits."""
import ctypes

import pytest
import torch

import paper_2504_04673_amd as sagnn
from paper_2504_04673_amd import binding
from tests.test_row_operators_host import EINVAL


def size(*args):
    b = ctypes.c_size_t(0)
    rc = sagnn.lib().softmax_xent_workspace_bytes(*args, ctypes.byref(b))
    return b.value if rc == 0 else rc


def piece(m, n, width):
    """Classes of a piece, as documented; `width` bytes a value."""
    least = 1024 if m * width * 1024 <= 4 << 30 else 256
    most = max(least, min((512 << 20) // (m * width) // 256 * 256, 32768), -(-n // 384))
    pieces = -(-n // most)
    return n if pieces == 1 else -(-(-(-n // pieces)) // 256) * 256


@pytest.mark.parametrize("m,n", [(100, 24), (5000, 100_000), (100_000, 47), (1_000_000, 2_000_000), (100_000, 16_000_000), (2_200_000, 1200), (1_000_000, 5000), (30_000, 16_777_216)])
@pytest.mark.parametrize("dtype,width", [(0, 4), (1, 2)])
def test_backward_is_p_of_a_piece_and_little_else_where_features_are_narrow(dtype, width, m, n):
    k, classes = 8, piece(m, n, width)
    got, p = size(dtype, m, k, n, 0, 1), m * -(-classes // 8) * 8 * width * (2 if dtype == 1 and m <= 1024 else 1)
    # copies of H, 1 and 2; sums of dH, 32 shares at most; the bias's of a tile of 32 rows; the list; dW of a piece in 512 parts and two at the most, twice
    rest = 3 * 2 * m * k * width + 32 * 2 * m * k * 4 + (m + 31) // 32 * classes * 4 + 8 * m + 2 * 1030 * 2 * k * (classes + 8) * 4 + (1 << 16)
    assert p <= got <= p + rest


@pytest.mark.parametrize("m,n", [(100, 5000), (8192, 131072), (3, 16_777_216)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_forward_is_eight_bytes_a_row_and_tile(dtype, m, n):
    got = size(dtype, m, 64, n, 0, 0)
    assert m * (8 * -(-n // 256) + 4) <= got <= m * (8 * -(-n // 32) + 4) + 512


def test_joint_limit():
    """4096 by 524288 tiles of 32 are 2^31."""
    assert size(1, 131_072, 8, 16_777_216, 0, 0) == EINVAL and size(1, 131_072 - 32, 8, 16_777_216, 0, 0) > 0
    assert size(0, 131_072, 8, 16_777_216, 0, 1) == EINVAL


@pytest.mark.parametrize("dtype,prec", [(1, 0), (0, 0), (0, 1), (0, 2)])
@pytest.mark.parametrize("m,k,n", [(2_000_000, 602, 47), (8192, 1024, 131_072), (700, 64, 300), (1, 8, 2), (0, 8, 5)])
def test_calls_without_weights_need_no_room_for_weighted_rows(dtype, prec, m, k, n):
    def one(weighted):
        b = ctypes.c_size_t(0)
        assert sagnn.lib().softmax_xent_bwd_workspace_bytes(dtype, m, k, n, prec, weighted, ctypes.byref(b)) == 0
        return b.value

    assert size(dtype, m, k, n, prec, 1) == max(one(0), one(1))
    low = dtype == 1 or prec == 1
    if low and m > 1024:
        # two copies of H in rows of whole eights
        assert one(1) >= one(0) + 2 * m * -(-k // 8) * 8 * (2 if dtype == 1 else 4)
    elif not low:
        assert one(0) == one(1)
    b = ctypes.c_size_t(0)
    query = sagnn.lib().softmax_xent_bwd_workspace_bytes
    assert query(dtype, m, k, n, prec, 2, ctypes.byref(b)) == EINVAL and query(dtype, -1, k, n, prec, 0, ctypes.byref(b)) == EINVAL
    assert query(dtype, m, k, n, prec, 0, None) == EINVAL


def test_the_binding_asks_for_what_its_call_needs(monkeypatch):
    """The library refuses a call with a byte less (tests of refusals); with weights, and without, it is asked which."""
    asked = []
    monkeypatch.setattr(binding, "_xent_args", lambda *a: (2_000_000, 602, 47, (1, 0, 602, 0, 47, 0, None, 0)))

    def ask(*args):
        asked.append(args)
        raise LookupError

    monkeypatch.setattr(binding, "_bytes_of", ask)
    for grad, weighted in ((1.0, 0), (torch.zeros(3), 1)):
        with pytest.raises(LookupError):
            binding.softmax_xent_bwd(None, None, None, None, grad)
        assert asked.pop() == ("softmax_xent_bwd_workspace_bytes", 1, 2_000_000, 602, 47, sagnn.GEMM_FP32, weighted)
