"""What the header says of the cross entropy's workspace and of its limits."""
import ctypes

import pytest

import paper_2504_04673_amd as sagnn
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
