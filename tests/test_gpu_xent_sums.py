"""The cross entropy's sums over very many classes: their error does not grow with the classes.

Tolerance of lse (u = 2^-24): sums of positive terms 64 u in a tile, the tiles' in 64 bits, rounded once; an exponential 2^-23 (1 + |x|) of itself, in a tile and again
between tiles, which counts as much as its share of the sum; a logarithm and its addition 2^-22 + 2 u |lse|; z's own error, 0 here.
"""
import pytest
import torch

import paper_2504_04673_amd as sagnn
from tests.test_gpu_row_operators import gen

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def check(bias, m, dtype, trans):
    """Features of zeros: the logits are the bias."""
    n, k = bias.numel(), 8
    W = torch.zeros((n, k) if trans else (k, n), dtype=dtype, device="cuda")
    H = torch.zeros(m, k, dtype=dtype, device="cuda")
    labels = torch.arange(m, dtype=torch.int32, device="cuda") * 7 % n
    loss, lse = sagnn.softmax_xent(H, W, labels, bias=bias, transW=trans)
    z = bias.double()
    ref = torch.logsumexp(z, 0)
    far = float((torch.exp(z - ref) * (2 + 2 * (z - z.max()).abs())).sum())
    bound = 65 * U + 2.0 ** -23 * far + 2.0 ** -22 + 2 * U * abs(float(ref))
    assert float((lse.double() - ref).abs().max()) <= bound
    assert float((loss.double() - (ref - z[labels.long()])).abs().max()) <= bound + U * float((ref - z[labels.long()]).abs().max())


@pytest.mark.parametrize("dtype,trans", [(torch.float32, False), (torch.bfloat16, True)], ids=["fp32", "bf16"])
@pytest.mark.parametrize("m,n", [(1, 16_777_216), (3, 4_000_003), (5, 1_000_000), (33, 262_144), (20, 60_000), (3, 130), (70, 1)])
def test_equal_classes_below_one(m, n, dtype, trans):
    bias = torch.full((n,), -1.0 / 3.0, device="cuda")
    check(bias, m, dtype, trans)
    for top in (0.1, 0.77, 1.9, 2.7, 3.9):       # (which decides how the sums of the others lie between values of 32 bits)
        for places in (slice(0, 1), slice(0, 8192, 32), slice(n - 1, n)):       # one larger class in the first tile, in each of the first, in the last
            bias.fill_(-1.0 / 3.0)
            bias[places] = top
            check(bias, m, dtype, trans)


@pytest.mark.parametrize("m,n", [(1, 3_000_000), (17, 300_000)])
def test_classes_in_order(m, n):
    """Logits that rise a little from each class to the next, so that every tile has a new maximum; and that fall; and at random."""
    bias = torch.linspace(-4.0, 4.0, n, device="cuda")
    check(bias, m, torch.float32, True)
    check(bias.flip(0).contiguous(), m, torch.float32, True)
    check(torch.randn(n, generator=gen(n), device="cuda") * 3.0, m, torch.bfloat16, True)
