"""Rows of 8 bits, bit by bit: the norm's own fp32 rows, divided by the scale in 32 bits and rounded to nearest even."""
import pytest
import torch

import paper_2504_04673_amd as sagnn
from tests.test_gpu_row_operators import gen, normal

pytestmark = pytest.mark.gpu


def codes(Y, scale):
    """A quotient of 32 bits is that of 64 rounded to 32: twice and two bits more hold every quotient apart from the middle between two."""
    q = (Y.double() / scale.double()[:, None]).float()
    q = torch.where(scale[:, None] > 0, q, Y * 0.0)
    return q.clamp(-448.0, 448.0).cpu().to(torch.float8_e4m3fn).view(torch.uint8)


@pytest.mark.parametrize("m,c", [(20000, 1000), (4096, 4096), (3000, 7001), (5, 13)])
@pytest.mark.parametrize("residual", [False, True])
def test_codes(m, c, residual):
    g = gen(m + c)
    X, gamma = normal(g, m, c) * torch.rand((m, 1), generator=g, device="cuda") * 100.0, 1.0 + normal(g, c, scale=0.3)
    R = normal(g, m, c) if residual else None
    Y, _, _ = sagnn.rms_norm(X, gamma, residual=R)
    Q, scale, _, _ = sagnn.rms_norm_e4m3(X, gamma, residual=R)
    assert torch.equal(scale, (Y.abs().amax(1).double() / 448.0).float())
    assert torch.equal(Q.view(torch.uint8).cpu(), codes(Y, scale))


def test_codes_at_the_middle_between_two():
    """Values in the middle between two of 8 bits, and the next of 32 bits to either side, under scales that are no power of two."""
    values = torch.arange(1, 127, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    middle = torch.cat([(values[1:] + values[:-1]) / 2, values[:1] / 2, torch.full((1,), 448.0, device="cuda")])
    scales = 2.0 ** torch.linspace(-3.0, 3.0, 4000, device="cuda")
    near = middle * scales[:, None]
    X = torch.cat([near, torch.nextafter(near, torch.full_like(near, 1e9)), torch.nextafter(near, torch.zeros_like(near)), -near], 1)
    X[:, -1] = -near[:, -1]
    # (gamma takes the norm off again, up to rounding: what counts is that the codes are those of its own rows)
    gamma = torch.full((X.shape[1],), 100.0, device="cuda")
    Y, _, _ = sagnn.rms_norm(X, gamma, eps=0.0)
    Q, scale, _, _ = sagnn.rms_norm_e4m3(X, gamma, eps=0.0)
    assert torch.equal(Q.view(torch.uint8).cpu(), codes(Y, scale))


@pytest.mark.parametrize("size", [2.0 ** -120, 2.0 ** -95, 2.0 ** -90, 2.0 ** -60, 1e30, 3e36])
def test_codes_of_small_and_large_rows(size):
    """Scales down to the smallest and up to the largest, through gamma; and rows with an infinite scale."""
    g = gen(5)
    X, gamma = normal(g, 6000, 512), (0.5 + torch.rand(512, generator=g, device="cuda")) * size
    Y, _, _ = sagnn.rms_norm(X, gamma)
    Q, scale, _, _ = sagnn.rms_norm_e4m3(X, gamma)
    assert torch.equal(Q.view(torch.uint8).cpu(), codes(Y, scale))
    gamma[7] = float("inf")
    Q, scale, _, _ = sagnn.rms_norm_e4m3(X, gamma)
    assert scale.isinf().all() and Q[:, 7].float().isnan().all() and not Q[:, :7].float().any() and not Q[:, 8:].float().any()
