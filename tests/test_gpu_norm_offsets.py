"""Group norm of values whose mean is far from zero against their deviation, or that are all equal.

mean and rstd are computed in 64 bits from values taken relative to one of them and rounded once: 2 and 8 times 2^-24.  y: mean is
rounded to 2^-24 of itself before it is taken off, then two operations on what is left: 2^-24 |mean| rstd |gamma| + 2^-21 of
|x - mean| rstd |gamma| + |beta|."""
import pytest
import torch

import paper_2504_04673_amd as sagnn

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
FORMS = [(40, 40), (40, 0), (700, 1), (20000, 0), (600000, 0)]      # rows, max_rows: whole segments, longer than said, parts, many parts


def call(X, groups, gamma, beta, seg, known, act, in_place):
    X = X.clone() if in_place else X
    return sagnn.group_norm_act(X, groups, gamma, beta, seg=seg, max_rows=known, act=act, out=X if in_place else None)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows,known", FORMS)
@pytest.mark.parametrize("dtype,c,groups", [(torch.float32, 16, 2), (torch.float32, 6, 2), (torch.float32, 15, 15), (torch.bfloat16, 16, 2)])
def test_equal_values_give_beta(rows, known, dtype, c, groups, in_place):
    """Mean is the value and y is beta, to the last bit; so ReLU's slope is decided by beta alone."""
    seg = torch.tensor([0, rows, rows + 1, rows + 9], dtype=torch.int32, device="cuda")
    values = torch.tensor([3.7, -1e6, 1 / 3], device="cuda").to(dtype)
    X = values.repeat_interleave(seg.diff())[:, None].expand(-1, c).contiguous()
    gamma, beta = torch.full((c,), 1.7, device="cuda"), torch.zeros(c, device="cuda")
    for b in (0.0, 0.3):
        beta.fill_(b)
        Y, mean, rstd = call(X, groups, gamma, beta, seg, known, sagnn.ACT_IDENTITY, in_place)
        assert torch.equal(mean, values.float()[:, None].expand(3, groups)) and bool((Y == beta.to(dtype)).all())
        assert bool(((rstd - 1e-5 ** -0.5).abs() <= 4 * U * 1e-5 ** -0.5).all())
    _, dgamma, dbeta = sagnn.group_norm_act_bwd(X, torch.ones_like(X), mean, rstd, groups, gamma, torch.zeros_like(beta), seg=seg, max_rows=known,
                                                act=sagnn.ACT_RELU)
    assert not dgamma.any() and not dbeta.any()              # (z is 0 everywhere, where ReLU is flat)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("far", [1e3, 1e5, -1e6])
@pytest.mark.parametrize("rows,known", FORMS)
@pytest.mark.parametrize("c,groups", [(16, 2), (6, 2), (15, 15)])
def test_mean_far_from_zero(rows, known, far, c, groups, in_place):
    g = torch.Generator(device="cuda").manual_seed(rows)
    X = torch.randn(rows + 9, c, generator=g, device="cuda") + far
    X[rows:] -= 3 * far                                       # (a segment of its own)
    gamma, beta = torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda")
    seg = torch.tensor([0, rows, rows + 9], dtype=torch.int32, device="cuda")
    Y, mean, rstd = call(X, groups, gamma, beta, seg, known, sagnn.ACT_IDENTITY, in_place)
    for b, (lo, hi) in enumerate([(0, rows), (rows, rows + 9)]):
        x = X[lo:hi].double().view(hi - lo, groups, -1)
        mu = x.mean((0, 2), keepdim=True)
        rs = ((x - mu).square().mean((0, 2), keepdim=True) + 1e-5).rsqrt()
        assert bool(((mean[b] - mu.flatten()).abs() <= 2 * U * mu.abs().flatten()).all())
        assert bool(((rstd[b] - rs.flatten()).abs() <= 8 * U * rs.flatten()).all())
        ga, be = gamma.double().view(groups, -1), beta.double().view(groups, -1)
        xh = (x - mu) * rs
        bound = U * mu.abs() * rs * ga.abs() + 8 * U * (xh.abs() * ga.abs() + be.abs()) + 1e-30
        assert bool(((Y[lo:hi].view_as(x) - (xh * ga + be)).abs() <= bound).all())


def test_first_value_far_from_the_others():
    """The value that the sums are taken from is itself 10^6 deviations of the others away."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for rows, known in FORMS:
        X = torch.randn(rows, 8, generator=g, device="cuda")
        X[0, 0] = 1e6
        seg = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
        _, mean, rstd = sagnn.group_norm_act(X, 1, seg=seg, max_rows=known)
        x = X.double()
        rs = (x.var(correction=0) + 1e-5).rsqrt()
        assert abs(float(mean) - float(x.mean())) <= 2 * U * abs(float(x.mean())) and abs(float(rstd) - float(rs)) <= 8 * U * float(rs)


@pytest.mark.parametrize("rows,known", FORMS)
def test_first_value_that_is_not_finite(rows, known):
    """An infinite value makes the mean infinite, a NaN makes it one, wherever in the segment it stands."""
    for value in (float("inf"), float("-inf"), float("nan")):
        for at in (0, rows // 2):
            X = torch.ones(rows, 4, device="cuda")
            X[at, 1] = value
            Y, mean, rstd = sagnn.group_norm_act(X, 2, seg=torch.tensor([0, rows], dtype=torch.int32, device="cuda"), max_rows=known)
            assert mean[0, 0].isnan() if value != value else mean[0, 0] == value
            assert rstd[0, 0].isnan() and bool(Y[:, :2].isnan().all()) and mean[0, 1] == 1.0 and not Y[:, 2:].any()
