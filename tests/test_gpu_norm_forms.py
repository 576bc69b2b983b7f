"""Both forms of group norm where they are least at home: whole segments longer than the caller said, and segments in parts with many
groups.  max_rows only chooses between forms, so every value of it gives the same results.

Tolerances: mean and rstd to 2 and 8 times 2^-24; y to 2^-20 of |x - mean| rstd |gamma| + |mean| rstd |gamma| + |beta| (SiLU: slope below 1.1, an
exponential good to (4 + |z|) 2^-22); gradients to 1e-5 of the sum of the absolute values of their terms, grown by 1 + |mean| rstd for the
rounding of mean, SiLU's slope known to the error of z; bfloat16 results are rounded once more, by 2^-8."""
import ctypes

import pytest
import torch

import paper_2504_04673_amd as sagnn
from paper_2504_04673_amd import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F, B = torch.float32, torch.bfloat16


def workspace(X, n_seg, max_rows, groups, backward):
    b = ctypes.c_size_t(0)
    m, c = X.shape
    assert sagnn.lib().group_norm_workspace_bytes(binding._DTYPE[X.dtype], m, n_seg, max_rows, c, groups, c, backward, ctypes.byref(b)) == 0
    return b.value


def in_parts(X, n_seg, max_rows, groups, backward):
    """Whether the call goes by parts: whole segments need no workspace forward, a row of sums for each (2048 at most) backward."""
    rows = min(n_seg, 2048)
    whole = -(-rows * X.shape[1] * 8 // 256) * 256 if backward and rows > 1 else 0
    return workspace(X, n_seg, max_rows, groups, backward) != whole


def inputs(sizes, c, dtype, act, groups, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda") * scale

    seg = torch.tensor([0, *torch.tensor(sizes).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
    m = int(seg[-1]) + 5
    X = (normal(m, c) * (0.5 + torch.rand(c, generator=g, device="cuda")) + normal(c, scale=2.0)).to(dtype)
    G, gamma, beta = normal(m, c).to(dtype), 1.0 + normal(c, scale=0.3), normal(c, scale=0.3)
    if act == sagnn.ACT_RELU:                                 # nothing where ReLU's slope could go either way
        G[reference(X, G, groups, gamma, beta, seg, 0)["z"].abs() <= 1e-3] = 0.0
    X[m - 5:], G[m - 5:] = float("nan"), float("inf")         # (rows behind the last segment: not used)
    return seg, X, G, gamma, beta


def reference(X, G, groups, gamma, beta, seg, act, eps=1e-5):
    """Results in 64 bits and the scale of each one's error."""
    (m, c), o, n_seg = X.shape, seg.tolist(), seg.numel() - 1
    ga, be = gamma.double().view(groups, -1), beta.double().view(groups, -1)
    r = {k: torch.zeros(m, c, dtype=torch.float64, device="cuda") for k in ("z", "y", "y_", "dx", "dx_")}
    r.update({k: torch.zeros(groups, c // groups, dtype=torch.float64, device="cuda") for k in ("dgamma", "dgamma_", "dbeta", "dbeta_")})
    r["mean"] = torch.zeros(n_seg, groups, dtype=torch.float64, device="cuda")
    r["rstd"] = torch.full_like(r["mean"], eps ** -0.5)
    for b in range(n_seg):
        lo, hi = o[b], o[b + 1]
        if lo == hi:
            continue
        x, h = (t[lo:hi].double().view(hi - lo, groups, -1) for t in (X, G))
        mu = x.mean((0, 2), keepdim=True)
        rs = ((x - mu).square().mean((0, 2), keepdim=True) + eps).rsqrt()
        r["mean"][b], r["rstd"][b] = mu.flatten(), rs.flatten()
        xh = (x - mu) * rs
        z = xh * ga + be
        sig = torch.sigmoid(z)
        size = (xh.abs() + mu.abs() * rs) * ga.abs() + be.abs()
        slope = (torch.ones_like(z), (z > 0).double(), sig * (1 + z * (1 - sig)))[act]
        put = lambda name, t: r[name][lo:hi].copy_(t.reshape(hi - lo, c))
        put("z", z)
        put("y", (z, z.clamp(min=0.0), z * sig)[act])
        put("y_", 16 * U * size * (1.1 if act == 2 else 1.0) + (4 * U * (4 + z.abs()) * z.abs() if act == 2 else 0.0))
        grow = 1 + mu.abs() * rs
        hs = (h * slope).abs() + (h.abs() * (size + 1) if act == 2 else 0.0)
        h = h * slope
        r["dgamma"] += (h * xh).sum(0)
        r["dbeta"] += h.sum(0)
        r["dgamma_"] += (hs * (xh.abs() + 1) * grow).sum(0)
        r["dbeta_"] += (hs * grow).sum(0)
        h, hs = h * ga, hs * ga.abs()
        put("dx", rs * (h - h.mean((0, 2), keepdim=True) - xh * (h * xh).mean((0, 2), keepdim=True)))
        put("dx_", rs * grow * (hs + hs.mean((0, 2), keepdim=True) + (xh.abs() + 1) * (hs * (xh.abs() + 1)).mean((0, 2), keepdim=True)))
    return r


def close(got, ref, bound, what):
    bad = ~((got.double().reshape(ref.shape) - ref).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off"


def check(seg, X, G, gamma, beta, groups, act, known, in_place):
    r, n = reference(X, G, groups, gamma, beta, seg, act), int(seg[-1])
    rounding = 1.01 * 2.0 ** -8 if X.dtype is B else 0.0
    kw = dict(seg=seg, max_rows=known, act=act)
    xs, gs = X.clone(), G.clone()
    Y, mean, rstd = sagnn.group_norm_act(xs, groups, gamma, beta, out=xs if in_place else None, **kw)
    close(mean, r["mean"], 2 * U * r["mean"].abs() + 1e-12, "mean")
    close(rstd, r["rstd"], 8 * U * r["rstd"], "rstd")
    close(Y[:n], r["y"][:n], r["y_"][:n] + rounding * r["y"][:n].abs() + 1e-30, "y")
    dX, dgamma, dbeta = sagnn.group_norm_act_bwd(X, gs, mean, rstd, groups, gamma, beta, out=gs if in_place else None, **kw)
    close(dX[:n], r["dx"][:n], 1e-5 * r["dx_"][:n] + rounding * r["dx"][:n].abs() + 1e-30, "dx")
    close(dgamma, r["dgamma"], 1e-5 * r["dgamma_"] + 1e-30, "dgamma")
    close(dbeta, r["dbeta"], 1e-5 * r["dbeta_"] + 1e-30, "dbeta")
    assert not Y[n:].any() and not dX[n:].any()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("known", [1, 20, 513, 0])
@pytest.mark.parametrize("c,groups", [(16, 2), (30, 2), (36, 4), (64, 8), (256, 32), (602, 7), (7, 7)])
def test_segments_longer_than_the_caller_said(c, groups, known, dtype, in_place):
    sizes = [513, 3, 0, 2100, 1, 900]
    for act in (sagnn.ACT_IDENTITY, sagnn.ACT_RELU, sagnn.ACT_SILU):
        seg, X, G, gamma, beta = inputs(sizes, c, dtype, act, groups, c + act)
        if known == 1:                                        # (the form that keeps rows in registers, with up to 2100 of them)
            assert not in_parts(X, len(sizes), known, groups, 0) and not in_parts(X, len(sizes), known, groups, 1)
        check(seg, X, G, gamma, beta, groups, act, known, in_place)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("sizes", [[4000, 0, 1500], [1200] + [1, 0, 2] * 30 + [2500]], ids=["few", "many"])
@pytest.mark.parametrize("c,groups", [(1000, 250), (1024, 1024), (4096, 1024), (16384, 4), (528, 44), (1030, 515)])
def test_parts_of_many_groups(c, groups, sizes, dtype, in_place):
    for act in (sagnn.ACT_RELU, sagnn.ACT_SILU):
        seg, X, G, gamma, beta = inputs(sizes, c, dtype, act, groups, c + act)
        assert in_parts(X, len(sizes), 0, groups, 0) and in_parts(X, len(sizes), 0, groups, 1)
        check(seg, X, G, gamma, beta, groups, act, 0, in_place)


@pytest.mark.parametrize("dtype", [F, B])
def test_gradient_along_directions_that_the_group_takes_out(dtype):
    """A segment and group moved as a whole, or stretched about its mean, has the same result: the gradient along both is nothing but
    rounding and eps.  (Without its two means it would be of the order of the sum of |dx|.)"""
    for rows, known in ((30, 30), (4000, 0), (900, 1)):
        seg, X, G, gamma, beta = inputs([rows, rows // 3], 32, dtype, sagnn.ACT_SILU, 4, rows)
        _, mean, rstd = sagnn.group_norm_act(X, 4, gamma, beta, seg=seg, max_rows=known, act=sagnn.ACT_SILU)
        dX, _, _ = sagnn.group_norm_act_bwd(X, G, mean, rstd, 4, gamma, beta, seg=seg, max_rows=known, act=sagnn.ACT_SILU)
        for b, (lo, hi) in enumerate([(0, rows), (rows, rows + rows // 3)]):
            d, x = (t[lo:hi].double().view(hi - lo, 4, -1) for t in (dX, X))
            xh = (x - mean[b].double()[:, None]) * rstd[b].double()[:, None]
            total = d.abs().sum((0, 2))
            # each value rounded by 2^-9 (bfloat16), errors of either sign: 4 deviations of their sum; fp32: 1e-5 of the sum
            noise = lambda w: 1e-5 * (d.abs() * w).sum((0, 2)) * 4 + (4 * 2.0 ** -9 * (d * w).square().sum((0, 2)).sqrt() if dtype is B else 0.0)
            assert bool((d.sum((0, 2)).abs() <= noise(1.0)).all()) and bool((total > 100 * noise(1.0)).all() if dtype is F else True)
            # stretching: eps keeps 1e-5 rstd^2 of it
            left = (d * xh).sum((0, 2)).abs()
            assert bool((left <= noise(xh.abs()) + 4e-5 * rstd[b].double().square() * (d.abs() * xh.abs()).sum((0, 2))).all())


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("rows,known", [(40, 40), (700, 1), (4000, 0)])
def test_gradients_that_are_not_finite_where_relu_is_flat(rows, known, value, dtype):
    """0 times an infinity is a NaN: an overflow in the gradient is not hidden by ReLU."""
    seg, X, G, gamma, beta = inputs([rows, 30], 16, dtype, sagnn.ACT_RELU, 4, rows)
    z = reference(X, G, 4, gamma, beta, seg, 0)["z"]
    at = int((z[:rows, 5] < -0.5).nonzero()[0])
    G[at, 5] = value
    _, mean, rstd = sagnn.group_norm_act(X, 4, gamma, beta, seg=seg, max_rows=known, act=sagnn.ACT_RELU)
    dX, dgamma, dbeta = sagnn.group_norm_act_bwd(X, G, mean, rstd, 4, gamma, beta, seg=seg, max_rows=known, act=sagnn.ACT_RELU)
    bad = torch.zeros(X.shape, dtype=torch.bool, device="cuda")
    bad[:rows, 4:8] = True
    assert torch.equal(dX.isnan(), bad)
    for t in (dgamma, dbeta):
        assert torch.equal(t.isnan(), torch.arange(16, device="cuda") == 5)
