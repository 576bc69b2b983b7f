"""Sizes at the ends of what the grouped products and the norm take: more workgroups than a launch has (2^32 threads), and as
many types as there may be.  What the results have to be is known exactly or to a rounding."""
import pytest
import torch

import paper_2504_04673_amd as sagnn

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def offsets(*places):
    return torch.tensor(places, dtype=torch.int32, device="cuda")


def test_product_of_more_rows_than_a_launch_takes():
    """2^31 - 1 rows of one column: 2^24 tiles of 128 rows and 256 threads."""
    m = (1 << 31) - 1
    X = torch.empty(m, 1, dtype=torch.bfloat16, device="cuda")
    for lo in range(0, m, 1 << 28):
        part = X[lo:lo + (1 << 28)]
        part.copy_(torch.arange(lo, lo + len(part), device="cuda").remainder_(251)[:, None])
    W = torch.tensor([[[2.0]], [[-3.0]]], dtype=torch.bfloat16, device="cuda")
    cut = m - 1000
    off = offsets(0, cut, m - 7)
    for Y in (sagnn.grouped_gemm_act(X, W, off), sagnn.grouped_gemm_bwd(None, W, off, X, want_dw=False)[0]):
        for lo in range(0, m, 1 << 28):
            hi = min(lo + (1 << 28), m)
            rows = torch.arange(lo, hi, device="cuda")[:, None]
            factor = torch.where(rows < cut, 2.0, torch.where(rows < m - 7, -3.0, 0.0))
            assert torch.equal(Y[lo:hi], (X[lo:hi].float() * factor).bfloat16())     # (integers below 2^10, rounded once)
        del Y


def test_joining_the_parts_of_as_many_types_as_there_may_be():
    """65536 types, matrices of 255 x 257: the sums of a cut type are joined in one launch."""
    types, k, n, m = 65536, 255, 257, 2000
    X, G = torch.ones(m, k, device="cuda"), torch.ones(m, n, device="cuda")
    off = torch.full((types + 1,), m - 3, dtype=torch.int32, device="cuda")
    off[0], off[types - 1], off[types] = 0, m - 2, m - 1
    _, dW = sagnn.grouped_gemm_bwd(X, torch.empty(types, k, n, device="cuda"), off, G, want_dx=False)
    rows = off.diff().float()
    assert rows[0] == m - 3 and int((rows > 0).sum()) == 3
    for lo in range(0, types, 4096):
        part = dW[lo:lo + 4096]
        assert torch.equal(part.amin((1, 2)), rows[lo:lo + 4096]) and torch.equal(part.amax((1, 2)), rows[lo:lo + 4096])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_products_of_as_many_types_as_there_may_be(dtype):
    """Integers whose products and sums are exact."""
    types, k, n = 65536, 8, 16
    g = torch.Generator(device="cuda").manual_seed(1)
    sizes = torch.randint(0, 4, (types,), generator=g, device="cuda")
    off = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)]).to(torch.int32)
    m = int(off[-1]) + 5
    kind = torch.repeat_interleave(torch.arange(types, device="cuda"), sizes)

    def whole(*shape):
        return torch.randint(-4, 5, shape, generator=g, device="cuda").to(dtype)

    X, W, G = whole(m, k), whole(types, k, n), whole(m, n)
    Y = sagnn.grouped_gemm_act(X, W, off)
    assert torch.equal(Y[:m - 5].float(), (X[:m - 5, :, None].float() * W[kind].float()).sum(1)) and not Y[m - 5:].any()
    dX, dW = sagnn.grouped_gemm_bwd(X, W, off, G)
    assert torch.equal(dX[:m - 5].float(), (G[:m - 5, None].float() * W[kind].float()).sum(2).to(dtype).float()) and not dX[m - 5:].any()
    ref = torch.zeros(types, k, n, device="cuda").index_add_(0, kind, X[:m - 5, :, None].float() * G[:m - 5, None].float())
    assert torch.equal(dW, ref)


def test_norm_of_more_segments_and_groups_than_a_launch_joins():
    """70,000 segments of two rows by 1024 groups of a channel: 71.7 million pairs, a wavefront for each."""
    segments, c = 70000, 1024
    g = torch.Generator(device="cuda").manual_seed(2)
    X = torch.randn(2 * segments, c, generator=g, device="cuda")
    seg = torch.arange(0, 2 * segments + 1, 2, dtype=torch.int32, device="cuda")
    Y, mean, rstd = sagnn.group_norm_act(X, c, seg=seg, eps=1e-2)
    x = X.view(segments, 2, c)
    for lo in range(0, segments, 10000):
        v = x[lo:lo + 10000].double()
        mu, half = v.mean(1), (v[:, 0] - v[:, 1]) / 2
        rs = (half.square() + 1e-2).rsqrt()
        assert bool(((mean[lo:lo + 10000] - mu).abs() <= 2 * U * mu.abs() + 1e-12).all())
        assert bool(((rstd[lo:lo + 10000] - rs).abs() <= 8 * U * rs).all())
        # mean, rstd and four operations rounded
        bound = 16 * U * (half.abs() + mu.abs()) * rs + 1e-30
        y = Y.view(segments, 2, c)[lo:lo + 10000]
        assert bool(((y[:, 0] - half * rs).abs() <= bound).all()) and bool(((y[:, 1] + half * rs).abs() <= bound).all())
    G = torch.randn(2 * segments, c, generator=g, device="cuda")
    dX, dgamma, dbeta = sagnn.group_norm_act_bwd(X, G, mean, rstd, c, seg=seg)
    sums = torch.zeros(2, c, dtype=torch.float64, device="cuda")
    terms = torch.zeros_like(sums)
    for lo in range(0, segments, 10000):
        v, h = x[lo:lo + 10000].double(), G.view(segments, 2, c)[lo:lo + 10000].double()
        mu, rs = v.mean(1, keepdim=True), rstd[lo:lo + 10000, None].double()
        xh = (v - mu) * rs
        size = (v.abs() + mu.abs()) * rs
        dx = rs * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
        bound = 1e-5 * rs * (h.abs() + h.abs().mean(1, keepdim=True) + size * (h.abs() * size).mean(1, keepdim=True))
        assert bool(((dX.view(segments, 2, c)[lo:lo + 10000] - dx).abs() <= bound).all())
        sums += torch.stack([(h * xh).sum((0, 1)), h.sum((0, 1))])
        terms += torch.stack([(h.abs() * size).sum((0, 1)), h.abs().sum((0, 1))])
    assert bool(((torch.stack([dgamma, dbeta]) - sums).abs() <= 1e-5 * terms).all())


def test_norm_of_as_many_segments_as_there_may_be():
    """2^26 segments of a value, a workgroup for each: mean is the value, y is beta; and rows behind them."""
    n = 1 << 26
    X = torch.arange(n + 100, device="cuda").remainder_(127).to(torch.bfloat16)[:, None]
    seg = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    beta = torch.tensor([1.5], device="cuda")
    Y, mean, rstd = sagnn.group_norm_act(X, 1, None, beta, seg=seg, max_rows=1, eps=0.25)
    assert torch.equal(mean[:, 0], X[:n, 0].float()) and bool((rstd == 2.0).all())
    assert bool((Y[:n] == 1.5).all()) and not Y[n:].any()
    dX, dgamma, dbeta = sagnn.group_norm_act_bwd(X, torch.ones_like(X), mean, rstd, 1, seg=seg, max_rows=1)
    assert not dX.any() and not dgamma.any() and float(dbeta) == n
