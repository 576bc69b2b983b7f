"""Softmax cross entropy of a linear layer against plain implementations in 64 bits.

Tolerances, element-wise (u = 2^-24):
  z      1e-5 of the sum of its terms' absolute values (fp32 sums in runs), the bias's addition u of that sum again
  lse    the largest error of a row's z; an exponential errs by (1 + |x|) 2^-23 of itself, which counts as much as its share of the sum; sums of
         positive terms: 64 u in a tile (32 in a lane, a tree of the rest), 4 u for each tile that is joined; a logarithm and its addition 2^-22 + 2 u |lse|
  loss   that of lse, that of z and u |loss|
  P      |g| p times (the errors of z and lse and (2 + |z - lse|) 2^-23), 3 u |g| (p + 1) for the difference and g; bfloat16 products: 2^-8 of its value on top
  dH, dW the sums of those times the other factor, 1e-5 of the sum of the terms' absolute values (4e-5 for bfloat16, whose tile of several
         runs is another), the rounding to bfloat16 2^-8
  dbias  the sum of P's errors without the rounding, 1e-5 of the sum of absolute values
"""
import pytest
import torch

import paper_2504_04673_amd as sagnn
from tests.test_gpu_row_operators import close, gen, normal, view

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
PREC = {"fp32": sagnn.GEMM_FP32, "x3": sagnn.GEMM_FP32_BF16X3, "rounded": sagnn.GEMM_BF16, "bf16": sagnn.GEMM_FP32}
SHAPES = [(1, 1, 1), (1, 8, 2), (3, 5, 7), (2, 16, 128), (33, 24, 129), (100, 64, 41), (257, 100, 172), (64, 128, 1000), (5, 256, 5003), (130, 602, 47),
          (1000, 16, 300), (300, 72, 70000), (20000, 40, 90), (4, 1025, 33), (2, 6000, 10), (513, 264, 520), (700, 136, 2056), (2000, 512, 256),
          (4099, 200, 54321)]             # (the last piece of the classes is narrower, and its gradient cut into more parts)


class Plain:
    def __init__(self, H, W, labels, bias, trans, g, mode):
        def operand(t):
            return (t.bfloat16() if mode == "rounded" else t).double()

        h, w = operand(H), operand(W.t().contiguous() if trans else W)
        m, n = h.shape[0], w.shape[1]
        b = torch.zeros(n, dtype=torch.float64, device="cuda") if bias is None else bias.double()
        z = h @ w + b
        ez = (1e-5 + U) * (h.abs() @ w.abs() + b.abs())
        top = z.amax(1, keepdim=True)
        lse = torch.logsumexp(z, 1)
        p = torch.exp(z - lse[:, None])
        self.lse = lse
        self.lse_bound = ez.amax(1) + 2.0 ** -23 * (p * (1 + (z - top).abs())).sum(1) + (64 + 4 * n / 64) * U + 2.0 ** -22 + 2 * U * lse.abs()
        known = (labels >= 0) & (labels < n)
        at = torch.where(known, labels, 0).long()[:, None]
        self.loss = torch.where(known, lse - z.gather(1, at)[:, 0], 0.0)
        self.loss_bound = torch.where(known, self.lse_bound + ez.gather(1, at)[:, 0] + U * self.loss.abs(), 0.0)
        g = torch.where(known, g.double() if isinstance(g, torch.Tensor) else torch.full((m,), g, dtype=torch.float64, device="cuda"), 0.0)[:, None]
        hit = torch.zeros_like(p).scatter_(1, at, 1.0)
        P = (p - hit) * g
        dP = g.abs() * (p * (ez + self.lse_bound[:, None] + (2 + (z - lse[:, None]).abs()) * 2.0 ** -23) + 3 * U * (p + hit))
        self.dbias, self.dbias_bound = P.sum(0), dP.sum(0) + 1e-5 * P.abs().sum(0) + 1e-37
        low = mode in ("rounded", "bf16")
        if low:
            dP = dP * (1 + 2.0 ** -8) + P.abs() * 2.0 ** -8
        sums = 4e-5 if mode == "bf16" else 1e-5
        last = 2.0 ** -8 if mode == "bf16" else U
        wa, ha = w.abs().t().contiguous(), h.abs().t().contiguous()
        self.dH, self.dW = P @ w.t().contiguous(), h.t().contiguous() @ P
        self.dH_bound = (dP + sums * P.abs()) @ wa * 1.001 + last * self.dH.abs() + 1e-37
        self.dW_bound = ha @ (dP + sums * P.abs()) * 1.001 + last * self.dW.abs() + 1e-37
        if trans:
            self.dW, self.dW_bound = self.dW.t(), self.dW_bound.t()


def inputs(seed, m, k, n, dtype, trans, biased, labelled, strided):
    g = gen(seed)
    H = normal(g, m, k, dtype=dtype)
    W = normal(g, *((n, k) if trans else (k, n)), scale=2.0 * k ** -0.5, dtype=dtype)
    bias = normal(g, n) if biased else None
    labels = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    if labelled < 1:
        out = torch.tensor([-1, n, -(1 << 31), (1 << 31) - 1], dtype=torch.int32, device="cuda")
        drop = torch.rand(m, generator=g, device="cuda") >= labelled
        labels = torch.where(drop, out[torch.randint(0, 4, (m,), generator=g, device="cuda")], labels)
    if strided:
        H, W = view(H, 3, 1), view(W, 5, 3)
    return H, W, labels, bias


@pytest.mark.parametrize("mode", ["fp32", "x3", "rounded", "bf16"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_loss_and_gradients(m, k, n, mode):
    dtype = torch.bfloat16 if mode == "bf16" else torch.float32
    for i, (trans, biased, labelled, strided) in enumerate([(False, True, 1.0, False), (True, False, 0.4, False), (True, True, 0.7, True), (False, False, 0.5, True), (False, True, 1.0, True)]):
        H, W, labels, bias = inputs(m + k + n + i, m, k, n, dtype, trans, biased, labelled, strided)
        g = 1.0 / m if i % 2 else normal(gen(i), m, scale=1.0 / m)
        what = f"case {i}"
        ref = Plain(H, W, labels, bias, trans, g, mode)
        loss, lse = sagnn.softmax_xent(H, W, labels, bias=bias, transW=trans, prec=PREC[mode])
        close(lse, ref.lse, ref.lse_bound, "lse, " + what)
        close(loss, ref.loss, ref.loss_bound, "loss, " + what)
        dH, dW, dbias = sagnn.softmax_xent_bwd(H, W, labels, lse, g, bias=bias, transW=trans, prec=PREC[mode])
        close(dH, ref.dH, ref.dH_bound, "dH, " + what)
        close(dW, ref.dW, ref.dW_bound, "dW, " + what)
        assert dH.dtype is dW.dtype is dtype
        if biased:
            close(dbias, ref.dbias, ref.dbias_bound, "dbias, " + what)
        else:
            assert dbias is None
        if m * n < 1 << 20:
            again = sagnn.softmax_xent_bwd(H, W, labels, lse, g, bias=bias, transW=trans, prec=PREC[mode])
            assert torch.equal(again[0], dH) and torch.equal(again[1], dW) and (bias is None or torch.equal(again[2], dbias))
            first = sagnn.softmax_xent_bwd(H, W, labels, lse, g, bias=bias, transW=trans, prec=PREC[mode], want_dw=False)
            other = sagnn.softmax_xent_bwd(H, W, labels, lse, g, bias=bias, transW=trans, prec=PREC[mode], want_dh=False)
            assert torch.equal(first[0], dH) and first[1] is None and other[0] is None and torch.equal(other[1], dW)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("n", [30, 300])
def test_rows_without_a_label_meet_nothing(dtype, n):
    H, W, labels, bias = inputs(1, 200, 40, n, dtype, False, True, 0.5, False)
    ignored = (labels < 0) | (labels >= n)
    clean = H.clone()
    clean[ignored] = 0
    H[ignored] = float("nan")
    H[ignored.nonzero()[:3, 0], 5] = float("inf")
    loss, lse = sagnn.softmax_xent(H, W, labels, bias=bias)
    assert not loss[ignored].any() and torch.equal(loss, sagnn.softmax_xent(clean, W, labels, bias=bias)[0])
    assert lse[ignored].isnan().all()
    grads = sagnn.softmax_xent_bwd(H, W, labels, lse, 0.01, bias=bias)
    ref = sagnn.softmax_xent_bwd(clean, W, labels, lse, 0.01, bias=bias)
    assert all(torch.equal(a, b) and a.isfinite().all() for a, b in zip(grads, ref)) and not grads[0][ignored].any()
    none = torch.full_like(labels, -1)
    loss, lse = sagnn.softmax_xent(clean, W, none)
    dH, dW, dbias = sagnn.softmax_xent_bwd(H, W, none, lse, 0.01, bias=bias)
    assert not loss.any() and not dH.any() and not dW.any() and not dbias.any()
    few = sagnn.softmax_xent_bwd(H[:5], W, none[:5], lse[:5], 0.01, bias=bias)
    assert not any(t.any() for t in few)
    z = clean[:0]
    loss, lse = sagnn.softmax_xent(z, W, labels[:0])
    dH, dW, dbias = sagnn.softmax_xent_bwd(z, W, labels[:0], lse, bias=bias)
    assert loss.shape == (0,) and dH.shape == z.shape and not dW.any() and not dbias.any()


@pytest.mark.parametrize("n", [20, 400])
def test_logits_without_bounds(n):
    H, W, labels, bias = inputs(3, 70, 24, n, torch.float32, False, True, 1.0, False)
    labels = labels.clamp(max=n - 3)
    # classes that are taken out: neither the loss nor a gradient has them
    bias[n - 2:] = -float("inf")
    loss, lse = sagnn.softmax_xent(H, W, labels, bias=bias)
    ref = sagnn.softmax_xent(H, W[:, :n - 2].contiguous(), labels, bias=bias[:n - 2].contiguous())
    assert torch.allclose(lse, ref[1], rtol=1e-6, atol=1e-6) and torch.allclose(loss, ref[0], rtol=1e-6, atol=2e-6)
    dH, dW, dbias = sagnn.softmax_xent_bwd(H, W, labels, lse, 0.1, bias=bias)
    assert dH.isfinite().all() and dW.isfinite().all() and not dW[:, n - 2:].any() and not dbias[n - 2:].any()
    # one of them as a label: an infinite loss, and the formula's gradient
    odd = labels.clone()
    odd[5] = n - 1
    loss, lse = sagnn.softmax_xent(H, W, odd, bias=bias)
    assert float(loss[5]) == float("inf") and loss[:5].isfinite().all() and loss[6:].isfinite().all()
    assert float(sagnn.softmax_xent_bwd(H, W, odd, lse, 0.1, bias=bias)[2][n - 1]) == pytest.approx(-0.1)
    # all of them: no sum, and nothing to divide by
    none = torch.full_like(bias, -float("inf"))
    loss, lse = sagnn.softmax_xent(H, W, labels, bias=none)
    assert (lse == -float("inf")).all() and loss.isnan().all()
    # an infinite one
    none = torch.zeros_like(bias)
    none[n - 1] = float("inf")
    loss, lse = sagnn.softmax_xent(H, W, labels, bias=none)
    assert (lse == float("inf")).all() and (loss == float("inf")).all()
    # far from zero, and far apart; the lowest value of the type as a mask
    far = torch.linspace(-1e4, 1e4, n, device="cuda")
    loss, lse = sagnn.softmax_xent(H, W, labels, bias=far)
    assert torch.allclose(lse.double(), torch.logsumexp(H.double() @ W.double() + far.double(), 1), rtol=1e-6)
    assert sagnn.softmax_xent_bwd(H, W, labels, lse, bias=far)[0].isfinite().all()
    low = torch.full_like(bias, torch.finfo(torch.float32).min)
    loss, lse = sagnn.softmax_xent(H, W, labels, bias=low)
    assert torch.allclose(lse.double(), low.double()[0].expand(70), rtol=1e-6) and sagnn.softmax_xent_bwd(H, W, labels, lse, bias=low)[0].isfinite().all()
    H[7, 3] = float("nan")
    loss, lse = sagnn.softmax_xent(H, W, labels)
    assert lse[7].isnan() and loss[7].isnan() and lse[:7].isfinite().all() and lse[8:].isfinite().all()


def test_gradients_against_differences():
    H, W, labels, bias = inputs(9, 6, 10, 13, torch.float32, True, True, 0.8, False)
    g = torch.rand(6, generator=gen(4), device="cuda")

    def loss(h, w, b):
        z = h.double() @ w.double().t() + b.double()
        known = (labels >= 0) & (labels < 13)
        at = torch.where(known, labels, 0).long()[:, None]
        return float(((torch.logsumexp(z, 1) - z.gather(1, at)[:, 0]) * known * g).sum())

    lse = sagnn.softmax_xent(H, W, labels, bias=bias, transW=True)[1]
    grads = sagnn.softmax_xent_bwd(H, W, labels, lse, g, bias=bias, transW=True)
    for t, d, f in ((H, grads[0], lambda x: loss(x, W, bias)), (W, grads[1], lambda x: loss(H, x, bias)), (bias, grads[2], lambda x: loss(H, W, x))):
        for at in range(0, t.numel(), 7):
            plus, minus = t.double().clone(), t.double().clone()
            plus.view(-1)[at] += 1e-5
            minus.view(-1)[at] -= 1e-5
            # (differences in 64 bits: 1e-10 of the third derivative; the gradient to 1e-5 of its terms, some units)
            assert abs((f(plus) - f(minus)) / 2e-5 - float(d.reshape(-1)[at])) < 1e-4


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
def test_captured_and_replayed(dtype):
    H, W, labels, bias = inputs(5, 600, 64, 1500, dtype, True, True, 0.6, False)

    def step():
        loss, lse = sagnn.softmax_xent(H, W, labels, bias=bias, transW=True)
        return (loss, lse, *sagnn.softmax_xent_bwd(H, W, labels, lse, 0.01, bias=bias, transW=True))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        H.copy_(normal(gen(20 + i), 600, 64, dtype=dtype))
        labels.copy_(torch.randint(-500, 1500, (600,), generator=gen(30 + i), device="cuda", dtype=torch.int32))
        ref = step()
        for t in got:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_calls_on_two_streams():
    H, W, labels, bias = inputs(6, 2000, 128, 3000, torch.bfloat16, True, True, 0.9, False)
    loss, lse = sagnn.softmax_xent(H, W, labels, bias=bias, transW=True)
    ref = sagnn.softmax_xent_bwd(H, W, labels, lse, 1e-3, bias=bias, transW=True)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                l2, lse2 = sagnn.softmax_xent(H, W, labels, bias=bias, transW=True)
                got.append((l2, lse2, *sagnn.softmax_xent_bwd(H, W, labels, lse2, 1e-3, bias=bias, transW=True)))
    torch.cuda.synchronize()
    for l2, lse2, *d in got:
        assert torch.equal(l2, loss) and torch.equal(lse2, lse) and all(torch.equal(a, b) for a, b in zip(d, ref))


def test_weights_behind_four_gigabytes():
    """2.5 million classes of 1024 values: only the last hundred are far from zero."""
    n, k = 2_500_000, 1024
    W = torch.zeros(n, k, dtype=torch.bfloat16, device="cuda")
    W[-100:] = normal(gen(1), 100, k, dtype=torch.bfloat16, scale=0.1)
    H = normal(gen(2), 3, k, dtype=torch.bfloat16)
    labels = torch.tensor([n - 1, n - 50, 7], dtype=torch.int32, device="cuda")
    loss, lse = sagnn.softmax_xent(H, W, labels, transW=True)
    z = H.double() @ W[-100:].double().t().contiguous()
    ref = torch.logsumexp(torch.cat([z, torch.full((3, 1), 0.0, device="cuda", dtype=torch.float64) + torch.log(torch.tensor(n - 100.0))], 1), 1)
    assert torch.allclose(lse.double(), ref, rtol=0, atol=1e-5 * float((H.double().abs() @ W[-100:].double().abs().t().contiguous()).max()) + 1e-3)
    assert torch.allclose(loss[:2].double(), (ref[:2] - z[[0, 1], [99, 50]]), rtol=0, atol=2e-3)
    dH, dW, _ = sagnn.softmax_xent_bwd(H, W, labels, lse, transW=True)
    p = torch.exp(z - ref[:, None])
    p[0, 99] -= 1
    p[1, 50] -= 1
    # (each term of P errs by 2^-8 and lse by 1e-3; dW by 2^-8 more)
    want = p.t().contiguous() @ H.double()
    assert torch.all((dW[-100:].double() - want).abs() <= (2.0 ** -7 + 2e-3) * (p.abs().t().contiguous() @ H.double().abs()) + 1e-6)
    want = p @ W[-100:].double()
    assert torch.all((dH.double() - want).abs() <= (2.0 ** -7 + 2e-3) * (p.abs() @ W[-100:].double().abs()) + 1e-6)


def test_so_many_rows_that_pieces_are_narrower():
    """2.2 million rows by 1200 classes: P of 1024 classes would be more than 4 GiB.  Against the same call on a few of the rows."""
    m, k, n = 2_200_000, 8, 1200
    H, W, labels, bias = inputs(3, m, k, n, torch.bfloat16, True, True, 0.5, False)
    loss, lse = sagnn.softmax_xent(H, W, labels, bias=bias, transW=True)
    dH, dW, dbias = sagnn.softmax_xent_bwd(H, W, labels, lse, 1e-3, bias=bias, transW=True)
    few = slice(m - 300, m)
    ref = Plain(H[few], W, labels[few], bias, True, 1e-3, "bf16")
    close(lse[few], ref.lse, ref.lse_bound, "lse")
    close(loss[few], ref.loss, ref.loss_bound, "loss")
    close(dH[few], ref.dH, ref.dH_bound, "dH")
    # sums over all rows in parts of 64 bits
    want, bound, wb, bb = 0.0, 0.0, 0.0, 0.0
    for a in range(0, m, 100_000):
        part = Plain(H[a:a + 100_000], W, labels[a:a + 100_000], bias, True, 1e-3, "bf16")
        want, bound, wb, bb = want + part.dW, bound + part.dW_bound, wb + part.dbias, bb + part.dbias_bound
    close(dW, want, bound, "dW")
    close(dbias, wb, bb, "dbias")


def unrounded(H, W, labels, g, bias=None):
    """Gradients in 64 bits, and the sums of their terms' absolute values."""
    h, w = H.double(), W.double()
    P = torch.softmax(h @ w + (0 if bias is None else bias.double()), 1)
    P.scatter_add_(1, labels.long()[:, None], torch.full_like(P[:, :1], -1.0))
    P *= g.double()[:, None] if isinstance(g, torch.Tensor) else g
    wt, ht = w.t().contiguous(), h.t().contiguous()
    return P @ wt, ht @ P, P.abs() @ wt.abs(), ht.abs() @ P.abs()


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("m,k,n", [(1, 24, 3), (1, 64, 2), (2, 40, 900), (9, 128, 47), (33, 100, 172), (130, 64, 2), (257, 16, 40000), (512, 264, 130)])
def test_few_bfloat16_rows_meet_one_rounding(m, k, n, weights):
    """P in two terms errs by 2^-16 of itself (what a rounding leaves is 2^-8 of it at most, and is rounded by 2^-8 of that); all else as with fp32 operands, 4e-5 for the sums,
    the result's rounding 2^-8 and the factor's 2 u."""
    H, W, labels, bias = inputs(m + k + n, m, k, n, torch.bfloat16, False, True, 1.0, False)
    g = normal(gen(m), m).abs() + 0.1 if weights else 1.0 + 2.0 ** -8
    _, lse = sagnn.softmax_xent(H, W, labels, bias=bias)
    dH, dW, _ = sagnn.softmax_xent_bwd(H, W, labels, lse, g, bias=bias)
    ref = Plain(H, W, labels, bias, False, g, "fp32")
    rH, rW, aH, aW = unrounded(H, W, labels, g, bias)
    close(dH, rH, ref.dH_bound + (3e-5 + 2.0 ** -16) * 1.001 * aH + (2.0 ** -8 + 2 * U) * rH.abs(), "dH")
    close(dW, rW, ref.dW_bound + (3e-5 + 2.0 ** -16) * 1.001 * aW + (2.0 ** -8 + 2 * U) * rW.abs(), "dW")


@pytest.mark.parametrize("m,k,n", [(600, 72, 4096), (3000, 100, 1024), (2500, 512, 8192)])
def test_a_factor_of_all_rows_is_not_rounded(m, k, n):
    """W of zeros, or H of zeros: p = 1 / n, a power of two, and P is off by 1 / n in the label's place at most; sums 4e-5, the result's rounding 2^-8.  The factor 1 + 2^-8, halfway
    between two bfloat16 values, would be off by 2^-8 more in every term."""
    H, W, labels, _ = inputs(m, m, k, n, torch.bfloat16, False, False, 1.0, False)
    g = 1.0 + 2.0 ** -8
    for h, w in ((H, torch.zeros_like(W)), (torch.zeros_like(H), W)):
        _, lse = sagnn.softmax_xent(h, w, labels)
        dH, dW, _ = sagnn.softmax_xent_bwd(h, w, labels, lse, g)
        rH, rW, aH, aW = unrounded(h, w, labels, g)
        close(dH, rH, 2.0 ** -8 * rH.abs() + (1.0 / n + 6e-5) * aH, "dH")
        close(dW, rW, 2.0 ** -8 * rW.abs() + (1.0 / n + 6e-5) * aW, "dW")


@pytest.mark.parametrize("m", [70, 700])
def test_no_labelled_row_whatever_the_factor(m):
    H, W, labels, bias = inputs(m, m, 40, 300, torch.bfloat16, False, True, 1.0, False)
    labels.fill_(-1)
    _, lse = sagnn.softmax_xent(H, W, labels, bias=bias)
    for g in (float("inf"), float("nan")):
        assert not any(t.any() for t in sagnn.softmax_xent_bwd(H, W, labels, lse, g, bias=bias))


@pytest.mark.parametrize("m,k,n", [(758, 512, 2), (1024, 72, 300)])
def test_weighted_bfloat16_rows_meet_one_rounding(m, k, n):
    test_few_bfloat16_rows_meet_one_rounding(m, k, n, True)
