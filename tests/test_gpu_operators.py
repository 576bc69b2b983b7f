"""Grouped products, group norm and gradient clipping against plain implementations in 64 bits.

Tolerances, all element-wise (u = 2^-24, the rounding of fp32; a bfloat16 result is rounded once more, by 2^-8):
  products  1e-5 * sum |terms| for sums in fp32 in any order (168 u: runs of some hundred terms and their joins); operands
            rounded to bfloat16 are rounded before both sides
  norm      z = (x - mean) rstd gamma + beta: mean, rstd and four operations rounded, 2^-20 of |x - mean| rstd |gamma| +
            |mean| rstd |gamma| + |beta|; SiLU has slope below 1.1 and an exponential good to (2 + |z|) 2^-22
  gradients 1e-5 of the sum of the absolute values of the terms, grown by 1 + |mean| rstd for the rounding of mean
  clipping  norm to 2^-23 (sums in 64 bits, one rounding), values to three roundings
"""
import numpy as np
import pytest
import torch

import paper_2504_04673_amd as sagnn
from paper_2504_04673_amd import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
PREC = {"fp32": sagnn.GEMM_FP32, "x3": sagnn.GEMM_FP32_BF16X3, "rounded": sagnn.GEMM_BF16, "bf16": sagnn.GEMM_FP32}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def offsets(sizes):
    return torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")


def close(got, ref, bound, what):
    got, bad = got.double(), None
    err = (got - ref).abs()
    bad = ~(err <= bound)                                 # (NaN counts)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / bound)[bad].max()):.3g} times the bound"


def rounding(dtype, ref):
    return ref.abs() * (2.0 ** -8 if dtype is torch.bfloat16 else 0.0)


# ---------------------------------------------------------------------------------------------
# grouped products

def operand(t, mode):
    return (t.bfloat16() if mode == "rounded" else t).double()


def plain_product(X, W, off, trans, mode):
    """Y and sum |terms|."""
    n = W.shape[1 if trans else 2]
    Y = torch.zeros(X.shape[0], n, dtype=torch.float64, device=X.device)
    A = torch.zeros_like(Y)
    o = off.tolist()
    for g in range(len(o) - 1):
        x, w = operand(X[o[g]:o[g + 1]], mode), operand(W[g], mode)
        w = w.t().contiguous() if trans else w
        Y[o[g]:o[g + 1]] = x @ w
        A[o[g]:o[g + 1]] = x.abs() @ w.abs()
    return Y, A


def plain_wgrad(X, G, off, mode):
    o = off.tolist()
    parts = [(operand(X[a:b], mode).t().contiguous(), operand(G[a:b], mode)) for a, b in zip(o[:-1], o[1:])]
    return torch.stack([x @ g for x, g in parts]), torch.stack([x.abs() @ g.abs() for x, g in parts])


SIZES = [
    [1], [0], [5, 0, 1], [64, 64, 64], [33, 0, 0, 200, 1, 7], [300, 31, 129], [1000], [0, 0, 700, 0], [2] * 70, [0] * 65 + [40, 3] + [1] * 130,
]
WIDTHS = [(1, 1), (3, 5), (16, 24), (32, 32), (64, 128), (100, 40), (130, 257), (256, 256), (602, 41), (72, 1000)]


@pytest.mark.parametrize("mode", ["fp32", "x3", "rounded", "bf16"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{sum(s)}")
def test_product_of_ragged_groups(sizes, mode):
    dtype = torch.bfloat16 if mode == "bf16" else torch.float32
    for i, (k, n) in enumerate(WIDTHS):
        g = gen(i)
        off = offsets(sizes)
        m = sum(sizes) + (0, 3)[i % 2]                      # rows behind the last group
        trans, act, masked = i % 3 == 1, i % 2, i % 4 == 2
        X = normal(g, m, k, dtype=dtype)
        X[sum(sizes):] = float("nan")                       # (not used)
        W = normal(g, len(sizes), *((n, k) if trans else (k, n)), dtype=dtype)
        mask = normal(g, m, n, dtype=dtype) if masked else None
        Y = sagnn.grouped_gemm_act(X, W, off, transW=trans, prec=PREC[mode], act=act, mask=mask)
        ref, terms = plain_product(X, W, off, trans, mode)
        if act == sagnn.ACT_RELU:
            ref = ref.clamp(min=0.0)
        if masked:
            ref = ref * (mask > 0)
        assert Y.dtype is dtype and Y.shape == (m, n)
        close(Y, ref, 1e-5 * terms + rounding(dtype, ref) + 1e-30, f"{k} x {n}")
        assert not Y[sum(sizes):].any()


@pytest.mark.parametrize("mode", ["fp32", "x3", "rounded", "bf16"])
@pytest.mark.parametrize("sizes", SIZES + [[20000, 1, 3000]], ids=lambda s: f"{len(s)}x{sum(s)}")
def test_gradients_of_ragged_groups(sizes, mode):
    dtype = torch.bfloat16 if mode == "bf16" else torch.float32
    for i, (k, n) in enumerate(WIDTHS):
        g = gen(100 + i)
        off = offsets(sizes)
        m = sum(sizes) + (0, 5)[i % 2]
        X, W, G = normal(g, m, k, dtype=dtype), normal(g, len(sizes), k, n, dtype=dtype), normal(g, m, n, dtype=dtype)
        X[sum(sizes):] = float("inf")
        G[sum(sizes):] = float("nan")
        mask = normal(g, m, k, dtype=dtype) if i % 2 else None
        dX, dW = sagnn.grouped_gemm_bwd(X, W, off, G, mask=mask, prec=PREC[mode])
        ref, terms = plain_product(G, W, off, True, mode)
        if mask is not None:
            ref = ref * (mask > 0)
        close(dX, ref, 1e-5 * terms + rounding(dtype, ref) + 1e-30, f"dX {k} x {n}")
        ref, terms = plain_wgrad(X, G, off, mode)
        assert dW.dtype is torch.float32
        close(dW, ref, 1e-5 * terms + 1e-30, f"dW {k} x {n}")
        if i == 3:                                          # one gradient alone: the same bits
            only_x, none = sagnn.grouped_gemm_bwd(None, W, off, G, mask=mask, prec=PREC[mode], want_dw=False)
            assert none is None and torch.equal(only_x, dX)
            none, only_w = sagnn.grouped_gemm_bwd(X, W, off, G, prec=PREC[mode], want_dx=False)
            assert none is None and torch.equal(only_w, dW)


@pytest.mark.parametrize("mode", ["fp32", "x3", "rounded", "bf16"])
@pytest.mark.parametrize("sizes", [[37, 0, 20], [9000, 5000, 71]], ids=lambda s: f"{sum(s)}")
def test_masks_of_every_width_in_four(sizes, mode):
    dtype = torch.bfloat16 if mode == "bf16" else torch.float32
    off, m = offsets(sizes), sum(sizes)
    for n in (1, 2, 3, 4, 5, 6, 7, 30, 33, 66, 127, 129, 131, 259):
        g = gen(n)
        X, W = normal(g, m, 24, dtype=dtype), normal(g, len(sizes), 24, n, dtype=dtype)
        wide = normal(g, m, n + 3, dtype=dtype)             # (rows that begin anywhere, and what lies beside them would pass other values)
        mask = wide[:, 1:n + 1]
        mask[::7] = float("nan")
        mask[1::7] = 0.0
        mask[2::7] = float("inf")
        Y = sagnn.grouped_gemm_act(X, W, off, mask=mask, prec=PREC[mode])
        ref, terms = plain_product(X, W, off, False, mode)
        ref = torch.where(mask > 0, ref, 0.0)
        close(Y, ref, 1e-5 * terms + rounding(dtype, ref) + 1e-30, f"{n} columns")
        assert not Y[~(mask > 0)].any()


@pytest.mark.parametrize("mode", ["fp32", "x3", "rounded", "bf16"])
@pytest.mark.parametrize("m,types,k,n", [(4100, 3, 512, 384), (3000, 2, 320, 576), (1500, 5, 1024, 136), (2600, 1, 264, 1544)])
def test_products_that_fill_large_tiles(m, types, k, n, mode):
    """Widths and groups of several of the largest tiles and a part of one in each direction."""
    dtype = torch.bfloat16 if mode == "bf16" else torch.float32
    g = gen(m)
    cut = np.sort(np.random.default_rng(m).integers(0, m + 1, types - 1))
    off = offsets(np.diff([0, *cut, m]))
    X, W, G = normal(g, m, k, dtype=dtype), normal(g, types, k, n, dtype=dtype), normal(g, m, n, dtype=dtype)
    ref, terms = plain_product(X, W, off, False, mode)
    close(sagnn.grouped_gemm_act(X, W, off, prec=PREC[mode]), ref, 1e-5 * terms + rounding(dtype, ref), "Y")
    Wt = W.transpose(1, 2).contiguous()
    close(sagnn.grouped_gemm_act(X, Wt, off, transW=True, prec=PREC[mode]), ref, 1e-5 * terms + rounding(dtype, ref), "Y, W transposed")
    mask = normal(g, m, k, dtype=dtype)
    dX, dW = sagnn.grouped_gemm_bwd(X, W, off, G, mask=mask, prec=PREC[mode])
    ref, terms = plain_product(G, W, off, True, mode)
    ref = ref * (mask > 0)
    close(dX, ref, 1e-5 * terms + rounding(dtype, ref) + 1e-30, "dX")
    ref, terms = plain_wgrad(X, G, off, mode)
    close(dW, ref, 1e-5 * terms, "dW")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [0, 1, 3, 8])
def test_products_on_slices_of_wider_matrices(shift, dtype):
    """Leading dimensions and first elements of every alignment; what lies beside an output stays as it was."""
    g = gen(shift)
    m, k, n, off = 517, 200, 136, offsets([100, 0, 350, 60])
    wide = {name: normal(g, rows, cols + 24 + shift % 2, dtype=dtype) for name, rows, cols in
            (("X", m, k), ("G", m, n), ("mask", m, n), ("out", m, n))}
    X, G, mask, out = (wide[a][:, shift:shift + w] for a, w in (("X", k), ("G", n), ("mask", n), ("out", n)))
    W = normal(g, 4, k + 2, n + shift, dtype=dtype)[:, 1:1 + k, shift:]
    mode = "bf16" if dtype is torch.bfloat16 else "x3"
    before = wide["out"].clone()
    Y = sagnn.grouped_gemm_act(X, W, off, prec=PREC[mode], mask=mask, out=out)
    ref, terms = plain_product(X, W, off, False, mode)
    ref = ref * (mask > 0)
    close(Y, ref, 1e-5 * terms + rounding(dtype, ref) + 1e-30, "Y")
    assert torch.equal(wide["out"][:, :shift], before[:, :shift]) and torch.equal(wide["out"][:, shift + n:], before[:, shift + n:])
    dX, dW = sagnn.grouped_gemm_bwd(X, W, off, G, prec=PREC[mode])
    ref, terms = plain_product(G, W, off, True, mode)
    close(dX, ref, 1e-5 * terms + rounding(dtype, ref), "dX")
    ref, terms = plain_wgrad(X, G, off, mode)
    close(dW, ref, 1e-5 * terms + 1e-30, "dW")


def test_products_behind_32_bit_offsets():
    """Rows, types and columns whose element numbers pass 2^31 and 2^32."""
    g, dtype = gen(5), torch.bfloat16
    m, k, n, ld = 70000, 40, 24, 65536
    X = torch.zeros(m, ld, dtype=dtype, device="cuda")[:, 7:7 + k]
    X.copy_(normal(g, m, k, dtype=dtype))
    off = offsets([30000, 0, 39999])
    W = torch.zeros(3, 1 << 31, dtype=torch.int8, device="cuda").view(dtype)[:, :k * n].unflatten(1, (k, n))
    W.copy_(normal(g, 3, k, n, dtype=dtype))
    G = normal(g, m, n, dtype=dtype)
    ref, terms = plain_product(X, W, off, False, "bf16")
    close(sagnn.grouped_gemm_act(X, W, off), ref, 1e-5 * terms + rounding(dtype, ref) + 1e-30, "Y")
    dX, dW = sagnn.grouped_gemm_bwd(X, W, off, G)
    ref, terms = plain_wgrad(X, G, off, "bf16")
    close(dW, ref, 1e-5 * terms + 1e-30, "dW")
    ref, terms = plain_product(G, W, off, True, "bf16")
    close(dX, ref, 1e-5 * terms + rounding(dtype, ref) + 1e-30, "dX")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_products_keep_infinities_and_nan_to_their_rows_and_groups(dtype):
    g = gen(9)
    off = offsets([70, 60, 80])
    X, W = normal(g, 210, 96, dtype=dtype), normal(g, 3, 96, 48, dtype=dtype)
    X[3, 5], X[100, 95] = float("inf"), float("nan")
    W[2, 10, 7] = float("nan")
    Y = sagnn.grouped_gemm_act(X, W, off, act=sagnn.ACT_RELU)
    bad = torch.zeros(210, 48, dtype=torch.bool, device="cuda")
    bad[100], bad[130:, 7] = True, True
    assert torch.equal(Y.isnan(), bad)
    assert torch.equal(Y[3].isinf(), W[0, 5] > 0) and not Y[4].isinf().any()
    _, dW = sagnn.grouped_gemm_bwd(X, W, off, torch.ones(210, 48, dtype=dtype, device="cuda"), want_dx=False)
    assert bool(dW[0, 5].isinf().all()) and bool(dW[1, 95].isnan().all()) and int(dW.isfinite().logical_not().sum()) == 2 * 48


def test_product_gradients_against_differences():
    """The loss <G, Y> is linear in X and in W: its differences are exact up to rounding."""
    g = gen(12)
    off = offsets([40, 0, 25, 64])
    X, W, G = normal(g, 129, 33), normal(g, 4, 33, 50), normal(g, 129, 50)
    dX, dW = sagnn.grouped_gemm_bwd(X, W, off, G)

    def loss(X, W):
        return float((sagnn.grouped_gemm_act(X, W, off).double() * G.double()).sum())

    terms = float((plain_product(X, W, off, False, "fp32")[1] * G.double().abs()).sum())
    for d in (normal(g, 129, 33), normal(g, 4, 33, 50)):
        if d.dim() == 2:
            diff, grad = (loss(X + d, W) - loss(X - d, W)) / 2, float((d.double() * dX.double()).sum())
        else:
            diff, grad = (loss(X, W + d) - loss(X, W - d)) / 2, float((d.double() * dW.double()).sum())
        assert abs(diff - grad) <= 4e-5 * terms               # 1e-5 each of three losses and a gradient, of terms up to twice as large


# ---------------------------------------------------------------------------------------------
# group norm

def plain_norm(X, groups, gamma, beta, seg, eps, act, G=None):
    """Everything in 64 bits: y, mean, rstd, and with G the gradients; beside each result the scale of its error."""
    o, (m, c) = seg.tolist(), X.shape
    d = c // groups
    x = X.double()
    gamma = torch.ones(c, device=X.device).double() if gamma is None else gamma.double()
    beta = torch.zeros(c, device=X.device).double() if beta is None else beta.double()
    r = {k: torch.zeros_like(x) for k in ("y", "y_scale", "dx", "dx_scale")}
    mean = torch.zeros(len(o) - 1, groups, dtype=torch.float64, device=X.device)
    rstd = torch.full_like(mean, eps ** -0.5 if eps > 0 else float("inf"))
    for k in ("dgamma", "dbeta", "dgamma_scale", "dbeta_scale"):
        r[k] = torch.zeros(c, dtype=torch.float64, device=X.device)
    for b in range(len(o) - 1):
        if o[b] == o[b + 1]:
            continue
        for q in range(groups):
            ch = slice(q * d, (q + 1) * d)
            v = x[o[b]:o[b + 1], ch]
            mu = v.mean()
            rs = ((v - mu).square().mean() + eps).rsqrt()
            mean[b, q], rstd[b, q] = mu, rs
            xh = (v - mu) * rs
            z = xh * gamma[ch] + beta[ch]
            sig = torch.sigmoid(z)
            y = (z, z.clamp(min=0.0), z * sig)[act]
            rows = slice(o[b], o[b + 1])
            size = (xh.abs() + mu.abs() * rs) * gamma[ch].abs() + beta[ch].abs()
            r["y"][rows, ch] = y
            r["y_scale"][rows, ch] = 16 * U * size * (1.1 if act == 2 else 1.0) + (4 * U * (4 + z.abs()) * z.abs() if act == 2 else 0.0)
            if G is not None:
                slope = (torch.ones_like(z), (z > 0).double(), sig * (1 + z * (1 - sig)))[act]
                g = G[rows, ch].double()
                h = g * slope
                grow = 1 + mu.abs() * rs
                # SiLU's slope is known to the error of z (its own slope is at most 1/2) and of the exponential
                hs = h.abs() + (g.abs() * (size + 1) if act == 2 else 0.0)
                r["dgamma"][ch] += (h * xh).sum(0)
                r["dbeta"][ch] += h.sum(0)
                r["dgamma_scale"][ch] += (hs * (xh.abs() + 1) * grow).sum(0)
                r["dbeta_scale"][ch] += (hs * grow).sum(0)
                hg, hgs = h * gamma[ch], hs * gamma[ch].abs()
                r["dx"][rows, ch] = rs * (hg - hg.mean() - xh * (hg * xh).mean())
                r["dx_scale"][rows, ch] = rs * grow * (hgs + hgs.mean() + (xh.abs() + 1) * (hgs * (xh.abs() + 1)).mean())
    r["mean"], r["rstd"] = mean, rstd
    return r


SEGMENTS = [[1], [7], [40, 0, 1, 2, 30], [64] * 5, [513, 3, 0, 0, 100], [0, 0, 0], [3000], [1] * 200, [0] * 70 + [9, 150] + [2] * 80]
CHANNELS = [(1, 1), (8, 8), (12, 4), (30, 2), (64, 8), (100, 4), (256, 32), (256, 1), (602, 7), (1030, 2)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", SEGMENTS, ids=lambda s: f"{len(s)}x{sum(s)}")
def test_norm_of_ragged_segments(sizes, dtype):
    for i, (c, groups) in enumerate(CHANNELS):
        if len(sizes) * groups > 2000:                       # (the plain form goes one by one)
            continue
        g = gen(i)
        act, known, extra = i % 3, i % 2, (0, 4)[i % 2]
        m, eps, seg = sum(sizes) + extra, 1e-3 if i % 4 == 3 else 1e-5, offsets(sizes)
        X = normal(g, m, c).mul_(0.5 + torch.rand(c, generator=g, device="cuda")).add_(normal(g, c, scale=3.0)).to(dtype)
        gamma, beta = (normal(g, c), normal(g, c)) if i % 4 else (None, None)
        G = normal(g, m, c, dtype=dtype)
        ref = plain_norm(X, groups, gamma, beta, seg, eps, act)
        if act == sagnn.ACT_RELU:                            # nothing where ReLU's slope could go either way
            G[ref["y"].abs() <= 1e-3] = 0.0
            z = plain_norm(X, groups, gamma, beta, seg, eps, 0)["y"]
            G[z.abs() <= 1e-3] = 0.0
        X[sum(sizes):], G[sum(sizes):] = float("nan"), float("inf")
        ref = plain_norm(X, groups, gamma, beta, seg, eps, act, G)
        longest = max(sizes) if known else 0
        Y, mean, rstd = sagnn.group_norm_act(X, groups, gamma, beta, seg=seg, max_rows=longest, eps=eps, act=act)
        close(mean, ref["mean"], 2 * U * ref["mean"].abs() + 1e-12, f"mean {c}/{groups}")
        close(rstd, ref["rstd"], 8 * U * ref["rstd"], f"rstd {c}/{groups}")
        close(Y, ref["y"], ref["y_scale"] + rounding(dtype, ref["y"]) * 1.01 + 1e-30, f"y {c}/{groups}")
        assert not Y[sum(sizes):].any()
        dX, dgamma, dbeta = sagnn.group_norm_act_bwd(X, G, mean, rstd, groups, gamma, beta, seg=seg, max_rows=longest, act=act)
        close(dX, ref["dx"], 1e-5 * ref["dx_scale"] + rounding(dtype, ref["dx"]) * 1.01 + 1e-30, f"dx {c}/{groups}")
        close(dgamma, ref["dgamma"], 1e-5 * ref["dgamma_scale"] + 1e-30, f"dgamma {c}/{groups}")
        close(dbeta, ref["dbeta"], 1e-5 * ref["dbeta_scale"] + 1e-30, f"dbeta {c}/{groups}")
        assert not dX[sum(sizes):].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 12, 40, 300])
@pytest.mark.parametrize("c,groups", [(1000, 250), (4096, 1024), (1024, 1024), (1000, 8), (16384, 4), (528, 44)])
def test_norm_of_many_and_of_wide_groups(c, groups, rows, dtype):
    g = gen(c + rows)
    X, G = normal(g, 3 * rows, c, dtype=dtype), normal(g, 3 * rows, c, dtype=dtype)
    known = rows if rows < 300 else 0
    x, h = (t.double().view(3, rows, groups, -1) for t in (X, G))
    n = rows * (c // groups)
    mean = x.mean((1, 3), keepdim=True)
    rstd = ((x - mean).square().mean((1, 3), keepdim=True) + 1e-2).rsqrt()
    xh = (x - mean) * rstd
    size = (x.abs() + mean.abs()) * rstd
    Y, m32, r32 = sagnn.group_norm_act(X, groups, n_seg=3, max_rows=known, eps=1e-2)
    close(Y, xh.view_as(X), 2.0 ** -20 * size.view_as(X) + 1.01 * rounding(dtype, xh.view_as(X)) + 1e-30, "y")
    dX, dgamma, dbeta = sagnn.group_norm_act_bwd(X, G, m32, r32, groups, torch.ones(c, device="cuda"), torch.zeros(c, device="cuda"), n_seg=3,
                                                 max_rows=known)
    s1, s2 = h.mean((1, 3), keepdim=True), (h * xh).mean((1, 3), keepdim=True)
    dx = (rstd * (h - s1 - xh * s2)).view_as(X)
    a1, a2 = h.abs().mean((1, 3), keepdim=True), (h.abs() * size).mean((1, 3), keepdim=True)
    close(dX, dx, 1e-5 * (rstd * (h.abs() + a1 + size * a2)).view_as(X) + 1.01 * rounding(dtype, dx) + 1e-30, "dx")
    close(dgamma, (h * xh).sum((0, 1)).flatten(), 1e-5 * (h.abs() * size).sum((0, 1)).flatten() + 1e-30, "dgamma")
    close(dbeta, h.sum((0, 1)).flatten(), 1e-5 * h.abs().sum((0, 1)).flatten() + 1e-30, "dbeta")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_seg,rows,c,groups", [(1, 1, 4, 1), (6, 50, 64, 4), (2, 1025, 48, 16), (300, 1, 128, 1), (1, 20000, 320, 32)])
def test_norm_of_equal_segments_is_that_of_their_offsets(n_seg, rows, c, groups, dtype):
    g = gen(rows)
    X, G = normal(g, n_seg * rows, c, dtype=dtype), normal(g, n_seg * rows, c, dtype=dtype)
    gamma, beta = normal(g, c), normal(g, c)
    seg = offsets([rows] * n_seg)
    a = sagnn.group_norm_act(X, groups, gamma, beta, n_seg=n_seg, act=sagnn.ACT_SILU, max_rows=rows)
    b = sagnn.group_norm_act(X, groups, gamma, beta, seg=seg, act=sagnn.ACT_SILU, max_rows=rows)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    p = sagnn.group_norm_act_bwd(X, G, *a[1:], groups, gamma, beta, n_seg=n_seg, act=sagnn.ACT_SILU, max_rows=rows)
    q = sagnn.group_norm_act_bwd(X, G, *a[1:], groups, gamma, beta, seg=seg, act=sagnn.ACT_SILU, max_rows=rows)
    assert all(torch.equal(x, y) for x, y in zip(p, q))


def test_norm_of_no_rows():
    X = torch.zeros(0, 12, device="cuda")
    Y, mean, rstd = sagnn.group_norm_act(X, 3, n_seg=2, eps=0.25)
    assert Y.shape == (0, 12) and not mean.any() and bool((rstd == 2.0).all())
    dX, dgamma, dbeta = sagnn.group_norm_act_bwd(X, X, mean, rstd, 3, n_seg=2)
    assert dX.shape == (0, 12) and not dgamma.any() and not dbeta.any()


@pytest.mark.parametrize("rows", [40, 5000])
def test_norm_far_from_zero_keeps_its_variance(rows):
    """Mean 1000 times the deviation: the squares' sum and the squared mean agree in their first twenty bits."""
    g = gen(1)
    X = normal(g, rows, 16) + 1000.0
    seg = offsets([rows])
    ref = plain_norm(X, 2, None, None, seg, 1e-5, 0)
    Y, mean, rstd = sagnn.group_norm_act(X, 2, seg=seg, max_rows=rows)
    close(rstd, ref["rstd"], 8 * U * ref["rstd"], "rstd")
    close(Y, ref["y"], ref["y_scale"], "y")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", [[60, 30, 45], [2500, 10, 1500]])
def test_norm_keeps_nan_to_its_segment_and_group(sizes, dtype):
    g = gen(4)
    m = sum(sizes)
    X, G = normal(g, m, 24, dtype=dtype), normal(g, m, 24, dtype=dtype)
    X[sizes[0] + 2, 9] = float("nan")                        # segment 1, group 1 of 3
    X[m - 1, 23] = float("inf")                              # segment 2, group 2
    bad = torch.zeros(m, 24, dtype=torch.bool, device="cuda")
    bad[sizes[0]:sizes[0] + sizes[1], 8:16], bad[sizes[0] + sizes[1]:, 16:] = True, True
    seg = offsets(sizes)
    Y, mean, rstd = sagnn.group_norm_act(X, 3, seg=seg, max_rows=max(sizes), act=sagnn.ACT_RELU)
    assert torch.equal(Y.isnan(), bad)
    dX, dgamma, dbeta = sagnn.group_norm_act_bwd(X, G, mean, rstd, 3, seg=seg, max_rows=max(sizes))
    assert torch.equal(dX.isnan(), bad)
    assert torch.equal(dgamma.isnan(), torch.arange(24, device="cuda") >= 8) and bool(dbeta.isfinite().all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("sizes", [[50, 20, 33], [3000, 200]])
def test_norm_on_slices_and_in_place(sizes, shift, dtype):
    g = gen(shift)
    m, c = sum(sizes), 72
    wide = normal(g, m, c + 9, dtype=dtype)
    X = wide[:, shift:shift + c]
    seg, gamma, beta = offsets(sizes), normal(g, c), normal(g, c)
    kw = dict(seg=seg, max_rows=max(sizes), act=sagnn.ACT_SILU)
    dense = X.contiguous()
    expected, mean, rstd = sagnn.group_norm_act(dense, 9, gamma, beta, **kw)
    G = normal(g, m, c + 5, dtype=dtype)[:, 3:3 + c]
    grads = sagnn.group_norm_act_bwd(dense, G.contiguous(), mean, rstd, 9, gamma, beta, **kw)
    got = sagnn.group_norm_act_bwd(X, G, mean, rstd, 9, gamma, beta, **kw)
    assert all(torch.equal(a, b) for a, b in zip(grads, got))
    before = wide.clone()
    Y, mean2, rstd2 = sagnn.group_norm_act(X, 9, gamma, beta, out=X, **kw)      # over its input
    assert torch.equal(Y, expected) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    assert torch.equal(wide[:, :shift], before[:, :shift]) and torch.equal(wide[:, shift + c:], before[:, shift + c:])
    dX, _, _ = sagnn.group_norm_act_bwd(dense, G, mean, rstd, 9, gamma, beta, out=G, **kw)
    assert torch.equal(dX, grads[0])


@pytest.mark.parametrize("rows", [30, 4000])
@pytest.mark.parametrize("act", [sagnn.ACT_IDENTITY, sagnn.ACT_SILU])
def test_norm_gradients_against_differences(act, rows):
    """Central differences of the loss <G, Y>.  Their error: the third derivative times e^2, and the loss's rounding over e."""
    g = gen(8)
    c, groups, seg = 32, 4, offsets([rows, rows // 2])
    m = rows + rows // 2
    X, G, gamma, beta = normal(g, m, c), normal(g, m, c), normal(g, c) + 1.0, normal(g, c)
    kw = dict(seg=seg, max_rows=rows, act=act)
    _, mean, rstd = sagnn.group_norm_act(X, groups, gamma, beta, **kw)
    dX, dgamma, dbeta = sagnn.group_norm_act_bwd(X, G, mean, rstd, groups, gamma, beta, **kw)

    def loss(X, gamma, beta):
        return float((sagnn.group_norm_act(X, groups, gamma, beta, **kw)[0].double() * G.double()).sum())

    e = 1e-2
    for at, grad in enumerate((dX, dgamma, dbeta)):
        d = normal(g, *grad.shape)
        args = [X, gamma, beta]
        up, down = [list(args), list(args)]
        up[at], down[at] = args[at] + e * d, args[at] - e * d
        diff, exact = (loss(*up) - loss(*down)) / (2 * e), float((grad.double() * d.double()).sum())
        size = float((G.abs().double() * 1.0).norm()) * float(d.double().norm()) / (1.0 if at == 0 else 1.0)
        assert abs(diff - exact) <= 10 * e * e * size + 1e-3 * abs(exact), (at, diff, exact)


# ---------------------------------------------------------------------------------------------
# clipping

def tensors(g, sizes, kinds, shift=0):
    out = []
    for i, n in enumerate(sizes):
        kind = kinds[i % len(kinds)]
        out.append(normal(g, n + shift + 4, dtype=kind)[shift:shift + n])
    return out


F, B = torch.float32, torch.bfloat16


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("sizes,kinds", [([1], [F]), ([0, 5, 0], [B]), ([16384, 16385, 16383, 1], [F, B]), ([100001, 7, 0, 3000], [F]),
                                         ([3, 17, 1000] * 130, [F, B, B]), ([700000], [B]), ([40000] * 125, [F])])
def test_clipping(sizes, kinds, shift):
    g = gen(len(sizes))
    grads = tensors(g, sizes, kinds, shift)
    norm64 = sum(float(t.double().square().sum()) for t in grads) ** 0.5
    norm = sagnn.grad_global_norm(grads)
    assert norm.shape == (1,) and abs(float(norm) - norm64) <= 2 * U * norm64
    for ratio in (0.3, 1.7):
        out = [torch.full_like(t, 7.0) for t in grads]
        before = [t.clone() for t in grads]
        n2 = sagnn.grad_clip_norm(grads, ratio * norm64, out=out)
        assert torch.equal(n2, norm)
        given = [torch.empty_like(t) for t in grads]
        assert sagnn.grad_clip_norm(grads, ratio * norm64, norm=norm, out=given) is norm
        c = min(1.0, ratio)
        for t, b, o, p in zip(grads, before, out, given):
            assert torch.equal(t, b)
            ref = t.double() * c
            close(o, ref, 4 * U * ref.abs() + (rounding(t.dtype, ref) if ratio < 1 else 0.0) + 1e-45, "out")
            close(p, ref, 4 * U * ref.abs() + (rounding(t.dtype, ref) if ratio < 1 else 0.0) + 1e-45, "out, norm given")
        whole = [t.clone() for t in grads]
        sagnn.grad_clip_norm(whole, ratio * norm64)
        assert all(torch.equal(a, b) for a, b in zip(whole, out))


@pytest.mark.parametrize("count", [211, 212, 213, 318, 319, 640])
def test_clipping_of_as_many_tensors_as_a_launch_takes_and_more(count):
    g = gen(count)
    sizes = [(i * 37) % 301 + 1 if i % 11 else 0 for i in range(count + count // 10)]       # (a tensor of no values takes no place)
    grads = tensors(g, sizes, [F, B, F])
    norm64 = sum(float(t.double().square().sum()) for t in grads) ** 0.5
    out, whole = [torch.empty_like(t) for t in grads], [t.clone() for t in grads]
    half = [w if i % 2 else torch.empty_like(w) for i, w in enumerate(whole)]               # (some in place, some not)
    norm = sagnn.grad_clip_norm(grads, 0.5 * norm64, out=out)
    assert abs(float(norm) - norm64) <= 2 * U * norm64
    for t, o in zip(grads, out):
        ref = t.double() * 0.5
        close(o, ref, 4 * U * ref.abs() + rounding(t.dtype, ref) + 1e-45, "out")
    sagnn.grad_clip_norm([w if i % 2 else t for i, (w, t) in enumerate(zip(whole, grads))], 0.5 * norm64, out=half)
    assert all(torch.equal(a, b) for a, b in zip(half, out))
    whole = [t.clone() for t in grads]
    sagnn.grad_clip_norm(tuple(whole), 0.5 * norm64)
    assert all(torch.equal(a, b) for a, b in zip(whole, out))


def test_lists_of_gradients_are_read_alike_in_both_ways():
    g = gen(3)
    grads = tensors(g, [5, 0, 300, 17], [F, B], 1)
    out = [torch.empty_like(t) for t in grads]
    ext = binding._extension("_gradlist", binding._build.GRADLIST)
    assert ext is not None
    for o in (None, out, grads):
        assert ext.rows(grads, o) == binding._rows_in_python(grads, o)
    assert ext.rows([], None) == binding._rows_in_python([], None) == b""
    t = grads[0]
    wrong = [([t.double()], None), ([t.cpu()], None), ([normal(g, 4, 6)[:, 1:3]], None), ([t], []), ([t], out[:2]), ([t], [t.cpu()]),
             ([t], [out[0][1:]]), ([t], [out[0].bfloat16()]), ([normal(g, 4, 6)], [normal(g, 6, 4).t()])]
    for rows in (ext.rows, binding._rows_in_python):
        for a in wrong:
            with pytest.raises(ValueError):
                rows(*a)
    with pytest.raises(ValueError):
        ext.rows([1], None)
    for call in (lambda: sagnn.grad_global_norm(x for x in grads), lambda: sagnn.grad_clip_norm((x.clone() for x in grads), 1.0)):
        assert float(call()) == pytest.approx(float(sagnn.grad_global_norm(grads)), rel=1e-6)


def test_clipping_writes_nothing_beside_its_tensors():
    flat = torch.arange(1, 5001, dtype=F, device="cuda")
    grads = [flat[1:2], flat[5:1000], flat[1001:1001], flat[1003:4999]]
    before = flat.clone()
    sagnn.grad_clip_norm(grads, 1.0)
    for i in (0, 2, 3, 4, 1000, 1001, 1002, 4999):
        assert flat[i] == before[i]
    assert abs(float(sagnn.grad_global_norm(grads)) - 1.0) < 1e-6


def test_clipping_of_values_beyond_the_range_of_their_squares():
    big, small = torch.full((1000,), 1e30, device="cuda"), torch.full((1000,), 1e-30, device="cuda")
    assert float(sagnn.grad_global_norm([big])) == pytest.approx(1e30 * 1000 ** 0.5, rel=1e-6)
    assert float(sagnn.grad_global_norm([small])) == pytest.approx(1e-30 * 1000 ** 0.5, rel=1e-6)
    sagnn.grad_clip_norm([big], 2.0)
    assert float(sagnn.grad_global_norm([big])) == pytest.approx(2.0, rel=1e-6)


def test_clipping_of_zeros_infinities_and_nan():
    zeros = torch.zeros(50, device="cuda")
    assert float(sagnn.grad_clip_norm([zeros], 1.0)) == 0.0 and not zeros.any()
    a, b = torch.tensor([1.0, float("inf")], device="cuda"), torch.ones(3, device="cuda")
    assert float(sagnn.grad_clip_norm([a, b], 1.0)) == float("inf")
    assert a[0] == 0.0 and bool(a[1].isnan()) and not b.any()
    a, b = torch.tensor([1.0, float("nan")], device="cuda"), torch.ones(3, device="cuda")
    assert bool(sagnn.grad_clip_norm([a, b], 1.0).isnan()) and bool(a.isnan().all()) and bool(b.isnan().all())
    assert float(sagnn.grad_global_norm([])) == 0.0 and float(sagnn.grad_clip_norm([], 1.0)) == 0.0


# ---------------------------------------------------------------------------------------------
# all of them

def _step(seed):
    """One pass of everything, on inputs of its own."""
    g = gen(seed)
    off = offsets([700, 0, 1500, 300])
    X, W, G = normal(g, 2500, 96, dtype=B), normal(g, 4, 96, 128, dtype=B), normal(g, 2500, 128, dtype=B)
    gamma, beta = normal(g, 128), normal(g, 128)

    def run():
        Y = sagnn.grouped_gemm_act(X, W, off)
        N, mean, rstd = sagnn.group_norm_act(Y, 8, gamma, beta, seg=off, act=sagnn.ACT_RELU)
        dY, dgamma, dbeta = sagnn.group_norm_act_bwd(Y, G, mean, rstd, 8, gamma, beta, seg=off, act=sagnn.ACT_RELU)
        dX, dW = sagnn.grouped_gemm_bwd(X, W, off, dY)
        clipped = [torch.empty_like(t) for t in (dW, dgamma, dbeta)]
        norm = sagnn.grad_clip_norm([dW, dgamma, dbeta], 1.0, out=clipped)
        return [Y, N, mean, rstd, dX, norm, *clipped]

    return run


def test_operators_give_the_same_bits_every_time_and_on_any_stream():
    run = _step(1)
    first = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_operators_in_a_graph():
    run, other = _step(2), _step(3)
    eager = [t.clone() for t in run()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = run()
    for _ in range(3):
        for t in recorded:
            t.zero_()
        other()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, recorded))
