"""Weights of the rows in the cross entropy's gradients where products take bfloat16 operands: the weights themselves meet no rounding to bfloat16.

Tolerances (u = 2^-24): a weight on dH's rows 2 u; on dW's products 2^-16 of each term (two bfloat16 terms: what the first leaves is 2^-8 of the value at most, and is
rounded by 2^-8 of that), sums 4e-5, together 6e-5; P's own rounding half a step of bfloat16, a result's the same, 2^-8 |.| at most.
The norms, logits of deviation 2 and n classes: p of a label is m e^(2 x), x normal, m = 1 / (n e^2).  A label's P lies between a half and one, in steps of 2^-8: it is off by
p where p < c = 2^-9, and uniformly by c at most elsewhere.  n = 2000: m^2 e^8 Phi(1.68 - 4) + c^2 (1 - Phi(1.68)) = 0.00056^2; the other classes' p, rounded by 0.0016 of
themselves in the mean square, 0.0016 sqrt(sum of p^2 <= e^4 / n) = 0.00027; the result's own rounding 0.0016: 1.07 times that in all, 1.1 allowed.  n = 172: 0.00088 and, with a sum of p^2 of
a tenth, 0.0005: 1.18, 1.25 allowed.  dW has the label's part in one row of 172 and the others' in all: less than dH, 1.1 allowed.
"""
import ctypes

import pytest
import torch

import paper_2504_04673_amd as sagnn
from paper_2504_04673_amd import binding
from tests.test_gpu_row_operators import close, gen, normal
from tests.test_gpu_xent import PREC, Plain, inputs, unrounded

pytestmark = pytest.mark.gpu
MODES = ["bf16", "rounded"]


def held(mode, t):
    """Values of bfloat16 in the mode's type, so that products round none of them."""
    return t if mode == "bf16" else t.float()


@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("m,k,n,labelled", [(3000, 100, 1024, 1.0), (1100, 72, 4096, 1.0), (6000, 64, 1024, 0.6)])
@pytest.mark.parametrize("mode", MODES)
def test_equal_weights_are_not_rounded(mode, m, k, n, labelled, trans):
    """H of zeros or W of zeros: p = 1 / n, a power of two, and a label's P is off by 1 / n.  The weight 1 + 2^-8 lies halfway between two bfloat16 values:
    rounded, all terms would be off by 2^-8."""
    H, W, labels, _ = inputs(m, m, k, n, torch.bfloat16, False, False, labelled, False)
    H, W = held(mode, H), held(mode, W)
    g = torch.full((m,), 1.0 + 2.0 ** -8, device="cuda")
    last = 2.0 ** -8 if mode == "bf16" else 2.0 ** -23
    known = (labels >= 0) & (labels < n)
    for h, w in ((H, torch.zeros_like(W)), (torch.zeros_like(H), W)):
        w_ = w.t().contiguous() if trans else w
        _, lse = sagnn.softmax_xent(h, w_, labels, transW=trans, prec=PREC[mode])
        dH, dW, _ = sagnn.softmax_xent_bwd(h, w_, labels, lse, g, transW=trans, prec=PREC[mode])
        rH, rW, aH, aW = unrounded(h[known], w, labels[known], 1.0 + 2.0 ** -8)
        close(dH[known], rH, last * rH.abs() + (1.0 / n + 6e-5) * aH, "dH")
        close(dW.t() if trans else dW, rW, last * rW.abs() + (1.0 / n + 6e-5) * aW, "dW")
        assert not dH[~known].any()


def off(got, ref):
    return float((got.double() - ref).norm() / ref.norm())


@pytest.mark.parametrize("kind", ["none", "random", "equal", "by class"])
@pytest.mark.parametrize("m,k,n,times_h,times_w", [(3000, 256, 2000, 1.1, 1.1), (20000, 128, 172, 1.25, 1.1)])
def test_weighted_gradients_err_as_unweighted_ones_do(m, k, n, times_h, times_w, kind):
    H, W, labels, bias = inputs(m, m, k, n, torch.bfloat16, False, True, 1.0, False)
    r = gen(7)
    g = {"none": 1.0 + 2.0 ** -8, "random": torch.rand(m, generator=r, device="cuda"), "equal": torch.full((m,), 1.0 + 2.0 ** -8, device="cuda"),
         "by class": torch.rand(n, generator=r, device="cuda")[labels.long()]}[kind]
    _, lse = sagnn.softmax_xent(H, W, labels, bias=bias)
    dH, dW, _ = sagnn.softmax_xent_bwd(H, W, labels, lse, g, bias=bias)
    rH, rW, _, _ = unrounded(H, W, labels, g, bias)
    assert off(dH, rH) <= times_h * off(rH.bfloat16(), rH)
    assert off(dW, rW) <= times_w * off(rW.bfloat16(), rW)


@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("mode", [*MODES, "fp32", "x3"])
def test_both_factors_and_weights_of_zero(mode, trans):
    """grad_all and d_grad together, as the library takes them: the call with their product; rows of weight 0 have no part."""
    m, k, n = 2500, 40, 300
    H, W, labels, bias = inputs(2, m, k, n, torch.bfloat16 if mode == "bf16" else torch.float32, trans, True, 0.7, False)
    g = torch.rand(m, generator=gen(3), device="cuda")
    g[::3] = 0
    _, lse = sagnn.softmax_xent(H, W, labels, bias=bias, transW=trans, prec=PREC[mode])
    want = sagnn.softmax_xent_bwd(H, W, labels, lse, 4.0 * g, bias=bias, transW=trans, prec=PREC[mode])
    dH, dW, dbias = torch.empty_like(H), torch.empty_like(W), torch.empty_like(bias)
    dtype, need = binding._DTYPE[H.dtype], ctypes.c_size_t(0)
    assert sagnn.lib().softmax_xent_workspace_bytes(dtype, m, k, n, PREC[mode], 1, ctypes.byref(need)) == 0
    ws = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    assert binding._calls().softmax_xent_bwd(dtype, H.data_ptr(), k, W.data_ptr(), W.shape[1], int(trans), bias.data_ptr(), labels.data_ptr(), lse.data_ptr(), g.data_ptr(),
                                             4.0, m, k, n, PREC[mode], dH.data_ptr(), k, dW.data_ptr(), dbias.data_ptr(), ws.data_ptr(), need.value,
                                             torch.cuda.current_stream().cuda_stream) == 0
    # (a power of two changes no rounding)
    assert torch.equal(dH, want[0]) and torch.equal(dW, want[1]) and torch.equal(dbias, want[2])
    assert not dH[::3].any()
    ref = Plain(H, W, labels, bias, trans, 4.0 * g, mode)
    close(dH, ref.dH, ref.dH_bound, "dH")
    close(dW, ref.dW, ref.dW_bound, "dW")
    close(dbias, ref.dbias, ref.dbias_bound, "dbias")


def test_weighted_step_captured_and_replayed():
    H, W, labels, bias = inputs(5, 1500, 64, 400, torch.bfloat16, True, True, 0.6, False)
    g = torch.rand(1500, generator=gen(1), device="cuda")

    def step():
        loss, lse = sagnn.softmax_xent(H, W, labels, bias=bias, transW=True)
        return (loss, lse, *sagnn.softmax_xent_bwd(H, W, labels, lse, g, bias=bias, transW=True))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        H.copy_(normal(gen(20 + i), 1500, 64, dtype=torch.bfloat16))
        g.copy_(torch.rand(1500, generator=gen(40 + i), device="cuda"))
        labels.copy_(torch.randint(-200, 400, (1500,), generator=gen(30 + i), device="cuda", dtype=torch.int32))
        ref = step()
        for t in got:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("m,k,n,labelled", [(20, 40, 4096, 1.0), (600, 72, 4096, 1.0), (3000, 100, 1024, 0.6), (2500, 512, 8192, 1.0), (40, 200, 65536, 1.0)])
def test_a_factor_of_all_rows_is_not_rounded_on_its_way_into_products(m, k, n, labelled, trans):
    """fp32 tensors whose products round operands: as for equal weights above."""
    H, W, labels, _ = inputs(m, m, k, n, torch.bfloat16, False, False, labelled, False)
    H, W, g = H.float(), W.float(), 1.0 + 2.0 ** -8
    known = (labels >= 0) & (labels < n)
    for h, w in ((H, torch.zeros_like(W)), (torch.zeros_like(H), W)):
        w_ = w.t().contiguous() if trans else w
        _, lse = sagnn.softmax_xent(h, w_, labels, transW=trans, prec=sagnn.GEMM_BF16)
        dH, dW, _ = sagnn.softmax_xent_bwd(h, w_, labels, lse, g, transW=trans, prec=sagnn.GEMM_BF16)
        rH, rW, aH, aW = unrounded(h[known], w, labels[known], g)
        close(dH[known], rH, (1.0 / n + 6e-5) * aH, "dH")
        close(dW.t() if trans else dW, rW, (1.0 / n + 6e-5) * aW, "dW")
    for g in (float("inf"), float("nan")):
        none = torch.full_like(labels, -1)
        assert not any(t.any() for t in sagnn.softmax_xent_bwd(H, w_, none, lse, g, transW=trans, prec=sagnn.GEMM_BF16)[:2])
