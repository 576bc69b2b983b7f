"""Gradients of the norm's affine map over many rows: equal terms, whose additions may all round the same way, stay within 1e-5 of
the sum of their absolute values, however the rows lie in segments."""
import pytest
import torch

import paper_2504_04673_amd as sagnn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,c,rows,known", [
    (4_000_000, 512, 4_000_000, 0),           # one segment in parts, wide: a thread has every row of its part
    (2_500_000, 1024, 1_250_000, 0),
    (40_000_000, 8, 40_000_000, 0),
    (3_000_000, 8, 1, 0),                     # parts with thousands of segments each
    (3_000_001, 12, 3, 0),
    (6_000_000, 8, 2, 2),                     # whole segments, thousands for each workgroup
    (3_000_000, 64, 3_000_000, 1),            # a whole segment far longer than the caller said
])
def test_equal_gradients(m, c, rows, known, dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    X = torch.randn(m, c, generator=g, device="cuda", dtype=torch.float32).to(dtype)
    seg = torch.cat([torch.arange(0, m, rows, device="cuda"), torch.tensor([m], device="cuda")]).to(torch.int32)
    n_seg = seg.numel() - 1
    G = torch.empty(m, c, dtype=dtype, device="cuda")
    # mean 0 and rstd 1: dgamma sums x, too, here made of equal terms in half of the channels
    X[:, ::2] = 0.7
    mean, rstd = torch.zeros(n_seg, 1, device="cuda"), torch.ones(n_seg, 1, device="cuda")
    for value in (0.1, 1 / 3, 1.3, 1.9921875):
        G.fill_(value)
        v, x = float(G[0, 0]), float(X[0, 0])
        _, dgamma, dbeta = sagnn.group_norm_act_bwd(X, G, mean, rstd, 1, seg=seg, max_rows=known)
        assert bool(((dbeta.double() - m * v).abs() <= 1e-5 * m * v).all()), (value, float((dbeta.double() / (m * v) - 1).abs().max()))
        sums = dgamma.double()[::2]
        assert bool(((sums - m * v * x).abs() <= 1e-5 * m * v * x).all()), (value, float((sums / (m * v * x) - 1).abs().max()))
