"""A training step of the typed network against the same step in 64 bits (dense matrices, torch's differentiation), and a few
steps that have to learn."""
import numpy as np
import pytest
import torch

import paper_2504_04673_amd as sagnn
from paper_2504_04673_amd import typed_gcn

pytestmark = pytest.mark.gpu


def dense(graph):
    n = graph.n
    A = torch.zeros(n, n, dtype=torch.float64, device="cuda")
    rows = torch.repeat_interleave(torch.arange(n, device="cuda"), graph.rowptr.diff().long())
    A.index_put_((rows, graph.colidx.long()), graph.val.double(), accumulate=True)
    return A


def reference(net, graph, H, target):
    """Loss and gradients of all parameters."""
    A, off = dense(graph), graph.off.tolist()
    params = [p.double().requires_grad_() for p in net.parameters()]
    layers, hidden = len(net.W), len(net.gamma)
    h = H.double()
    for i in range(layers):
        t = A @ h
        z = torch.cat([t[a:b] @ params[i][g] for g, (a, b) in enumerate(zip(off[:-1], off[1:]))])
        if i + 1 == layers:
            break
        parts = []
        for a, b in zip(off[:-1], off[1:]):
            v = z[a:b].reshape(b - a, net.n_groups, -1)
            mean = v.mean((0, 2), keepdim=True)
            parts.append(((v - mean) * ((v - mean).square().mean((0, 2), keepdim=True) + 1e-5).rsqrt()).reshape(b - a, -1))
        h = torch.relu(torch.cat(parts) * params[layers + i] + params[layers + hidden + i])
    loss = (z - target.double()).square().mean()
    loss.backward()
    return float(loss.detach()), [p.grad for p in params]


@pytest.mark.parametrize("prec", [sagnn.GEMM_FP32, sagnn.GEMM_FP32_BF16X3])
def test_training_step_of_a_typed_network(prec):
    graph, H, target = typed_gcn.synthetic(700, 5, 32, 8, seed=3)
    net = typed_gcn.TypedGCN(graph, (32, 64, 48, 8), n_groups=4, prec=prec, seed=1)
    loss, grads = reference(net, graph, H, target)
    out, kept = net.forward(H)
    diff = out - target
    assert float(diff.square().mean()) == pytest.approx(loss, rel=1e-5)
    got = net.backward(diff * (2.0 / diff.numel()), kept)
    # a handful of roundings of 2^-24 a layer, sums of some thousand terms: 1e-4 of each gradient's norm; ReLU's slope is
    # taken at values that differ by rounding, a few of 75,000 of them
    for g, r in zip(got, grads):
        assert g.shape == r.shape
        assert float((g.double() - r).norm()) <= 1e-3 * float(r.norm()) + 1e-12
    before = [p.clone() for p in net.parameters()]
    norm64 = float(sum(r.square().sum() for r in grads)) ** 0.5
    step_loss, norm = net.step(H, target, rate=0.5, max_norm=0.5 * norm64)
    assert float(norm) == pytest.approx(norm64, rel=1e-3)
    for p, b, r in zip(net.parameters(), before, grads):
        assert float((p.double() - (b.double() - 0.25 * r)).norm()) <= 1e-3 * float(r.norm()) + 1e-6 * float(b.double().norm())


def test_typed_network_learns():
    graph, H, target = typed_gcn.synthetic(5000, 6, 32, 8, seed=4)
    net = typed_gcn.TypedGCN(graph, (32, 64, 8), seed=2)
    losses = [float(net.step(H, target, rate=1.0)[0]) for _ in range(40)]
    assert all(np.isfinite(losses)) and losses[-1] < 0.9 * losses[0]
