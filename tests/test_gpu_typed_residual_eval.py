"""Gradients of the residual network behind a forward pass that drew no masks, or masks of another share than the network has by then."""
import pytest
import torch

import paper_2504_04673_amd as sagnn
from paper_2504_04673_amd import typed_gcn
from tests.test_gpu_typed_residual import reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("training", [False, True])
def test_backward_is_of_the_forward_pass_that_was(training):
    graph, H, labels, count = typed_gcn.synthetic_classes(700, 5, 36, 11, seed=3)
    net = typed_gcn.TypedResidualGCN(graph, 36, 64, 2, 11, p=0.3, p_in=0.2, seed=1)
    Y, kept = net.forward(H, 7, training=training)
    loss, lse = sagnn.softmax_xent(Y, net.head, labels, bias=net.bias, transW=True)
    G, dhead, dbias = sagnn.softmax_xent_bwd(Y, net.head, labels, lse, 1.0 / count, bias=net.bias, transW=True)
    net.p, net.p_in = (0.7, 0.7) if training else (net.p, net.p_in)
    got = net.backward(G, kept, 7, dhead, dbias)
    net.p, net.p_in = (0.3, 0.2) if training else (0.0, 0.0)
    ref, grads, _ = reference(net, graph, H, labels, count, 7)
    assert float(loss.sum() / count) == pytest.approx(ref, rel=1e-5)
    # as for a training step: a few of 90,000 values lie on the other side of ReLU's corner
    for g, r in zip(got, grads):
        assert float((g.double() - r).norm()) <= 1e-3 * float(r.norm()) + 1e-12
