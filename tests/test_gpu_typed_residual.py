"""The residual network over typed vertices: its loss and gradients against the same network in 64 bits (dense matrices, torch's differentiation, the
masks of the plain generator), a step that is captured and replayed, and its rows in 8 bits."""
import pytest
import torch

import paper_2504_04673_amd as sagnn
from paper_2504_04673_amd import typed_gcn
from tests.philox import kept
from tests.test_gpu_typed_gcn import dense

pytestmark = pytest.mark.gpu


def reference(net, graph, H, labels, count, step):
    """Loss and gradients of all parameters."""
    A, off = dense(graph), graph.off.tolist()
    parts = list(zip(off[:-1], off[1:]))
    params = [p.double().requires_grad_() for p in net.parameters()]
    n = len(net.W1)

    def drop(x, p, seed):
        return torch.where(torch.from_numpy(kept(*x.shape, p, seed, step)).cuda(), x * (65536.0 / (65536 - int(p * 65536 + 0.5))), 0.0) if p else x

    def norm(s, gamma):
        return s * (s.square().mean(1, keepdim=True) + 1e-6).rsqrt() * gamma

    s = drop(H.double(), net.p_in, net.seed)
    y = norm(s, params[2 * n])
    for i in range(n):
        t = A @ y
        u = torch.relu(torch.cat([t[a:b] @ params[i][g] for g, (a, b) in enumerate(parts)]))
        z = torch.cat([u[a:b] @ params[n + i][g] for g, (a, b) in enumerate(parts)])
        s = s + drop(z, net.p, net.seed + 1 + i)
        y = norm(s, params[2 * n + 1 + i])
    logits = y @ params[-2].t() + params[-1]
    has = labels >= 0
    loss = (torch.logsumexp(logits, 1) - logits.gather(1, labels.clamp(min=0).long()[:, None])[:, 0])[has].sum() / count
    loss.backward()
    return float(loss.detach()), [p.grad for p in params], y.detach()


@pytest.mark.parametrize("prec", [sagnn.GEMM_FP32, sagnn.GEMM_FP32_BF16X3])
@pytest.mark.parametrize("p,p_in", [(0.3, 0.2), (0.0, 0.0)])
def test_training_step_of_a_residual_network(prec, p, p_in):
    graph, H, labels, count = typed_gcn.synthetic_classes(700, 5, 36, 11, seed=3)
    net = typed_gcn.TypedResidualGCN(graph, 36, 64, 2, 11, p=p, p_in=p_in, prec=prec, seed=1)
    ref, grads, y = reference(net, graph, H, labels, count, 7)
    loss, got = net.gradients(H, labels, count, 7)
    assert float(loss.sum() / count) == pytest.approx(ref, rel=1e-5)
    # a handful of roundings of 2^-24 a block, sums of some thousand terms; ReLU's slope is taken at values that differ by rounding, a few of
    # 90,000 of them: 1e-3 of each gradient's norm
    for g, r in zip(got, grads):
        assert g.shape == r.shape
        assert float((g.double() - r).norm()) <= 1e-3 * float(r.norm()) + 1e-12
    before = [q.clone() for q in net.parameters()]
    norm64 = float(sum(r.square().sum() for r in grads)) ** 0.5
    step_loss, norm = net.step(H, labels, count, 7, rate=0.5, max_norm=0.5 * norm64)
    assert float(norm) == pytest.approx(norm64, rel=1e-3) and float(step_loss) == pytest.approx(ref, rel=1e-5)
    for q, b, r in zip(net.parameters(), before, grads):
        assert float((q.double() - (b.double() - 0.25 * r)).norm()) <= 1e-3 * float(r.norm()) + 1e-6 * float(b.double().norm())


def test_captured_step_of_a_residual_network():
    """The gradients of a step in a graph whose step number it counts up itself, between eager steps of other numbers."""
    graph, H, labels, count = typed_gcn.synthetic_classes(3000, 4, 64, 200, seed=5)
    net = typed_gcn.TypedResidualGCN(graph, 64, 96, 2, 200, p=0.2, p_in=0.1, seed=9)
    number = torch.zeros(1, dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        net.gradients(H, labels, count, number)
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured, stream=side):
            loss, grads = net.gradients(H, labels, count, number)
            number.add_(1)
    torch.cuda.current_stream().wait_stream(side)
    number.fill_(40)
    for i in range(4):
        captured.replay()
        torch.cuda.synchronize()
        ref_loss, ref = net.gradients(H, labels, count, 40 + i)
        assert torch.equal(loss, ref_loss) and all(torch.equal(a, b) for a, b in zip(grads, ref))
        net.gradients(H, labels, count, 3)


def test_rows_in_8_bits():
    graph, H, labels, count = typed_gcn.synthetic_classes(700, 5, 36, 11, seed=6)
    net = typed_gcn.TypedResidualGCN(graph, 36, 64, 2, 11, p=0.5, p_in=0.5, seed=2)
    Q, scale = net.rows_e4m3(H)
    rows = torch.tensor([5, 699, 0, 5], dtype=torch.int32, device="cuda")
    got = sagnn.spmm_pack_rows_e4m3(Q, scale, rows)
    net.p = net.p_in = 0.0
    y = reference(net, graph, H, labels, count, 0)[2][rows.long()]
    # half a step of e4m3: 2^-4 of a value, 2^-10 of the scale below its normal values; the network's own roundings 1e-4
    assert torch.all((got.double() - y).abs() <= 2.0 ** -4 * y.abs() + (2.0 ** -10 * scale[rows.long()].double())[:, None] + 1e-4 * y.abs().amax())


def test_the_command_runs(capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["typed_gcn", "--vertices", "3000", "--types", "3", "--steps", "2", "--classes", "17"])
    typed_gcn.main()
    assert capsys.readouterr().out.count("loss") == 2
