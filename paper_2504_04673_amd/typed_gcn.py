"""A graph network over vertices of several types, trained on one GPU: every layer aggregates (sparse product), multiplies by
the weights of the vertex's type, normalises over the vertices of each type and applies ReLU; the last one ends
with the product.  All of it, gradients and clipping included, runs in the library's kernels; torch holds the tensors, takes
the loss's gradient and subtracts.

    T = A H,  Z[r] = T[r] W[type(r)],  H' = ReLU(group_norm(Z))

    python -m paper_2504_04673_amd.typed_gcn [--vertices N] [--types K] [--steps S]

makes a random graph with random types, orders its vertices by type (spmm_perm_from_labels) and prints the loss,
the gradients' norm and the time of each step.
"""
from __future__ import annotations

import argparse
import time
from dataclasses import dataclass

import numpy as np
import torch

from . import binding as sagnn


@dataclass
class TypedGraph:
    """A symmetric matrix whose rows are ordered by type, prepared for products of a few widths."""
    rowptr: torch.Tensor
    colidx: torch.Tensor
    val: torch.Tensor
    off: torch.Tensor             # int32, types + 1: the rows of each type
    perm: torch.Tensor            # old number of each row
    inv: torch.Tensor             # row of each old number

    @classmethod
    def order(cls, rowptr, colidx, val, labels, n_types):
        """From CSR on the device and a type (int32) for each vertex."""
        perm, inv, off = sagnn.spmm_perm_from_labels(labels, n_types)
        rows = sagnn.spmm_csr_permute_symmetric(rowptr, colidx, val, inv)
        return cls(*rows, torch.from_numpy(off.astype(np.int32)).to(labels.device), perm, inv)

    @property
    def n(self) -> int:
        return self.rowptr.numel() - 1

    def multiply(self, H, ws):
        return sagnn.spmm_csr_tallskinny(self.rowptr, self.colidx, self.val, H, ws=ws)

    def prepare(self, f):
        return sagnn.spmm_csr_prepare(self.rowptr, self.colidx, self.val, self.n, f)


class TypedGCN:
    """Layers of the given widths over the types of `graph`, hidden ones normalised in groups of channels.  The rows are
    normalised type by type: a type's rows are one segment, so that each type has statistics of its own."""

    def __init__(self, graph: TypedGraph, widths, n_groups=4, prec=sagnn.GEMM_FP32, seed=0):
        self.graph, self.n_groups, self.prec = graph, n_groups, prec
        dev, types = graph.off.device, graph.off.numel() - 1
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.W = [torch.randn((types, a, b), generator=gen, device=dev) * a ** -0.5 for a, b in zip(widths[:-1], widths[1:])]
        self.gamma = [torch.ones(b, device=dev) for b in widths[1:-1]]
        self.beta = [torch.zeros(b, device=dev) for b in widths[1:-1]]
        self.ws = {f: graph.prepare(f) for f in set(widths[:-1])}
        self.longest = int((graph.off[1:] - graph.off[:-1]).max())

    def parameters(self):
        return [*self.W, *self.gamma, *self.beta]

    def forward(self, H):
        """Output and what the backward pass needs of each layer: (T, Z, mean, rstd)."""
        kept = []
        for i, W in enumerate(self.W):
            T = self.graph.multiply(H, self.ws[W.shape[1]])
            Z = sagnn.grouped_gemm_act(T, W, self.graph.off, prec=self.prec)
            if i + 1 == len(self.W):
                kept.append((T, Z, None, None))
                return Z, kept
            H, mean, rstd = sagnn.group_norm_act(Z, self.n_groups, self.gamma[i], self.beta[i], seg=self.graph.off,
                                                 max_rows=self.longest, act=sagnn.ACT_RELU)
            kept.append((T, Z, mean, rstd))

    def backward(self, G, kept):
        """Gradients in the order of parameters(), from G = dLoss/d(output).  The graph's matrix is symmetric, so the product
        with its transpose is the product with itself."""
        dW, dgamma, dbeta = [None] * len(self.W), [None] * len(self.gamma), [None] * len(self.beta)
        for i in reversed(range(len(self.W))):
            T, Z, mean, rstd = kept[i]
            if i + 1 < len(self.W):
                G, dgamma[i], dbeta[i] = sagnn.group_norm_act_bwd(Z, G, mean, rstd, self.n_groups, self.gamma[i], self.beta[i],
                                                                  seg=self.graph.off, max_rows=self.longest, act=sagnn.ACT_RELU)
            dT, dW[i] = sagnn.grouped_gemm_bwd(T, self.W[i], self.graph.off, G, prec=self.prec, want_dx=i > 0)
            if i > 0:
                G = self.graph.multiply(dT, self.ws[dT.shape[1]])
        return [*dW, *dgamma, *dbeta]

    def step(self, H, target, rate=0.05, max_norm=1.0):
        """One step of gradient descent on the mean squared error.  Returns (loss, norm of the gradients before they were
        clipped), both on the device."""
        out, kept = self.forward(H)
        diff = out - target
        grads = self.backward(diff * (2.0 / diff.numel()), kept)
        norm = sagnn.grad_clip_norm(grads, max_norm)
        for p, g in zip(self.parameters(), grads):
            p.sub_(g, alpha=rate)
        return diff.square().mean(), norm


def synthetic(n, n_types, f, f_out, degree=8, seed=0):
    """A random graph with random types on the GPU, its rows ordered by type: (graph, H, target)."""
    from . import synth
    g = synth.er_graph(n, degree, seed)
    rng = np.random.default_rng(seed)
    csr = [torch.from_numpy(a).cuda() for a in (g.rowptr, g.colidx, g.val)]
    graph = TypedGraph.order(*csr, torch.from_numpy(rng.integers(0, n_types, n).astype(np.int32)).cuda(), n_types)
    H = sagnn.spmm_pack_rows(torch.from_numpy(synth.normal((n, f), seed, synth.STREAM_H)).cuda(), graph.perm)
    # something to learn: a linear map of each type
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    target = sagnn.grouped_gemm_act(H, torch.randn((n_types, f, f_out), generator=gen, device="cuda") * f ** -0.5, graph.off)
    return graph, H, target


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--vertices", type=int, default=100_000)
    ap.add_argument("--types", type=int, default=8)
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args()
    graph, H, target = synthetic(args.vertices, args.types, 64, 16)
    net = TypedGCN(graph, (64, 128, 128, 16))
    for step in range(args.steps):
        t = time.perf_counter()
        loss, norm = net.step(H, target)
        loss, norm = float(loss), float(norm)
        print(f"step {step}: loss {loss:.5f}, norm {norm:.5f}, {(time.perf_counter() - t) * 1e3:.2f} ms", flush=True)


if __name__ == "__main__":
    main()
