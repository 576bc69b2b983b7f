"""The operators of a typed, normalised GNN's training step, as cases that can be timed and checked.

  grouped product   rows ordered by type, a weight matrix for each type: forward, and the gradients of both operands
  group norm        mean and variance over the vertices of a graph and a group of channels, affine map, activation:
                    forward, and the gradients of input and affine map
  gradient clipping the global 2-norm over all gradient tensors of a model, and the tensors scaled to a bound on it

`listed()` names twelve cases, `draw(rng)` gives more of the same ranges, `prepare` makes the inputs on the GPU from a
seed, `run` is one pass: the plain form in elementary torch operations, or with `own` the library's calls.  `exact`
has the outputs in 64 bits.  Widths and vertex counts are those of the benchmark's graphs (16 to 602 features, thousands
to two million vertices) and, for the products that fill the matrix cores, powers of two.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
EPS = 1e-5


def listed():
    return [
        # a few seed vertices of eight types, inference: the call's latency is everything
        {"name": "types_96_fwd_bf16", "op": "gemm", "way": "fwd", "m": 96, "k": 256, "n": 256, "g": 8, "type": "bf16"},
        # a citation-sized graph with four vertex types, a hidden layer with ReLU: about as much arithmetic as traffic
        {"name": "types_170k_fwd_fp32", "op": "gemm", "way": "fwd", "m": 170003, "k": 128, "n": 128, "g": 4, "type": "fp32",
         "act": "relu"},
        # raw features of odd width, a relation for each of 41 labels, training in fp32 on the bf16 matrix cores
        {"name": "relations_30k_bwd_fp32x3", "op": "gemm", "way": "bwd", "m": 30011, "k": 602, "n": 256, "g": 41, "type": "fp32x3"},
        # many types and wide layers: arithmetic only
        {"name": "experts_32k_fwd_bf16", "op": "gemm", "way": "fwd", "m": 32768, "k": 2048, "n": 4096, "g": 64, "type": "bf16"},
        # a wide typed layer's backward pass, previous layer's ReLU mask applied
        {"name": "experts_16k_bwd_bf16", "op": "gemm", "way": "bwd", "m": 16384, "k": 2048, "n": 1024, "g": 16, "type": "bf16",
         "mask": True},
        # a batch of molecules: 128 graphs of some 24 vertices
        {"name": "molecules_fwd_fp32", "op": "norm", "way": "fwd", "m": 3007, "c": 64, "q": 8, "b": 128, "type": "fp32", "act": "relu"},
        # sixteen communities of a two-million-vertex graph, wide hidden layer
        {"name": "communities_2m_fwd_bf16", "op": "norm", "way": "fwd", "m": 2000000, "c": 256, "q": 32, "b": 16, "type": "bf16",
         "act": "silu"},
        # a whole citation-sized graph as one segment, training
        {"name": "graph_170k_bwd_fp32", "op": "norm", "way": "bwd", "m": 170003, "c": 100, "q": 4, "b": 1, "type": "fp32", "act": "relu"},
        # a batch of four thousand sampled subgraphs, training
        {"name": "subgraphs_1m_bwd_bf16", "op": "norm", "way": "bwd", "m": 1000000, "c": 256, "q": 16, "b": 4000, "type": "bf16",
         "act": "silu"},
        # the weights of a three-layer network
        {"name": "clip_6_small", "op": "clip", "tensors": 6, "total": 170000, "type": "fp32", "packed": False, "ratio": 0.5},
        # a typed network: some two hundred tensors of all sizes, in two types, packed without gaps into flat buffers
        {"name": "clip_211_mixed", "op": "clip", "tensors": 211, "total": 20000003, "type": "mixed", "packed": True, "ratio": 0.3},
        # the largest: gradients of half a billion weights
        {"name": "clip_64_500m", "op": "clip", "tensors": 64, "total": 500000000, "type": "bf16", "packed": False, "ratio": 0.1},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A third powers of two, a third multiples of 4, a third what the data gives."""
    r = rng.random()
    if r < 1 / 3:
        return 1 << rng.randint(math.ceil(math.log2(lo)), int(math.log2(hi)))
    w = _log(rng, lo, hi)
    return max(4, w // 4 * 4) if r < 2 / 3 else w


def draw(rng):
    op = rng.choice(["gemm", "gemm", "norm", "norm", "clip"])
    if op == "gemm":
        way, kind = rng.choice(["fwd", "bwd"]), rng.choice(["fp32", "fp32x3", "fp32_bf16", "bf16", "bf16"])
        k, n = _width(rng, 8, 4096), _width(rng, 8, 4096)
        # fp32 instructions do a sixteenth of the bf16 ones' work in a time
        most = 32768 * 2048 * 4096 // (16 if kind == "fp32" else 4 if kind == "fp32x3" else 1) // (2 if way == "bwd" else 1)
        return {"op": op, "way": way, "m": _log(rng, 1, max(2, min(1000000, most // (k * n), 500000000 // max(k, n)))), "k": k, "n": n,
                "g": _log(rng, 1, 64), "type": kind, "act": rng.choice(["none", "relu"]) if way == "fwd" else "none",
                "mask": way == "bwd" and rng.random() < 0.5, "trans": way == "fwd" and rng.random() < 0.3, "pad": rng.choice([0, 0, 37])}
    if op == "norm":
        d = rng.choice([1, 2, 3, 4, 8, 8, 16, 25, 32, 64])
        q = max(1, min(_log(rng, 1, 128), 1024 // d))
        m = _log(rng, 1, max(2, min(2000000, 500000000 // (d * q))))
        return {"op": op, "way": rng.choice(["fwd", "bwd"]), "m": m, "c": d * q, "q": q, "b": _log(rng, 1, max(2, min(20000, m // 4))),
                "type": rng.choice(["fp32", "bf16"]), "act": rng.choice(["none", "relu", "silu"])}
    return {"op": op, "tensors": _log(rng, 1, 400), "total": _log(rng, 1000, 250000000), "type": rng.choice(["fp32", "bf16", "mixed"]),
            "packed": rng.random() < 0.5, "ratio": rng.choice([0.1, 0.5, 0.9, 2.0])}


# ---------------------------------------------------------------------------------------------
# inputs

def _offsets(rng, total, parts, skew):
    """Ragged parts of `total` rows: sizes vary by a factor of up to about 1 + 2 skew around their mean, and one in
    sixteen or so is empty (where there are several)."""
    w = rng.uniform(1.0, 1.0 + 2.0 * skew, parts)
    if parts > 3:
        w[rng.random(parts) < 1 / 16] = 0.0
    if w.sum() == 0:
        w[:] = 1.0
    off = np.round(np.concatenate([[0.0], np.cumsum(w)]) / w.sum() * total).astype(np.int64)
    off[-1] = total
    return off


def _tensor_sizes(count, total):
    """Matrices and vectors of a model (the same for every seed): sizes over two decades that add up to `total`."""
    rng = np.random.default_rng(count)
    w = np.exp(rng.uniform(0.0, math.log(100.0), count))
    cut = np.round(np.concatenate([[0.0], np.cumsum(w)]) / w.sum() * total).astype(np.int64)
    cut[-1] = total
    return np.diff(cut)


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV).manual_seed(int(seed))

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return torch.randn(shape, generator=gen, device=DEV).mul_(scale).to(dtype)

    dtype = torch.bfloat16 if case["type"] == "bf16" else torch.float32
    s = {"case": case}
    if case["op"] == "gemm":
        m, k, n, g, trans = case["m"], case["k"], case["n"], case["g"], case.get("trans", False)
        pad = min(case.get("pad", 0), m - 1)                      # rows behind the last type: a buffer's unused end
        s["off"] = _offsets(rng, m - pad, g, 1.5)
        s["d_off"] = torch.from_numpy(s["off"].astype(np.int32)).to(DEV)
        s["X"] = normal(m, k, dtype=dtype)
        s["W"] = normal(g, *((n, k) if trans else (k, n)), scale=k ** -0.5, dtype=dtype)
        if case["way"] == "bwd":
            s["G"] = normal(m, n, scale=1e-2, dtype=dtype)
            s["mask"] = torch.relu(normal(m, k, dtype=dtype)) if case.get("mask") else None
        return s
    if case["op"] == "norm":
        m, c, q, b = case["m"], case["c"], case["q"], case["b"]
        s["seg"] = _offsets(rng, m, b, 1.0)
        s["d_seg"] = torch.from_numpy(s["seg"].astype(np.int32)).to(DEV)
        s["longest"] = int(np.diff(s["seg"]).max())
        # channels of different scale, their means up to a few deviations from zero
        s["X"] = normal(m, c).mul_(0.5 + torch.rand(c, generator=gen, device=DEV)).add_(normal(c)).to(dtype)
        s["gamma"], s["beta"] = 1.0 + normal(c, scale=0.2), normal(c, scale=0.2)
        if case["way"] == "bwd":
            s["G"] = normal(m, c, scale=1e-2, dtype=dtype)
            s["mean"], s["rstd"] = [t.float() for t in _stats64(s)]
        return s
    sizes = _tensor_sizes(case["tensors"], case["total"])
    kinds = [torch.float32, torch.bfloat16] if case["type"] == "mixed" else [dtype]
    step = 1 if case["packed"] else 256                           # packed: a tensor begins where the one before it ends
    s["grads"], s["out"], s["flat"], s["flat_out"] = [None] * len(sizes), [None] * len(sizes), [], []
    for i, kind in enumerate(kinds):
        at = [0]
        for z in sizes[i::len(kinds)]:
            at.append(at[-1] + -(-int(z) // step) * step)
        flat = normal(max(at[-1], 1), scale=1e-3, dtype=kind)
        out = torch.zeros_like(flat)
        for j, z in enumerate(sizes[i::len(kinds)]):
            s["grads"][i + j * len(kinds)], s["out"][i + j * len(kinds)] = flat[at[j]:at[j] + int(z)], out[at[j]:at[j] + int(z)]
        s["flat"].append(flat)
        s["flat_out"].append(out)
    # the bound as a share of what the norm will be near
    s["max_norm"] = float(case["ratio"] * 1e-3 * math.sqrt(case["total"]))
    return s


# ---------------------------------------------------------------------------------------------
# one pass

def run(s):
    return {"gemm": _run_gemm, "norm": _run_norm, "clip": _run_clip}[s["case"]["op"]](s)


def _prec(case):
    import paper_2504_04673_amd as sagnn
    return {"fp32": sagnn.GEMM_FP32, "fp32x3": sagnn.GEMM_FP32_BF16X3, "fp32_bf16": sagnn.GEMM_BF16, "bf16": sagnn.GEMM_FP32}[case["type"]]


def _operand(t, case):
    """What enters the product: the value itself, or rounded to bfloat16 where the case asks for that."""
    return t.bfloat16().float() if case["type"] == "fp32_bf16" else t.float()


def _run_gemm(s):
    case, X, W = s["case"], s["X"], s["W"]
    trans, relu = case.get("trans", False), case.get("act") == "relu"
    if own:
        import paper_2504_04673_amd as sagnn
        if case["way"] == "fwd":
            return sagnn.grouped_gemm_act(X, W, s["d_off"], transW=trans, prec=_prec(case), act=sagnn.ACT_RELU if relu else sagnn.ACT_IDENTITY)
        return sagnn.grouped_gemm_bwd(X, W, s["d_off"], s["G"], mask=s["mask"], prec=_prec(case))
    off = s["off"]
    parts = [(g, int(a), int(b)) for g, (a, b) in enumerate(zip(off[:-1], off[1:]))]
    rest = len(X) - int(off[-1])
    if case["way"] == "fwd":
        Y = [_operand(X[a:b], case) @ _operand(W[g].T if trans else W[g], case) for g, a, b in parts]
        Y = torch.cat(Y + [Y[0].new_zeros(rest, case["n"])])
        return (torch.relu(Y) if relu else Y).to(X.dtype)
    G = s["G"]
    dX = [_operand(G[a:b], case) @ _operand(W[g], case).T for g, a, b in parts]
    dX = torch.cat(dX + [dX[0].new_zeros(rest, case["k"])])
    dX = dX if s["mask"] is None else dX * (s["mask"] > 0)
    dW = torch.stack([_operand(X[a:b], case).T @ _operand(G[a:b], case) for g, a, b in parts])
    return dX.to(X.dtype), dW


def _padded(s):
    """Row numbers of every segment, one under the other, and which of them are there."""
    seg = torch.from_numpy(s["seg"]).to(DEV)
    at = seg[:-1, None] + torch.arange(max(s["longest"], 1), device=DEV)
    there = at < seg[1:, None]
    return torch.where(there, at, 0), there


def _run_norm(s):
    case, X = s["case"], s["X"]
    m, c, q, b = case["m"], case["c"], case["q"], case["b"]
    if own:
        import paper_2504_04673_amd as sagnn
        act = {"none": sagnn.ACT_IDENTITY, "relu": sagnn.ACT_RELU, "silu": sagnn.ACT_SILU}[case["act"]]
        if case["way"] == "fwd":
            return sagnn.group_norm_act(X, q, s["gamma"], s["beta"], seg=s["d_seg"], max_rows=s["longest"], eps=EPS, act=act)
        return sagnn.group_norm_act_bwd(X, s["G"], s["mean"], s["rstd"], q, s["gamma"], s["beta"], seg=s["d_seg"],
                                        max_rows=s["longest"], act=act)
    at, there = _padded(s)
    count = (there.sum(1, dtype=torch.float32) * (c // q)).clamp(min=1.0)[:, None]
    there = there[:, :, None]

    def sums(v):                                                  # b x longest x c -> b x q
        return v.sum(1).reshape(b, q, c // q).sum(2)

    def wide(v):                                                  # b x q -> b x 1 x c
        return v.repeat_interleave(c // q, 1)[:, None]

    x = X[at].float() * there
    mean = sums(x) / count if case["way"] == "fwd" else s["mean"]
    x = (x - wide(mean)) * there
    rstd = (sums(x * x) / count + EPS) ** -0.5 if case["way"] == "fwd" else s["rstd"]
    x = x * wide(rstd)
    z = x * s["gamma"] + s["beta"]
    there = there[:, :, 0]
    if case["way"] == "fwd":
        y = {"none": lambda: z, "relu": lambda: torch.relu(z), "silu": lambda: z / (1.0 + torch.exp(-z))}[case["act"]]()
        return y[there].to(X.dtype), mean, rstd
    h = s["G"][at].float() * there[:, :, None]
    if case["act"] == "relu":
        h = h * (z > 0)
    elif case["act"] == "silu":
        t = 1.0 / (1.0 + torch.exp(-z))
        h = h * (t * (1.0 + z * (1.0 - t)))
    del z
    dgamma, dbeta = (h * x).sum((0, 1)), h.sum((0, 1))
    h = h * s["gamma"]
    dx = (h - wide(sums(h) / count) - x * wide(sums(h * x) / count)) * wide(rstd)
    return dx[there].to(X.dtype), dgamma, dbeta


def _run_clip(s):
    if own:
        import paper_2504_04673_amd as sagnn
        norm = sagnn.grad_clip_norm(s["grads"], s["max_norm"], out=s["out"])
        return norm, s["flat_out"]
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    scale = (s["max_norm"] / norm).clamp(max=1.0)
    [o.copy_(g.float() * scale) for g, o in zip(s["grads"], s["out"])]
    return norm.reshape(1), s["flat_out"]


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    size = 2 if case["type"] == "bf16" else 4
    if case["op"] == "gemm":
        m, k, n, g = case["m"], case["k"], case["n"], case["g"]
        weights = min(g, m) * k * n                               # (a type without rows is not read)
        if case["way"] == "fwd":
            return {"bytes": (m * k + weights + m * n) * size, "flops": 2 * m * k * n}
        mask = m * k * size if case.get("mask") else 0
        return {"bytes": (2 * m * k + m * n + weights) * size + 4 * g * k * n + mask, "flops": 4 * m * k * n}
    if case["op"] == "norm":
        m, c, stats = case["m"], case["c"], 8 * case["b"] * case["q"]
        if case["way"] == "fwd":
            return {"bytes": 2 * m * c * size + stats + 8 * c, "flops": 8 * m * c}
        return {"bytes": 3 * m * c * size + stats + 16 * c, "flops": 16 * m * c}
    size = 3 if case["type"] == "mixed" else size                 # (half of the tensors each)
    return {"bytes": 2 * case["total"] * size, "flops": 3 * case["total"]}


# ---------------------------------------------------------------------------------------------
# the same outputs from their definition in 64 bits

def _stats64(s):
    """Mean and reciprocal deviation of every segment and group: sums over rows by the segment's number."""
    case = s["case"]
    seg = torch.from_numpy(s["seg"]).to(DEV)
    rows = seg.diff()
    number = torch.repeat_interleave(torch.arange(case["b"], device=DEV), rows)
    d = case["c"] // case["q"]
    values = s["X"].double().reshape(case["m"], case["q"], d)
    n = (rows * d).clamp(min=1).double()[:, None]
    zero = torch.zeros(case["b"], case["q"], dtype=torch.float64, device=DEV)
    mean = zero.index_add(0, number, values.sum(2)) / n
    var = zero.index_add(0, number, (values - mean[number][:, :, None]).square().sum(2)) / n
    return mean, (var + EPS).rsqrt()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "gemm":
        def value(t):
            return t.bfloat16().double() if case["type"] == "fp32_bf16" else t.double()

        off, n_rows = s["off"], len(s["X"])
        if case["way"] == "fwd":
            Y = torch.zeros(n_rows, case["n"], dtype=torch.float64, device=DEV)
            for g in range(case["g"]):
                rows = slice(int(off[g]), int(off[g + 1]))
                w = value(s["W"][g])
                Y[rows] = torch.mm(value(s["X"][rows]), w.t() if case.get("trans") else w)
            return Y.clamp_(min=0.0) if case.get("act") == "relu" else Y
        dX = torch.zeros(n_rows, case["k"], dtype=torch.float64, device=DEV)
        dW = torch.zeros(case["g"], case["k"], case["n"], dtype=torch.float64, device=DEV)
        for g in range(case["g"]):
            rows = slice(int(off[g]), int(off[g + 1]))
            G = value(s["G"][rows])
            dX[rows] = torch.mm(G, value(s["W"][g]).t())
            dW[g] = torch.mm(value(s["X"][rows]).t(), G)
        if s["mask"] is not None:
            dX[s["mask"] <= 0] = 0.0
        return dX, dW
    if case["op"] == "norm":
        m, c, q, b = case["m"], case["c"], case["q"], case["b"]
        rows = torch.from_numpy(s["seg"]).to(DEV).diff()
        number = torch.repeat_interleave(torch.arange(b, device=DEV), rows)
        mean, rstd = _stats64(s) if case["way"] == "fwd" else (s["mean"].double(), s["rstd"].double())
        x = s["X"].double().reshape(m, q, c // q).sub_(mean[number][:, :, None]).mul_(rstd[number][:, :, None])
        gamma = s["gamma"].double().reshape(q, c // q)
        z = x * gamma + s["beta"].double().reshape(q, c // q)
        sig = torch.sigmoid(z)
        if case["way"] == "fwd":
            y = {"none": lambda: z, "relu": lambda: z.clamp(min=0.0), "silu": lambda: z * sig}[case["act"]]()
            return y.reshape(m, c), mean, rstd
        slope = {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(), "silu": lambda: sig + z * sig * (1.0 - sig)}[case["act"]]()
        h = slope.mul_(s["G"].double().reshape(m, q, c // q))
        del z, sig
        dgamma, dbeta = (h * x).sum(0).reshape(c), h.sum(0).reshape(c)
        h.mul_(gamma)
        n = (rows * (c // q)).clamp(min=1).double()[:, None]
        zero = torch.zeros(b, q, dtype=torch.float64, device=DEV)
        s1 = zero.index_add(0, number, h.sum(2)) / n
        s2 = zero.index_add(0, number, (h * x).sum(2)) / n
        dx = (h - s1[number][:, :, None] - x * s2[number][:, :, None]) * rstd[number][:, :, None]
        return dx.reshape(m, c), dgamma, dbeta
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in s["grads"]))
    scale = min(1.0, s["max_norm"] / norm)
    flats = []
    for flat, out in zip(s["flat"], s["flat_out"]):
        e = torch.zeros(flat.shape, dtype=torch.float64, device=DEV)
        for g in s["grads"]:
            if g.dtype == flat.dtype and g.numel():
                at = (g.data_ptr() - flat.data_ptr()) // flat.element_size()
                e[at:at + g.numel()] = g.double() * scale
        flats.append(e)
    return torch.tensor([norm], dtype=torch.float64), flats
