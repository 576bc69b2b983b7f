"""The operators between a deep graph network's layers and behind its last one, as cases that can be timed and checked.

  dropout           from a counter-based generator, with a residual: the mask is a function of seed, offset, row and column
  root-mean-square  norm of a residual sum with dropout: forward, and the gradients of both addends and of the scale
  8-bit rows        the same norm with rows of 8 bits and a scale each, and the gather that reads them
  cross entropy     of a linear layer's softmax over the classes, the logits not kept: loss, and the gradients of features,
                    weights and bias

`listed()` names twelve cases, `draw(rng)` gives more of the same ranges, `prepare` makes the inputs on the GPU from a
seed, `run` is one pass: the plain form in elementary torch operations, or with `own` the library's calls.  `exact`
has the outputs in 64 bits.  Widths and vertex counts are those of the benchmark's graphs (16 to 602 features, thousands
to two million vertices), class counts from two to the vertices of a graph whose links are predicted.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
EPS = 1e-6


def listed():
    return [
        # features of a few seed vertices: the call's latency is everything
        {"name": "drop_96_fp32", "op": "drop", "m": 96, "c": 64, "p": 0.5, "type": "fp32", "residual": False},
        # a hidden layer of a two-million-vertex graph, added to the layer before it
        {"name": "drop_2m_bf16", "op": "drop", "m": 2000000, "c": 256, "p": 0.1, "type": "bf16", "residual": True},
        # a sampled batch's few vertices between two layers
        {"name": "norm_96_fwd_bf16", "op": "norm", "way": "fwd", "m": 96, "c": 256, "p": 0.1, "type": "bf16", "residual": True},
        # a million vertices between two layers, training
        {"name": "norm_1m_fwd_bf16", "op": "norm", "way": "fwd", "m": 1000000, "c": 256, "p": 0.1, "type": "bf16", "residual": True},
        # raw features of odd width, training: the gradients of both addends
        {"name": "norm_170k_bwd_fp32", "op": "norm", "way": "bwd", "m": 170003, "c": 602, "p": 0.2, "type": "fp32", "residual": True},
        # two million rows that begin on no 16 bytes, plain norm
        {"name": "norm_2m_bwd_bf16", "op": "norm", "way": "bwd", "m": 2000000, "c": 100, "p": 0.0, "type": "bf16", "residual": False},
        # one rank's rows of a small graph in 8 bits, and those of them that another rank needs
        {"name": "rows_30k_8bit", "op": "rows", "m": 30011, "c": 100, "share": 0.6, "type": "fp32", "residual": False},
        # the same of a large one, between two layers
        {"name": "rows_2m_8bit", "op": "rows", "m": 2000000, "c": 256, "share": 0.4, "type": "bf16", "residual": True},
        # a few vertices' loss while evaluating
        {"name": "classes_96_fwd_bf16", "op": "xent", "way": "fwd", "m": 96, "k": 256, "n": 47, "type": "bf16", "labelled": 1.0},
        # a citation graph's vertices, two in five of them labelled, training in fp32 on the bf16 matrix cores
        {"name": "classes_170k_train_fp32x3", "op": "xent", "way": "train", "m": 170003, "k": 128, "n": 172, "type": "fp32x3",
         "labelled": 0.4},
        # links: which of 54321 vertices is the other end, their features as the weights
        {"name": "links_4k_train_fp32x3", "op": "xent", "way": "train", "m": 4099, "k": 200, "n": 54321, "type": "fp32x3",
         "labelled": 1.0, "trans": True},
        # the same over 131072 vertices with wide features: arithmetic only
        {"name": "links_8k_train_bf16", "op": "xent", "way": "train", "m": 8192, "k": 1024, "n": 131072, "type": "bf16",
         "labelled": 1.0, "trans": True},
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
    op = rng.choice(["drop", "norm", "norm", "rows", "xent", "xent", "xent"])
    if op == "xent":
        way, kind = rng.choice(["fwd", "train", "train"]), rng.choice(["fp32", "fp32x3", "bf16", "bf16"])
        k = _width(rng, 8, 2048)
        n = _log(rng, 2, 131072) if rng.random() < 0.6 else _log(rng, 2, 350)
        # fp32 instructions do a sixteenth of the bf16 ones' work in a time
        most = 8192 * 1024 * 131072 // (16 if kind == "fp32" else 4 if kind == "fp32x3" else 1)
        m = _log(rng, 1, max(2, min(1000000, most // (k * n), 8192 * 131072 // n)))
        return {"op": op, "way": way, "m": m, "k": k, "n": n, "type": kind, "labelled": rng.choice([1.0, 0.5]),
                "trans": rng.random() < 0.5, "bias": rng.random() < 0.5, "weights": rng.random() < 0.3}
    c = _width(rng, 8, 602) if rng.random() < 0.7 else _width(rng, 8, 8192)
    case = {"op": op, "m": _log(rng, 1, max(2, min(2000000, 2000000 * 256 // c))), "c": c, "p": rng.choice([0.0, 0.1, 0.5]),
            "type": rng.choice(["fp32", "bf16"]), "residual": rng.random() < 0.5}
    if op == "drop":
        return {**case, "p": rng.choice([0.1, 0.3, 0.5])}
    if op == "norm":
        return {**case, "way": rng.choice(["fwd", "bwd"])}
    return {**case, "m": min(case["m"], 1000000), "p": 0.0, "share": round(rng.uniform(0.05, 1.0), 3)}


# ---------------------------------------------------------------------------------------------
# inputs

def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return torch.randn(shape, generator=gen, device=DEV).mul_(scale).to(dtype)

    dtype = torch.bfloat16 if case["type"] == "bf16" else torch.float32
    m, s = case["m"], {"case": case, "seed": 1000003 * int(seed) + 17, "offset": int(seed) % 1000}
    if case["op"] == "xent":
        k, n = case["k"], case["n"]
        s["H"] = normal(m, k, dtype=dtype)
        # logits of a network that has learnt something: a deviation of 2
        s["W"] = normal(*((n, k) if case.get("trans") else (k, n)), scale=2.0 * k ** -0.5, dtype=dtype)
        s["bias"] = normal(n) if case.get("bias", True) else None
        labels = torch.randint(0, n, (m,), generator=gen, device=DEV, dtype=torch.int32)
        labelled = torch.rand(m, generator=gen, device=DEV) < case["labelled"]
        s["labels"] = torch.where(labelled, labels, -1)
        s["scale"] = 1.0 / max(1, int(case["labelled"] * m))
        s["weights"] = torch.rand(m, generator=gen, device=DEV) * s["scale"] if case.get("weights") else None
        return s
    c = case["c"]
    # rows of different size
    s["X"] = normal(m, c).mul_(0.5 + torch.rand((m, 1), generator=gen, device=DEV)).to(dtype)
    s["R"] = normal(m, c, dtype=dtype) if case["residual"] else None
    if case["op"] == "drop":
        return s
    s["gamma"] = 1.0 + normal(c, scale=0.2)
    if case["op"] == "rows":
        s["rows"] = torch.randperm(m, generator=gen, device=DEV)[:max(1, int(case["share"] * m))].sort().values.int()
    elif case["way"] == "bwd":
        s["G"], s["rstd"] = normal(m, c, scale=1e-2, dtype=dtype), (s["X"].double().square().mean(1) + EPS).rsqrt().float()
        s["grad_sum"] = normal(m, c, scale=1e-2, dtype=dtype) if case["residual"] else None
    return s


# ---------------------------------------------------------------------------------------------
# one pass

def run(s):
    return {"drop": _run_drop, "norm": _run_norm, "rows": _run_rows, "xent": _run_xent}[s["case"]["op"]](s)


_WORD = 0xFFFFFFFF


def _round(c, k0, k1):
    """One round of Philox-4x32 (Salmon, Moraes, Dror, Shaw, Parallel random numbers: as easy as 1, 2, 3, 2011)."""
    a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57                  # (64 bits wrap; the shift's sign is masked off)
    return ((b >> 32) & _WORD) ^ c[1] ^ k0, b & _WORD, ((a >> 32) & _WORD) ^ c[3] ^ k1, a & _WORD


def _kept(m, c, p, seed, offset):
    """Which values dropout keeps: 16 bits each of ten rounds over (column // 8, row, offset), against p in 65536ths.  And the
    scale of those."""
    cut = math.floor(p * 65536 + 0.5)
    eights = -(-c // 8)
    row = torch.arange(m, device=DEV)[:, None].expand(m, eights)
    col = torch.arange(eights, device=DEV)[None].expand(m, eights)
    w = (col, row, torch.full_like(row, offset & _WORD), torch.full_like(row, offset >> 32))
    keys = [((seed + i * 0x9E3779B9) & _WORD, ((seed >> 32) + i * 0xBB67AE85) & _WORD) for i in range(10)]
    w = _round(_round(_round(_round(_round(w, *keys[0]), *keys[1]), *keys[2]), *keys[3]), *keys[4])
    w = _round(_round(_round(_round(_round(w, *keys[5]), *keys[6]), *keys[7]), *keys[8]), *keys[9])
    halves = torch.stack([w[0] & 0xFFFF, w[0] >> 16, w[1] & 0xFFFF, w[1] >> 16, w[2] & 0xFFFF, w[2] >> 16, w[3] & 0xFFFF, w[3] >> 16], 2)
    return halves.reshape(m, eights * 8)[:, :c] >= cut, 65536.0 / (65536 - cut)


def _dropped(x, s):
    case = s["case"]
    if case.get("p", 0.0) == 0.0:
        return x
    kept, scale = _kept(case["m"], case["c"], case["p"], s["seed"], s["offset"])
    return torch.where(kept, x * scale, 0.0)


def _run_drop(s):
    case, X, R = s["case"], s["X"], s["R"]
    if own:
        import paper_2504_04673_amd as sagnn
        return sagnn.dropout_add(X, case["p"], s["seed"], s["offset"], residual=R)
    y = _dropped(X.float(), s)
    return (y if R is None else y + R.float()).to(X.dtype)


def _run_norm(s):
    case, X, R, gamma = s["case"], s["X"], s["R"], s["gamma"]
    if own:
        import paper_2504_04673_amd as sagnn
        if case["way"] == "fwd":
            return sagnn.rms_norm(X, gamma, residual=R, eps=EPS, p=case["p"], seed=s["seed"], offset=s["offset"])
        return sagnn.rms_norm_bwd(X, s["G"], s["rstd"], gamma, grad_sum=s["grad_sum"], p=case["p"], seed=s["seed"], offset=s["offset"])
    if case["way"] == "fwd":
        x = _dropped(X.float(), s)
        x = x if R is None else x + R.float()
        rstd = (x.square().mean(1) + EPS) ** -0.5
        return (x * rstd[:, None] * gamma).to(X.dtype), x.to(X.dtype), rstd
    x, rstd = X.float() * s["rstd"][:, None], s["rstd"][:, None]
    g = s["G"].float()
    dgamma = (g * x).sum(0)
    g = g * gamma
    g = (g - x * (g * x).mean(1, keepdim=True)) * rstd
    g = g if s["grad_sum"] is None else g + s["grad_sum"].float()
    return _dropped(g, s).to(X.dtype), g.to(X.dtype), dgamma


def _eighths(y):
    """The nearest values of e4m3 (four significant bits, steps of 2^-9 below 2^-6, at most 448), even ones where two are."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)
    return (torch.round(y / step) * step).clamp(-448.0, 448.0)


def _run_rows(s):
    X, R, gamma, rows = s["X"], s["R"], s["gamma"], s["rows"]
    if own:
        import paper_2504_04673_amd as sagnn
        Q, scale, S, rstd = sagnn.rms_norm_e4m3(X, gamma, residual=R, eps=EPS)
        return sagnn.spmm_pack_rows_e4m3(Q, scale, rows, dtype=torch.bfloat16), scale, S, rstd
    x = X.float() if R is None else X.float() + R.float()
    rstd = (x.square().mean(1) + EPS) ** -0.5
    y = x * rstd[:, None] * gamma
    scale = y.abs().amax(1) / 448.0
    q = _eighths(y / scale[:, None])
    return (q[rows] * scale[rows, None]).bfloat16(), scale, x.to(X.dtype), rstd


def _run_xent(s):
    case, H, W, bias, labels = s["case"], s["H"], s["W"], s["bias"], s["labels"]
    trans, train = case.get("trans", False), case["way"] == "train"
    if own:
        import paper_2504_04673_amd as sagnn
        prec = {"fp32": sagnn.GEMM_FP32, "fp32x3": sagnn.GEMM_FP32_BF16X3, "bf16": sagnn.GEMM_FP32}[case["type"]]
        loss, lse = sagnn.softmax_xent(H, W, labels, bias=bias, transW=trans, prec=prec)
        if not train:
            return loss, lse
        g = s["scale"] if s["weights"] is None else s["weights"]
        return loss, *sagnn.softmax_xent_bwd(H, W, labels, lse, g, bias=bias, transW=trans, prec=prec)
    h, w = H.float(), W.float()
    z = h @ (w.T if trans else w)
    if bias is not None:
        z = z + bias
    most = z.amax(1, keepdim=True)
    lse = (most + torch.log(torch.exp(z - most).sum(1, keepdim=True)))[:, 0]
    known = labels >= 0
    at = torch.where(known, labels, 0).long()[:, None]
    loss = torch.where(known, lse - z.gather(1, at)[:, 0], 0.0)
    if not train:
        return loss, lse
    g = known * (s["scale"] if s["weights"] is None else s["weights"])
    z = torch.exp(z - lse[:, None]) * g[:, None]
    z = z.scatter_add(1, at, -g[:, None])
    dH = z @ (w if trans else w.T)
    dW = z.T @ h if trans else h.T @ z
    return loss, dH.to(H.dtype), dW.to(W.dtype), None if bias is None else z.sum(0)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    size, m = 2 if case["type"] == "bf16" else 4, case["m"]
    if case["op"] == "xent":
        k, n = case["k"], case["n"]
        bias = 4 * n if case.get("bias", True) else 0
        once = (m * k + k * n) * size + 12 * m + bias
        if case["way"] == "fwd":
            return {"bytes": once, "flops": 2 * m * k * n}
        return {"bytes": 2 * once, "flops": 6 * m * k * n}
    c, two = case["c"], case["residual"]
    if case["op"] == "drop":
        return {"bytes": (3 if two else 2) * m * c * size, "flops": 2 * m * c}
    if case["op"] == "rows":
        # the rows in 8 bits are written, and those that are needed read
        some = max(1, int(case["share"] * m))
        return {"bytes": ((3 if two else 1) * size + 1) * m * c + 3 * some * c + 8 * (m + some), "flops": 6 * m * c}
    if case["way"] == "fwd":
        return {"bytes": (2 + (1 if two else 0) + (1 if two or case["p"] else 0)) * m * c * size + 4 * m + 4 * c, "flops": 6 * m * c}
    return {"bytes": (3 + (1 if two else 0) + (1 if case["p"] else 0)) * m * c * size + 4 * m + 8 * c, "flops": 12 * m * c}


# ---------------------------------------------------------------------------------------------
# the same outputs from their definition in 64 bits

def _product(a, b):
    """High and low word of a product of two words, by halves."""
    a0, a1, b0, b1 = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
    low, mid = a0 * b0, a1 * b0 + ((a0 * b0) >> 16)
    mid2 = a0 * b1 + (mid & 0xFFFF)
    return a1 * b1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (low & 0xFFFF)


def _drop64(x, case, s):
    if case.get("p", 0.0) == 0.0:
        return x
    m, c = x.shape
    n = (c + 7) // 8
    number = torch.arange(m * n, device=DEV)
    w = [number % n, number // n, torch.full_like(number, s["offset"]), torch.zeros_like(number)]
    k0, k1 = s["seed"] % 2 ** 32, s["seed"] // 2 ** 32
    for _ in range(10):
        h0, l0 = _product(w[0], 0xD2511F53)
        h2, l2 = _product(w[2], 0xCD9E8D57)
        w = [h2 ^ w[1] ^ k0, l2, h0 ^ w[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    cut = int(np.floor(case["p"] * 65536 + 0.5))
    out = x.clone()
    for i in range(8):
        half = (w[i // 2] >> (16 * (i % 2))) % 65536
        out[:, i::8] *= (half >= cut).reshape(m, n)[:, :out[:, i::8].shape[1]]
    return out.mul_(65536.0 / (65536 - cut))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "drop":
        y = _drop64(s["X"].double(), case, s)
        return y if s["R"] is None else y.add_(s["R"].double())
    if case["op"] == "xent":
        h, w = s["H"].double(), s["W"].double()
        w = w.t() if case.get("trans") else w
        z = torch.mm(h, w)
        if s["bias"] is not None:
            z += s["bias"].double()
        lse = torch.logsumexp(z, 1)
        known = s["labels"] >= 0
        row, label = known.nonzero()[:, 0], s["labels"][known].long()
        loss = torch.zeros(case["m"], dtype=torch.float64, device=DEV)
        loss[row] = lse[row] - z[row, label]
        if case["way"] == "fwd":
            return loss, lse
        z.sub_(lse[:, None]).exp_()
        z[row, label] -= 1.0
        z[~known] = 0.0
        z.mul_(s["scale"] if s["weights"] is None else s["weights"].double()[:, None])
        dW = torch.mm(h.t(), z)
        return loss, torch.mm(z, w.t()), dW.t() if case.get("trans") else dW, None if s["bias"] is None else z.sum(0)
    gamma = s["gamma"].double()
    if case.get("way") == "bwd":
        g, x, rstd = s["G"].double(), s["X"].double(), s["rstd"].double()[:, None]
        dgamma = torch.einsum("rc,rc,r->c", g, x, rstd[:, 0])
        inner = (g * gamma * x).sum(1, keepdim=True) * rstd.pow(3) / case["c"]
        ds = g.mul_(gamma).mul_(rstd) - x * inner
        if s["grad_sum"] is not None:
            ds += s["grad_sum"].double()
        return _drop64(ds, case, s), ds, dgamma
    x = _drop64(s["X"].double(), case, s)
    if s["R"] is not None:
        x = x + s["R"].double()
    rstd = 1.0 / torch.sqrt(torch.einsum("rc,rc->r", x, x) / case["c"] + EPS)
    y = x * gamma * rstd[:, None]
    if case["op"] == "norm":
        return y, x, rstd
    scale = y.abs().max(1).values / 448.0
    y = y[s["rows"]] / scale[s["rows"], None]
    # e4m3 by its own steps: the exponent of 64 bits, three more bits, and the smallest step below
    exponent = torch.frexp(y).exponent.clamp(min=-5)
    y = torch.ldexp(torch.round(torch.ldexp(y, 4 - exponent)), exponent - 4)
    return y * scale[s["rows"], None], scale, x, rstd
