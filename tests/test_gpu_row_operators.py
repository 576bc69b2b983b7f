"""Dropout, the root-mean-square norm and the rows of 8 bits against plain implementations in 64 bits.

Tolerances, element-wise (u = 2^-24; a bfloat16 result is rounded once more, by 2^-8):
  dropout   the mask exactly; a kept value meets three roundings, those of the scale 65536 / (65536 - cut) itself, of the product and of the
            sum, |sum| <= |x scale| + |r|: 3 u |x scale| + u |r|
  sum       the same; the norm of it: with d = that bound, the mean square errs by 2 sum |s| d relative to sum s^2, rstd by half of it and 2 u,
            y = s rstd gamma by three more roundings
  8 bits    half a step of e4m3 on top: 2^-4 |y|, or 2^-10 of the scale below the smallest normal value
  gradients a row's sum: 32 terms in a lane, 6 joins (and 16 of wavefronts): 54 u of the sum of absolute values; 1e-5 (168 u) covers it and the
            roundings of the other terms.  gamma's: 384 terms in turn, 128 u, and joins in 64 bits: 1e-5 again
"""
import numpy as np
import pytest
import torch

import paper_2504_04673_amd as sagnn
from paper_2504_04673_amd import binding
from tests.philox import kept

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SHAPES = [(1, 1), (3, 2), (5, 7), (1, 8), (33, 9), (70, 16), (1, 64), (301, 100), (1000, 128), (77, 257), (130, 512), (9, 513), (65, 602), (40, 1000), (17, 1024), (6, 1025),
          (12, 2048), (5, 2049), (1, 4096), (7, 4097), (3, 8191), (2, 16384), (4099, 24)]
TYPES = [torch.float32, torch.bfloat16]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def view(t, pad, first):
    """The same values in rows that lie `pad` elements further apart, the first `first` elements into its buffer."""
    m, c = t.shape
    buf = torch.full((m * (c + pad) + first,), float("nan"), device=t.device, dtype=t.dtype)
    v = buf[first:].as_strided((m, c), (c + pad, 1))
    v.copy_(t)
    return v


def close(got, ref, bound, what):
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)                                 # (NaN counts)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / bound)[bad].max()):.3g} times the bound"


def rounding(dtype, ref):
    return ref.abs() * (2.0 ** -8 if dtype is torch.bfloat16 else 0.0) + 1e-37


def mask(m, c, p, seed, offset, row0=0):
    return torch.from_numpy(kept(m, c, p, seed, offset, row0)).cuda()


def added(X, R, p, seed=11, offset=3, row0=0):
    """r + drop(x) in 64 bits, and how far 32 may be off."""
    x = X.double()
    if p:
        cut = int(p * 65536 + 0.5)
        x = torch.where(mask(*X.shape, p, seed, offset, row0), x * (65536.0 / (65536 - cut)) if cut < 65536 else x * 0, 0.0)
    r = torch.zeros_like(x) if R is None else R.double()
    return x + r, (3 * x.abs() + r.abs()) * (U * 1.001) if p or R is not None else torch.zeros_like(x)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("m,c", SHAPES)
def test_dropout(m, c, dtype):
    for i, (p, res) in enumerate([(0.1, True), (0.5, False), (0.0, True), (0.999, True)]):
        g = gen(m + c + i)
        X, R = normal(g, m, c, dtype=dtype), normal(g, m, c, dtype=dtype) if res else None
        seed, offset = (1 << 63) + 5 * i, (7 << 32) + i
        if i % 2:
            X, R = view(X, 3, 1), None if R is None else view(R, 5, 3)
        Y = sagnn.dropout_add(X, p, seed, offset, residual=R, out=view(torch.zeros_like(X), 1, 1) if i == 2 else None)
        ref, bound = added(X, R, p, seed, offset)
        close(Y, ref, bound + rounding(dtype, ref), f"p = {p}")
        if p and not res:
            assert torch.equal(Y == 0, ~mask(m, c, p, seed, offset) | (X == 0))


def test_dropout_at_its_ends():
    g = gen(1)
    X, R = normal(g, 50, 37), normal(g, 50, 37)
    X[3, 5], X[4, 6], X[5, 7] = float("nan"), float("inf"), -float("inf")
    assert torch.equal(sagnn.dropout_add(X, 1.0, 0, residual=R), R)                      # everything falls, NaN and infinity too
    Y = sagnn.dropout_add(X, 0.0, 0)
    assert torch.equal(Y.nan_to_num(), X.nan_to_num())
    Y, k = sagnn.dropout_add(X, 0.5, 9, 1), mask(50, 37, 0.5, 9, 1)
    assert torch.equal(torch.where(k, X * 2, 0.0).nan_to_num(), Y.nan_to_num()) and torch.equal(Y.isnan(), X.isnan() & k)
    assert sagnn.dropout_add(X[:0], 0.5, 9).shape == (0, 37)


def test_dropout_in_place_and_in_shares():
    X, R = normal(gen(2), 1000, 100, dtype=torch.bfloat16), normal(gen(3), 1000, 100, dtype=torch.bfloat16)
    whole = sagnn.dropout_add(X, 0.3, 5, 6, residual=R, row0=(1 << 32) - 1000)
    # ranks that have the rows between them, and a column's neighbours that others have
    parts = [sagnn.dropout_add(X[a:b], 0.3, 5, 6, residual=R[a:b], row0=(1 << 32) - 1000 + a) for a, b in ((0, 1), (1, 400), (400, 1000))]
    assert torch.equal(whole, torch.cat(parts))
    assert torch.equal(sagnn.dropout_add(X[:, :24], 0.3, 5, 6, residual=R[:, :24], row0=(1 << 32) - 1000), whole[:, :24])
    for out in (X.clone(), R.clone()):
        args = (out, R) if torch.equal(out, X) else (X, out)
        assert torch.equal(sagnn.dropout_add(args[0], 0.3, 5, 6, residual=args[1], row0=(1 << 32) - 1000, out=out), whole)
    # the gradient: the same call
    G = normal(gen(4), 1000, 100)
    dX = sagnn.dropout_add(G, 0.3, 5, 6)
    ref, bound = added(G, None, 0.3, 5, 6)
    close(dX, ref, bound + 1e-37, "gradient")


@pytest.mark.parametrize("dtype", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("m,c", SHAPES)
def test_rms_norm(m, c, dtype):
    for i, (p, res, scaled) in enumerate([(0.0, False, True), (0.0, True, True), (0.25, True, False), (0.5, False, True)]):
        g = gen(m + 3 * c + i)
        X = normal(g, m, c, dtype=dtype) * (1.0 + torch.arange(m, device="cuda")[:, None] % 5).to(dtype)
        R, gamma = normal(g, m, c, dtype=dtype) if res else None, 1.0 + normal(g, c, scale=0.3) if scaled else None
        if i % 2:
            X, R = view(X, 3, 1), None if R is None else view(R, 1, 5)
        eps = 1e-6 if i % 2 else 1e-2
        Y, S, rstd = sagnn.rms_norm(X, gamma, residual=R, eps=eps, p=p, seed=11, offset=3)
        s, d = added(X, R, p)
        gm = torch.ones(c, dtype=torch.float64, device="cuda") if gamma is None else gamma.double()
        square = s.square().sum(1)
        r = (square / c + eps).rsqrt()
        rel = (s.abs() * d).sum(1) / (square + eps * c) + 2 * U
        close(rstd, r, r * rel, "rstd")
        ybound = (d + s.abs() * (rel[:, None] + 3 * U)) * r[:, None] * gm.abs()
        y = s * r[:, None] * gm
        close(Y, y, ybound * 1.01 + rounding(dtype, y), "y")
        if res or p:
            close(S, s, d + rounding(dtype, s), "sum")
        else:
            assert S is X
        # 8 bits
        Q, scale, S8, rstd8 = sagnn.rms_norm_e4m3(X, gamma, residual=R, eps=eps, p=p, seed=11, offset=3)
        assert Q.dtype is torch.float8_e4m3fn and torch.equal(rstd8, rstd) and torch.equal(S8, S)
        top = y.abs().amax(1)
        close(scale, top / 448, ybound.amax(1) * 1.01 / 448 + top / 448 * U + 1e-37, "scale")
        assert torch.equal(Q.float().abs().amax(1), torch.where(top > 0, 448.0, 0.0).float())
        wide = sagnn.spmm_pack_rows_e4m3(Q, scale)
        assert torch.equal(wide, Q.float() * scale[:, None])
        close(wide, y, y.abs() * 2.0 ** -4 + scale.double()[:, None] * 2.0 ** -10 + 2 * ybound + 1e-37, "8 bits")


def test_rms_norm_of_odd_rows():
    X = torch.zeros(6, 40, device="cuda")
    X[1], X[2, 3], X[3, 4], X[4] = 1e30, float("nan"), float("inf"), 1e-25
    Y, _, rstd = sagnn.rms_norm(X)
    assert not Y[0].any() and not Y[5].any() and float(rstd[0]) == pytest.approx(1e3, rel=1e-6)
    assert torch.allclose(Y[1], torch.ones(40, device="cuda"), rtol=1e-6)                # (squares beyond 32 bits)
    assert Y[2].isnan().all() and float(rstd[3]) == 0 and Y[3, 4].isnan() and not Y[3, :4].any()
    assert torch.allclose(Y[4], torch.full((40,), 1e-22, device="cuda"), rtol=1e-6, atol=0)
    Q, scale, _, _ = sagnn.rms_norm_e4m3(X)
    wide = sagnn.spmm_pack_rows_e4m3(Q, scale)
    assert not wide[0].any() and float(scale[0]) == 0 and wide[2].isnan().all() and wide[3, 4].isnan()
    assert torch.allclose(wide[1], torch.ones(40, device="cuda"), rtol=1e-6) and torch.allclose(wide[4], Y[4], rtol=1e-5, atol=0)
    tiny = sagnn.rms_norm_e4m3(X[4:5], eps=1e-6, gamma=torch.full((40,), 1e-20, device="cuda"))
    assert float(tiny[1]) == 0 and not tiny[0].float().any()                             # (no scale below 2^-126)
    assert sagnn.rms_norm(X[:0])[0].shape == (0, 40) and sagnn.rms_norm_e4m3(X[:0])[1].shape == (0,)


def test_rms_norm_in_place():
    X, R, gamma = normal(gen(7), 300, 602), normal(gen(8), 300, 602), normal(gen(9), 602)
    Y, S, rstd = sagnn.rms_norm(X, gamma, residual=R, p=0.2, seed=1)
    x, r = X.clone(), R.clone()
    y2, s2, _ = sagnn.rms_norm(x, gamma, residual=r, p=0.2, seed=1, out=x, out_sum=r)
    assert y2 is x and s2 is r and torch.equal(x, Y) and torch.equal(r, S)
    wide = torch.zeros(300, 1300, device="cuda")
    y3, s3, _ = sagnn.rms_norm(X, gamma, residual=R, p=0.2, seed=1, out=wide[:, 3:605], out_sum=wide[:, 640:1242])
    assert torch.equal(y3, Y) and torch.equal(s3, S) and not wide[:, 605:640].any() and not wide[:, :3].any()
    with pytest.raises(sagnn.SagnnError):
        sagnn.rms_norm(X, gamma, residual=R, out=wide[:, :602], out_sum=wide[:, 300:902])
    with pytest.raises(ValueError, match="out_sum"):
        sagnn.rms_norm(X, out_sum=wide[:, :602])


@pytest.mark.parametrize("rows", [0, 1, 1000])
@pytest.mark.parametrize("c", [1, 4, 13, 16, 100, 602, 2051])
def test_pack_of_rows_in_8_bits(c, rows):
    g = gen(c)
    Q, scale = normal(g, 500, c, scale=40.0).to(torch.float8_e4m3fn), normal(g, 500)
    which = torch.randint(-3, 504, (rows,), generator=g, device="cuda", dtype=torch.int32)
    inside = (which >= 0) & (which < 500)
    at = which.clamp(0, 499).long()
    ref = torch.where(inside[:, None], Q.float()[at] * scale[at, None], 0.0)
    assert torch.equal(sagnn.spmm_pack_rows_e4m3(Q, scale, which), ref)
    assert torch.equal(sagnn.spmm_pack_rows_e4m3(Q, scale, which, dtype=torch.bfloat16), ref.bfloat16())
    wide = torch.full((rows, c + 5), 7.0, device="cuda")
    q = torch.zeros(500 * (c + 3) + 1, dtype=torch.uint8, device="cuda")[1:].view(torch.float8_e4m3fn).as_strided((500, c), (c + 3, 1))
    q.view(torch.uint8).copy_(Q.view(torch.uint8))
    assert torch.equal(sagnn.spmm_pack_rows_e4m3(q, scale, which, out=wide[:, 2:2 + c]), ref)
    assert torch.equal(wide[:, :2], torch.full((rows, 2), 7.0, device="cuda")) and torch.equal(wide[:, 2 + c:], torch.full((rows, 3), 7.0, device="cuda"))


def test_every_value_of_8_bits():
    codes = torch.arange(256, device="cuda", dtype=torch.uint8).reshape(4, 64).view(torch.float8_e4m3fn)
    wide = sagnn.spmm_pack_rows_e4m3(codes, torch.ones(4, device="cuda"))
    assert torch.equal(wide.nan_to_num(nan=-1.0), codes.float().nan_to_num(nan=-1.0))
    # and rounding to each: values between neighbours, ties too, in rows whose largest is 448 (gamma 448 / y's largest)
    finite = codes.float().flatten()
    finite = finite[finite.isfinite()].unique()
    mid = (finite[1:] + finite[:-1]) / 2
    x = torch.cat([finite, mid, mid * (1 + 2 ** -20), mid * (1 - 2 ** -20)])
    Q, scale, _, rstd = sagnn.rms_norm_e4m3(x[None], eps=0.0)
    sure = torch.ones_like(x, dtype=torch.bool)
    sure[finite.numel():finite.numel() + mid.numel()] = False     # (exact ties: the norm's own rounding decides)
    assert torch.equal(Q.float()[0][sure], x.to(torch.float8_e4m3fn).float()[sure])


def plain_bwd(S, G, D, rstd, gamma):
    """ds, sum of its terms' absolute values, dgamma, its terms'."""
    s, g, r = S.double(), G.double(), rstd.double()[:, None]
    xh = s * r
    gg = g * (1.0 if gamma is None else gamma.double())
    dot = (gg * xh).mean(1, keepdim=True)
    d = torch.zeros_like(s) if D is None else D.double()
    terms = r * (gg.abs() + xh.abs() * (gg * xh).abs().mean(1, keepdim=True)) + d.abs()
    return r * (gg - xh * dot) + d, terms, (g * xh).sum(0), (g * xh).abs().sum(0)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("m,c", SHAPES + [(70000, 3), (30000, 40), (800, 5000)])
def test_rms_norm_gradients(m, c, dtype):
    for i, (p, more, scaled) in enumerate([(0.0, False, True), (0.3, True, True), (0.0, True, False), (0.6, False, True)]):
        g = gen(m + 7 * c + i)
        S, G = normal(g, m, c, dtype=dtype), normal(g, m, c, dtype=dtype, scale=1e-2)
        D, gamma = normal(g, m, c, dtype=dtype, scale=1e-2) if more else None, 1.0 + normal(g, c, scale=0.3) if scaled else None
        if i % 2:
            S, G, D = view(S, 3, 1), view(G, 1, 1), None if D is None else view(D, 7, 3)
        rstd = (S.double().square().mean(1) + 1e-3).rsqrt().float()
        dX, dR, dgamma = sagnn.rms_norm_bwd(S, G, rstd, gamma, grad_sum=D, p=p, seed=11, offset=3)
        ref, terms, ref_gamma, gamma_terms = plain_bwd(S, G, D, rstd, gamma)
        close(dR, ref, 1e-5 * terms + rounding(dtype, ref), "dR")
        close(dgamma, ref_gamma, 1e-5 * gamma_terms + 1e-37, "dgamma")
        if p:
            scale = 65536.0 / (65536 - int(p * 65536 + 0.5))
            k = mask(m, c, p, 11, 3)
            close(dX, torch.where(k, ref * scale, 0.0), torch.where(k, (1e-5 * terms + rounding(dtype, ref)) * scale, 1e-37), "dX")
        else:
            assert dX is dR
        again = sagnn.rms_norm_bwd(S, G, rstd, gamma, grad_sum=D, p=p, seed=11, offset=3)
        assert all(torch.equal(a, b) for a, b in zip((dX, dR, dgamma), again))


def test_gradients_against_differences():
    g = gen(5)
    X, R, gamma, G = normal(g, 6, 20), normal(g, 6, 20), 1.0 + normal(g, 20, scale=0.3), normal(g, 6, 20)
    args = dict(p=0.4, seed=3, offset=8)

    def loss(x, r, c):
        s, _ = added(x, r, 0.4, 3, 8)
        return float((s * (s.square().mean(1, keepdim=True) + 1e-3).rsqrt() * c.double() * G.double()).sum())

    Y, S, rstd = sagnn.rms_norm(X, gamma, residual=R, eps=1e-3, **args)
    dX, dR, dgamma = sagnn.rms_norm_bwd(S, G, rstd, gamma, **args)
    for t, d, f in ((X, dX, lambda x: loss(x, R, gamma)), (R, dR, lambda r: loss(X, r, gamma)), (gamma, dgamma, lambda c: loss(X, R, c))):
        for at in range(0, t.numel(), 7):
            plus, minus = t.double().clone(), t.double().clone()
            plus.view(-1)[at] += 1e-5
            minus.view(-1)[at] -= 1e-5
            # (differences in 64 bits: 1e-10 of the third derivative; the gradient itself to 1e-5 of its terms, some units)
            assert abs((f(plus) - f(minus)) / 2e-5 - float(d.reshape(-1)[at])) < 1e-4


def test_gradients_of_no_rows_and_some():
    z = torch.zeros(0, 40, device="cuda")
    dX, dR, dgamma = sagnn.rms_norm_bwd(z, z, z[:, 0].contiguous())
    assert dX.shape == dR.shape == (0, 40) and not dgamma.any()
    S, G = normal(gen(1), 500, 72), normal(gen(2), 500, 72)
    rstd = S.square().mean(1).rsqrt()
    dX, dR, dgamma = sagnn.rms_norm_bwd(S, G, rstd, p=0.5)
    only = sagnn.rms_norm_bwd(S, G, rstd, p=0.5, want_dgamma=False)
    assert torch.equal(only[0], dX) and torch.equal(only[1], dR) and only[2] is None
    only = sagnn.rms_norm_bwd(S, G, rstd, p=0.5, want_dx=False)
    assert only[0] is None and torch.equal(only[1], dR) and torch.equal(only[2], dgamma)


def test_captured_steps_draw_anew():
    """A graph that counts its offset up, replayed between eager work: each replay is the eager call of that offset."""
    X, R, G, gamma = normal(gen(1), 700, 104), normal(gen(2), 700, 104), normal(gen(3), 700, 104), normal(gen(4), 104)
    offset = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step(off):
        Y, S, rstd = sagnn.rms_norm(X, gamma, residual=R, p=0.3, seed=5, offset=off)
        grads = sagnn.rms_norm_bwd(S, G, rstd, gamma, p=0.3, seed=5, offset=off)
        return (sagnn.dropout_add(Y, 0.3, 6, off), Y, S, *grads)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(offset)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step(offset)
            offset.add_(1)
    torch.cuda.current_stream().wait_stream(side)
    offset.fill_((3 << 32) + 5)
    seen = []
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        ref = step((3 << 32) + 5 + i)
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
        seen.append(got[0].clone())
    assert not torch.equal(seen[0], seen[1])


def test_calls_on_two_streams():
    X, gamma = normal(gen(1), 20000, 256, dtype=torch.bfloat16), normal(gen(2), 256)
    G = normal(gen(3), 20000, 256, dtype=torch.bfloat16)
    ref = sagnn.rms_norm(X, gamma)
    grads = sagnn.rms_norm_bwd(X, G, ref[2], gamma)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                Y, _, rstd = sagnn.rms_norm(X, gamma)
                got.append((Y, rstd, *sagnn.rms_norm_bwd(X, G, rstd, gamma)))
    torch.cuda.synchronize()
    for y, rstd, *d in got:
        assert torch.equal(y, ref[0]) and torch.equal(rstd, ref[2]) and all(torch.equal(a, b) for a, b in zip(d, grads))


def test_rows_behind_two_gigabytes():
    """Offsets beyond 32 bits: 140000 rows of 16384."""
    m, c = 140000, 16384
    X = torch.zeros(m, c, dtype=torch.bfloat16, device="cuda")
    X[-3:] = normal(gen(1), 3, c, dtype=torch.bfloat16)
    Y = sagnn.dropout_add(X, 0.5, 1, 2)
    ref, bound = added(X[-3:], None, 0.5, 1, 2, row0=m - 3)
    close(Y[-3:], ref, bound + rounding(torch.bfloat16, ref), "dropout")
    Q, scale, _, rstd = sagnn.rms_norm_e4m3(X)
    tail = sagnn.rms_norm_e4m3(X[-3:])
    assert torch.equal(Q[-3:].view(torch.uint8), tail[0].view(torch.uint8)) and torch.equal(scale[-3:], tail[1])
    rows = torch.tensor([m - 1, 0, m - 3], dtype=torch.int32, device="cuda")
    assert torch.equal(sagnn.spmm_pack_rows_e4m3(Q, scale, rows)[[0, 2]], sagnn.spmm_pack_rows_e4m3(*tail[:2])[[2, 0]])
    dX, _, dgamma = sagnn.rms_norm_bwd(X, Y, rstd, want_dgamma=True)
    few = sagnn.rms_norm_bwd(X[-3:], Y[-3:], rstd[-3:].contiguous())
    assert torch.equal(dX[-3:], few[0])
    close(dgamma, few[2].double(), 1e-5 * (Y[-3:].double() * X[-3:].double() * rstd[-3:, None].double()).abs().sum(0) + 1e-37, "dgamma")


def test_tensors_of_another_device_are_refused(monkeypatch):
    """The current device is asked for on the host: where it is another than the tensors', nothing is launched."""
    x, v, n = torch.zeros(4, 8, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1 + x.get_device())
    for f in (lambda: sagnn.dropout_add(x, 0.1, 0), lambda: sagnn.rms_norm(x), lambda: sagnn.rms_norm_e4m3(x), lambda: sagnn.rms_norm_bwd(x, x, v),
              lambda: sagnn.spmm_pack_rows_e4m3(x.to(torch.float8_e4m3fn), v), lambda: sagnn.softmax_xent(x, x, v.int(), transW=True),
              lambda: binding._drop_args(0.5, 0, n, 0)):
        with pytest.raises(ValueError, match="current device"):
            f()
