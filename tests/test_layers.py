"""Layer norm, dense layers and vocabulary losses on the GPU against the same
formulas in 64 bits.

Tolerances count roundings, with u = 2^-24 (fp32) and h(t) = half a step of
the output type (bf16 2^-8, fp32 2^-24, relative to the value):

  * a sum of K products in fp32 is off by at most (K + 8) u times the sum of
    their absolute values, and, its rounding errors being independent, in the
    Frobenius norm by at most sqrt(K + 8) u times that of these sums;
  * an operand rounded to bf16 before a product adds 2^-8 of the sum of
    absolute products at most, and in the norm 2^-8 of the result's own (the
    errors are independent of each other and of the signs);
  * the hardware's exp, sin and reciprocal, and the approximation of Phi, are
    good to 2e-6 (1 + |z|) at the arguments used here.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
BF, F32 = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, std=1.0, dtype=BF):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def strided(t, offset, extra):
    """A copy of matrix t that starts `offset` elements into its storage, with
    rows `extra` elements further apart; the gaps hold NaN."""
    m, n = t.shape
    buf = torch.full((m * (n + extra) + offset + 64,), float("nan"), dtype=t.dtype, device=t.device)
    v = buf[offset:offset + m * (n + extra)].view(m, n + extra)[:, :n]
    v.copy_(t)
    return v


def guarded(m, n, dtype, offset=3, extra=5):
    """An output matrix inside a larger buffer of a known value."""
    buf = torch.full((m * (n + extra) + offset + 64,), 77.0, dtype=dtype, device="cuda")
    v = buf[offset:offset + m * (n + extra)].view(m, n + extra)[:, :n]
    return buf, v


def check_guard(buf, v):
    """Nothing outside the view was written."""
    keep = v.clone()
    v.fill_(77.0)
    assert (buf == 77.0).all(), "wrote outside the output"
    v.copy_(keep)


def close(got, ref, bound, what):
    """|got - ref| <= bound element by element (bound of ref's shape)."""
    err = (got.double() - ref).abs()
    assert torch.isfinite(got).all(), what
    worst = (err / bound.clamp_min(1e-300)).max().item() if err.numel() else 0.0
    print(f"  {what}: worst {worst:.3f} of the bound")
    assert worst <= 1.0, (what, worst)


def close_norm(got, ref, tol, what):
    err = (got.double() - ref).norm().item()
    print(f"  {what}: {err:.3e} against {tol:.3e}")
    assert err <= tol, (what, err, tol)


# -------------------------------------------------------------- layer norm --

def norm_case(ffmlp, M, N, xt, yt, affine=True, offset=0, extra=0, seed=1, eps=1e-5, scale=1.0, shift=0.3):
    g = gen(seed)
    X = ((torch.randn(M, N, generator=g, device="cuda") + shift) * scale).to(xt)
    dY = randn(g, M, N, dtype=yt)
    gamma = 1 + 0.2 * torch.randn(N, generator=g, device="cuda") if affine else None
    beta = 0.3 * torch.randn(N, generator=g, device="cuda") if affine else None
    if offset or extra:
        X, dY = strided(X, offset, extra), strided(dY, offset, extra)
    ln = ffmlp.LayerNorm(N, eps=eps)
    stats = torch.empty(M, 2, device="cuda")
    buf, Y = guarded(M, N, yt)
    ln.forward(X, gamma, beta, Y=Y, stats=stats)
    check_guard(buf, Y)
    buf, dX = guarded(M, N, xt)
    ws = ln.workspace(M)
    ws.fill_(255)  # NaN as fp32
    _, dg, db = ln.backward(X, gamma, stats, dY, ws, dX=dX)
    check_guard(buf, dX)
    x, dy = X.double(), dY.double()
    ga = gamma.double() if affine else torch.ones(N, device="cuda", dtype=torch.float64)
    be = beta.double() if affine else torch.zeros(N, device="cuda", dtype=torch.float64)
    mean = x.mean(1, keepdim=True)
    r = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    xh = (x - mean) * r
    y = xh * ga + be
    # A sum over a row adds at most 64 numbers in a chain and ten more in a
    # tree: mean off by 80 u mean |x|, var and so r relatively by 80 u plus
    # what the mean's error adds (its square, below 80 u for these inputs).
    e_xh = r * (2 * U * (x.abs() + mean.abs()) + 80 * U * x.abs().mean(1, keepdim=True)) + 100 * U * xh.abs()
    close(Y, y, e_xh * ga.abs() + 4 * U * (y.abs() + be.abs()) + HALF[yt] * y.abs() + 1e-12, "Y")
    u = dy * ga
    c1, c2 = u.mean(1, keepdim=True), (u * xh).mean(1, keepdim=True)
    dx = r * (u - c1 - xh * c2)
    e_c1 = 80 * U * u.abs().mean(1, keepdim=True)
    e_c2 = 80 * U * (u * xh).abs().mean(1, keepdim=True) + (u.abs() * e_xh).mean(1, keepdim=True)
    e_dx = r * (4 * U * (u.abs() + c1.abs() + (xh * c2).abs()) + e_c1 + e_xh * c2.abs() + xh.abs() * e_c2)
    close(dX, dx, e_dx + 100 * U * dx.abs() + HALF[xt] * dx.abs() + 1e-12, "dX")
    rows = M + 80
    close(dg, (dy * xh).sum(0), rows * U * (dy * xh).abs().sum(0) + (dy.abs() * e_xh).sum(0) + 1e-12, "dgamma")
    close(db, dy.sum(0), rows * U * dy.abs().sum(0) + 1e-12, "dbeta")


@pytest.mark.parametrize("xt,yt", [(BF, BF), (F32, F32), (BF, F32), (F32, BF)])
@pytest.mark.parametrize("M,N", [(1, 1), (3, 7), (5, 64), (130, 100), (33, 129), (257, 512), (65, 1000), (70, 2048),
                                 (9, 4000), (20, 5003), (7, 16384), (5, 16385), (3, 40001)])
def test_layer_norm(ffmlp, gpu, M, N, xt, yt):
    norm_case(ffmlp, M, N, xt, yt, seed=M + N)


@pytest.mark.parametrize("M,N,offset,extra", [(50, 128, 1, 0), (50, 96, 8, 8), (41, 333, 5, 3), (6, 20000, 1, 1), (203, 100, 1, 1),
                                              (501, 13, 3, 2), (70, 250, 2, 0), (9, 2047, 1, 4)])
def test_layer_norm_strides(ffmlp, gpu, M, N, offset, extra):
    norm_case(ffmlp, M, N, BF, BF, offset=offset, extra=extra)
    norm_case(ffmlp, M, N, F32, F32, affine=False, offset=offset, extra=extra)


def test_layer_norm_many_rows(ffmlp, gpu):
    norm_case(ffmlp, 40003, 24, BF, BF)
    norm_case(ffmlp, 30001, 31, BF, F32)
    norm_case(ffmlp, 5000, 1024, F32, BF)


def test_layer_norm_constant_rows_and_large_offsets(ffmlp, gpu):
    """A constant row has variance 0: Y is beta, and everything stays finite.
    An offset of 1000 standard deviations costs no more than the mean's own
    rounding (the variance is taken about the mean)."""
    ln = ffmlp.LayerNorm(100)
    X = torch.full((3, 100), 5.0, device="cuda")
    beta = torch.randn(100, device="cuda")
    stats = torch.empty(3, 2, device="cuda")
    Y = ln.forward(X, None, beta, stats=stats)
    assert torch.equal(Y, beta.expand(3, 100))
    dX, dg, db = ln.backward(X, None, stats, torch.ones(3, 100, device="cuda"), ln.workspace(3))
    assert torch.isfinite(dX).all() and (dg == 0).all() and (db == 3).all()
    g = gen(5)
    X = torch.randn(8, 1000, generator=g, device="cuda") + 1000
    Y = ffmlp.LayerNorm(1000).forward(X)
    x = X.double()
    ref = (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    assert (Y.double() - ref).abs().max() < 82 * U * 1004


def test_layer_norm_in_place_and_empty(ffmlp, gpu):
    for N in (300, 20001):
        ln = ffmlp.LayerNorm(N)
        X = torch.randn(6, N, device="cuda")
        dY = torch.randn(6, N, device="cuda")
        stats = torch.empty(6, 2, device="cuda")
        Y = ln.forward(X, stats=stats)
        ws = ln.workspace(6)
        dX, dg, db = ln.backward(X, None, stats, dY, ws)
        d2 = dY.clone()
        _, dg2, db2 = ln.backward(X, None, stats, d2, ws, dX=d2)
        assert torch.equal(d2, dX) and torch.equal(dg, dg2) and torch.equal(db, db2)
        X2 = X.clone()
        ln.forward(X2, Y=X2)
        assert torch.equal(X2, Y)
    E = torch.empty(0, 300, device="cuda")
    ln = ffmlp.LayerNorm(300)
    assert ln.forward(E).shape == (0, 300)
    dX, dg, db = ln.backward(E, None, torch.empty(0, 2, device="cuda"), E, ln.workspace(0))
    assert (dg == 0).all() and (db == 0).all()


# ------------------------------------------------------------------- dense --

def act64(act, z):
    if act == "linear":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp_min(0), (z > 0).double()
    if act == "sigmoid":
        p = torch.sigmoid(z)
        return p, p * (1 - p)
    if act == "sine":
        return torch.sin(z), torch.cos(z)
    if act == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * (1 - p)
    phi = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
    return z * phi, phi + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


def dense_case(ffmlp, M, K, N, act="linear", yt=BF, gt=F32, dyt=BF, bias=True, residual=False, offset=0, extra=0,
               seed=1, backward=True):
    g = gen(seed)
    X, W = randn(g, M, K), randn(g, K, N, std=1 / math.sqrt(K))
    b = 0.3 * torch.randn(N, generator=g, device="cuda") if bias else None
    R = randn(g, M, N, dtype=yt) if residual else None
    dY = randn(g, M, N, dtype=dyt)
    if offset or extra:
        X, W, dY = strided(X, offset, extra), strided(W, offset, extra), strided(dY, offset, extra)
        R = strided(R, offset, extra) if residual else None
    layer = ffmlp.Dense(K, N, act)
    ws = layer.workspace(M)
    ws.fill_(255)
    buf, Y = guarded(M, N, yt, *((8, 8) if offset == 0 else (3, 5)))
    stash = layer.stash(M)
    layer.forward(W, X, b, residual=R, Y=Y, stash=stash, ws=ws)
    check_guard(buf, Y)
    x, w, dy = X.double(), W.double(), dY.double()
    z = x @ w + (b.double() if bias else 0)
    e_z = (K + 8) * U * (x.abs() @ w.abs() + (b.double().abs() if bias else 0))
    y, d = act64(act, z)
    e_act = 0 if act in ("linear", "relu") else 2e-6 * (1 + z.abs())
    ref = y + (R.double() if residual else 0)
    close(Y, ref, 1.13 * e_z + e_act + 2 * U * ref.abs() + HALF[yt] * ref.abs() + 1e-12, "Y")
    if not backward:
        return
    # a derivative within e_z of ReLU's corner may go either way
    e_d = 1.2 * e_z + e_act if act != "linear" else torch.zeros_like(z)
    if act == "relu":
        e_d = (z.abs() <= e_z).double()
    if stash is not None:
        close(stash, d, e_d + 2 * U * d.abs() + 1e-12, "stash")
        d = stash.double()  # what the backward pass is given
    buf, dX = guarded(M, K, gt)
    bufw, dW = guarded(K, N, gt)
    ws.fill_(255)
    _, _, db = layer.backward(W, X, dY, ws, stash=stash, dX=dX, dW=dW)
    check_guard(buf, dX)
    check_guard(bufw, dW)
    dz = dy * d
    close(db, dz.sum(0), (M + 80) * U * dz.abs().sum(0) + 1e-12, "db")
    dzb = 0.0 if act == "linear" and dyt == BF else HALF[BF]
    s = dz.abs() @ w.abs().t()
    ref = dz @ w.t()
    close(dX, ref, ((N + 8) * U + dzb) * s + HALF[gt] * (ref.abs() + dzb * s) + 1e-12, "dX")
    close_norm(dX, ref, (math.sqrt(N + 8) * U) * s.norm() + (dzb + HALF[gt]) * ref.norm() + 1e-12, "dX norm")
    s = x.abs().t() @ dz.abs()
    ref = x.t() @ dz
    close(dW, ref, ((M + 8) * U + dzb) * s + HALF[gt] * (ref.abs() + dzb * s) + 1e-12, "dW")
    close_norm(dW, ref, (math.sqrt(M + 8) * U) * s.norm() + (dzb + HALF[gt]) * ref.norm() + 1e-12, "dW norm")


SIZES = [(1, 1, 1), (1, 16, 8), (1, 777, 8200), (1, 100, 16401), (2, 3, 5), (7, 31, 33), (16, 64, 64), (17, 65, 130), (64, 128, 128), (65, 200, 136),
         (130, 96, 257), (16, 1000, 1003), (1, 2048, 512), (5, 4097, 129), (300, 520, 264), (129, 1032, 1000)]


@pytest.mark.parametrize("M,K,N", SIZES)
def test_dense_sizes(ffmlp, gpu, M, K, N):
    dense_case(ffmlp, M, K, N, seed=M + K + N)
    dense_case(ffmlp, M, K, N, "silu", yt=F32, gt=BF, dyt=F32, residual=True, seed=M + K + N)


@pytest.mark.parametrize("act", ["linear", "relu", "sigmoid", "sine", "gelu", "silu"])
@pytest.mark.parametrize("yt,gt,dyt", [(BF, F32, BF), (F32, BF, F32)])
def test_dense_activations(ffmlp, gpu, act, yt, gt, dyt):
    dense_case(ffmlp, 100, 136, 200, act, yt, gt, dyt, residual=True)
    dense_case(ffmlp, 9, 77, 61, act, yt, gt, dyt, bias=False)


@pytest.mark.parametrize("M,K,N,offset,extra", [(40, 64, 72, 8, 8), (40, 64, 72, 1, 0), (200, 257, 300, 3, 2),
                                                (12, 512, 1000, 1, 1), (12, 512, 1000, 8, 16), (500, 128, 512, 16, 8)])
def test_dense_strides(ffmlp, gpu, M, K, N, offset, extra):
    dense_case(ffmlp, M, K, N, "gelu", residual=True, offset=offset, extra=extra)
    dense_case(ffmlp, M, K, N, "linear", yt=F32, gt=BF, residual=True, offset=offset, extra=extra)


@pytest.mark.parametrize("M,K,N", [(2048, 1024, 2048), (2100, 512, 2304), (4096, 264, 1032), (1500, 2000, 2001),
                                   (8192, 256, 384)])
def test_dense_large_tiles(ffmlp, gpu, M, K, N):
    """Shapes that fill the chip: the large tile, edges inside it, and splits
    of a long batch in the weight gradient."""
    dense_case(ffmlp, M, K, N, "gelu", residual=True)


def test_dense_residual_in_place_empty_and_parts(ffmlp, gpu):
    g = gen(3)
    layer = ffmlp.Dense(200, 120)
    X, W, R = randn(g, 30, 200), randn(g, 200, 120), randn(g, 30, 120, dtype=F32)
    ws = layer.workspace(30)
    Y = layer.forward(W, X, residual=R, ws=ws)
    assert Y.dtype == F32
    R2 = R.clone()
    layer.forward(W, X, residual=R2, Y=R2, ws=ws)
    assert torch.equal(R2, Y)
    dX, dW, db = layer.backward(W, X, R, ws)
    none, dW2, _ = layer.backward(W, X, R, ws, input_gradient=False)
    assert none is None and torch.equal(dW, dW2)
    E = torch.empty(0, 200, dtype=BF, device="cuda")
    assert layer.forward(W, E).shape == (0, 120)
    dX, dW, db = layer.backward(W, E, torch.empty(0, 120, device="cuda"), layer.workspace(0))
    assert dX.shape == (0, 200) and (dW == 0).all() and (db == 0).all()


def test_dense_relu_masks_what_is_not_finite(ffmlp, gpu):
    """A delta behind a ReLU that is off is 0 even where dY is inf or NaN."""
    layer = ffmlp.Dense(32, 16, "relu")
    X = torch.ones(4, 32, dtype=BF, device="cuda")
    W = torch.ones(32, 16, dtype=BF, device="cuda")
    W[:, 3] = -1
    stash = layer.stash(4)
    ws = layer.workspace(4)
    layer.forward(W, X, stash=stash, ws=ws)
    dY = torch.ones(4, 16, device="cuda")
    dY[0, 3], dY[1, 3] = float("inf"), float("nan")
    dX, dW, db = layer.backward(W, X, dY, ws, stash=stash)
    assert torch.isfinite(dX).all() and torch.isfinite(dW).all() and db[3] == 0


def test_more_than_2_31_elements(ffmlp, gpu):
    """Offsets past 32 bits: the last rows of a 66000 x 33000 output, and of a
    norm of as many elements."""
    g = gen(17)
    M, K, N = 66000, 16, 33000
    X, W = randn(g, M, K), randn(g, K, N)
    layer = ffmlp.Dense(K, N, "relu")
    Y = layer.forward(W, X, ws=layer.workspace(M, mode=ffmlp.MLP_MODE_INFER))
    rows = torch.tensor([0, 1, M // 2, M - 2, M - 1], device="cuda")
    ref = (X[rows].double() @ W.double()).clamp_min(0)
    close(Y[rows], ref, (K + 8) * U * (X[rows].double().abs() @ W.double().abs()) + HALF[BF] * ref + 1e-12, "Y")
    Z = ffmlp.LayerNorm(N).forward(Y)
    y = Y[rows].double()
    ref = (y - y.mean(1, keepdim=True)) / (y.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    close(Z[rows], ref, (HALF[BF] + 200 * U) * ref.abs() + 200 * U, "Z")


# ---------------------------------------------------------- vocabulary losses --

def softmax64(H, W, T=1.0):
    h, w = H.double(), W.double()
    l = h @ w / T
    e_l = (h.shape[1] + 8) * U * (h.abs() @ w.abs()) / T + 4 * U * l.abs()
    return h, w, l, torch.logsumexp(l, 1, keepdim=True), e_l


def check_head(loss, rl, dH, dW, h, w, l, lse, e_l, q, index, live, T, gt, ents=None):
    """q [M, k] probabilities at index [M, k]; rows with live False do not count."""
    n = max(1, int(live.sum()))
    lp = l.gather(1, index) - lse
    e_lse = e_l.max(1, keepdim=True).values + 16 * U * (1 + lse.abs())
    ref = T * T * (torch.xlogy(q, q) - q * lp).sum(1) * live
    e_row = T * T * ((q * (e_l.gather(1, index) + e_lse + 16 * U * (lp.abs() + 1))).sum(1) + 64 * U) * live
    e_row = e_row + 8 * U * ref.abs()
    close(rl, ref, e_row + 1e-12, "row loss")
    total = ref.sum() / n
    close(loss, total.reshape(1), (e_row.sum() / n + 80 * U * ref.abs().sum() / n).reshape(1) + 1e-12, "loss")
    if dH is None:
        return
    p = torch.exp(l - lse) * live[:, None]
    P = p.scatter_add(1, index, -(q * live[:, None]))
    # P: the error of the exponent, q's own, then the rounding to bf16.  The
    # first piece of the vocabulary passes through fp16 as 2^15 p / p_max, p_max
    # the largest of a block of columns: half a step is 2^-11 of a normal value
    # and 2^-25 of the smallest ones, that is 2^-40 p_max <= 2^-40.
    e_P = p * (e_l + e_lse) + (32 * U + 2.0 ** -11) * p + 2.0 ** -40 * live[:, None]
    e_P = e_P.scatter_add(1, index, 64 * U * q) + HALF[BF] * P.abs()
    a = T / n
    ref, s = a * (P @ w.t()), a * (P.abs() @ w.abs().t())
    close(dH, ref, a * (e_P @ w.abs().t()) + (l.shape[1] + 8) * U * s + HALF[gt] * (ref.abs() + HALF[BF] * s) + 1e-14, "dH")
    ref, s = a * (h.t() @ P), a * (h.abs().t() @ P.abs())
    close(dW, ref, a * (h.abs().t() @ e_P) + (l.shape[0] + 8) * U * s + HALF[gt] * (ref.abs() + HALF[BF] * s) + 1e-14, "dW")


def ce_case(ffmlp, M, D, V, gt=F32, offset=0, extra=0, seed=1, skip=0.2, std=2.0):
    g = gen(seed)
    H, W = randn(g, M, D), randn(g, D, V, std=std / math.sqrt(D))
    if offset or extra:
        H, W = strided(H, offset, extra), strided(W, offset, extra)
    target = torch.randint(0, V, (M,), generator=g, device="cuda")
    target[torch.rand(M, generator=g, device="cuda") < skip] = -100
    if M > 2:
        target[0], target[1] = V - 1, 0
    head = ffmlp.SoftmaxHead(D, V)
    ws = head.workspace(M)
    ws.fill_(255)
    rl = torch.full((M,), float("nan"), device="cuda")
    bufh, dH = guarded(M, D, gt)
    bufw, dW = guarded(D, V, gt)
    _, _, loss = head.cross_entropy_step(W, H, target, ws, row_loss=rl, dH=dH, dW=dW)
    check_guard(bufh, dH)
    check_guard(bufw, dW)
    h, w, l, lse, e_l = softmax64(H, W)
    live = target != -100
    check_head(loss, rl, dH, dW, h, w, l, lse, e_l, live.double()[:, None], target.clamp_min(0)[:, None], live, 1.0, gt)
    wi = head.workspace(M, mode=ffmlp.MLP_MODE_INFER)
    wi.fill_(255)
    rl2 = torch.empty_like(rl)
    assert torch.equal(head.cross_entropy(W, H, target, wi, row_loss=rl2), loss) and torch.equal(rl, rl2)


HEADS = [(1, 1, 1), (1, 16, 2), (3, 5, 7), (33, 64, 100), (64, 128, 256), (65, 128, 257), (100, 72, 1000), (7, 136, 5003),
         (300, 256, 1024), (257, 33, 2049)]


@pytest.mark.parametrize("M,D,V", HEADS)
def test_cross_entropy(ffmlp, gpu, M, D, V):
    ce_case(ffmlp, M, D, V, F32, seed=M + V)
    ce_case(ffmlp, M, D, V, BF, seed=M + V + 1)


@pytest.mark.parametrize("M,D,V", [(40, 257, 1024), (65, 264, 7), (4097, 16, 40), (4096, 16, 40), (40, 256, 1025), (17, 255, 1023), (513, 100, 1000)])
def test_cross_entropy_few_words(ffmlp, gpu, M, D, V):
    """On either side of what the pass over whole rows takes."""
    ce_case(ffmlp, M, D, V, BF)
    distill_case(ffmlp, M, D, V, 5, 1.0, gt=BF, twice=True)


@pytest.mark.parametrize("M,D,V", [(2048, 128, 5000), (2050, 64, 4101), (1025, 200, 8192)])
def test_cross_entropy_large_tiles(ffmlp, gpu, M, D, V):
    ce_case(ffmlp, M, D, V)


def test_cross_entropy_in_pieces(ffmlp, gpu):
    """More logits than a piece holds (2^29): the second piece's are computed
    again, dH adds up over both."""
    assert 9000 * 66001 > 1 << 29
    ce_case(ffmlp, 9000, 16, 66001)


def test_distill_in_pieces(ffmlp, gpu):
    distill_case(ffmlp, 8200, 8, 65544, 3, 2.0, gt=BF)


@pytest.mark.parametrize("offset,extra", [(1, 0), (8, 8), (3, 5)])
def test_cross_entropy_strides(ffmlp, gpu, offset, extra):
    ce_case(ffmlp, 70, 96, 600, offset=offset, extra=extra)


def distill_case(ffmlp, M, D, V, top, T, zt=F32, gt=F32, seed=1, twice=False):
    g = gen(seed)
    H, W = randn(g, M, D), randn(g, D, V, std=2 / math.sqrt(D))
    index = torch.rand(M, V, generator=g, device="cuda").topk(min(top, V), 1).indices
    if top > V:
        index = torch.cat([index, index[:, :1].expand(M, top - V)], 1).contiguous()
    if twice and top > 1:
        index[:, top - 1] = index[:, 0]
    logits = (3 * torch.randn(M, top, generator=g, device="cuda")).to(zt)
    index[torch.rand(M, top, generator=g, device="cuda") < 0.2] = -1
    if M > 3:
        index[0], index[1] = -1, -5  # no entry
        logits[2, 0] = float("-inf")
        logits[3] = torch.finfo(zt).min / 4
    if top > 1:
        logits[torch.where(index < 0)] = float("nan")  # what is not there is not read
    head = ffmlp.SoftmaxHead(D, V)
    ws = head.workspace(M, top=top)
    ws.fill_(255)
    rl = torch.full((M,), float("nan"), device="cuda")
    bufh, dH = guarded(M, D, gt)
    bufw, dW = guarded(D, V, gt)
    _, _, loss = head.distill_step(W, H, index, logits, ws, temperature=T, row_loss=rl, dH=dH, dW=dW)
    check_guard(bufh, dH)
    check_guard(bufw, dW)
    h, w, l, lse, e_l = softmax64(H, W, T)
    z = torch.where(index >= 0, logits.double() / T, float("-inf"))
    live = torch.isfinite(z).any(1)
    q = torch.nan_to_num(torch.softmax(z, 1), nan=0.0)
    # the teacher's exponents are rounded at |z| / T
    check_head(loss, rl, dH, dW, h, w, l, lse, e_l, q, index.clamp_min(0), live, T, gt)
    wi = head.workspace(M, mode=ffmlp.MLP_MODE_INFER, top=top)
    rl2 = torch.empty_like(rl)
    assert torch.equal(head.distill(W, H, index, logits, wi, temperature=T, row_loss=rl2), loss) and torch.equal(rl, rl2)


@pytest.mark.parametrize("M,D,V,top,T", [(1, 1, 1, 1, 1.0), (5, 16, 3, 3, 2.0), (40, 64, 100, 8, 1.0), (66, 72, 1001, 33, 4.0),
                                         (130, 128, 4096, 64, 2.0), (9, 40, 700, 200, 0.5), (20, 32, 5, 9, 1.0)])
def test_distill(ffmlp, gpu, M, D, V, top, T):
    distill_case(ffmlp, M, D, V, top, T, seed=M + V)
    distill_case(ffmlp, M, D, V, top, T, zt=BF, gt=BF, seed=M + V + 1, twice=True)


def test_distill_large_tiles(ffmlp, gpu):
    distill_case(ffmlp, 1030, 64, 6000, 16, 2.0)


def test_distill_of_one_certain_entry_is_cross_entropy(ffmlp, gpu):
    """Lists of one entry have q = 1: the same loss and gradients, bit for bit."""
    g = gen(9)
    M, D, V = 77, 48, 900
    H, W = randn(g, M, D), randn(g, D, V, std=0.3)
    target = torch.randint(0, V, (M,), generator=g, device="cuda")
    target[5] = -100
    head = ffmlp.SoftmaxHead(D, V)
    a = head.cross_entropy_step(W, H, target, head.workspace(M))
    b = head.distill_step(W, H, target[:, None].contiguous(), torch.randn(M, 1, device="cuda"), head.workspace(M))
    for x, y in zip(a, b):
        assert torch.equal(x, y)


def test_losses_without_a_row_that_counts(ffmlp, gpu):
    head = ffmlp.SoftmaxHead(16, 40)
    H = torch.randn(6, 16, device="cuda").to(BF)
    W = torch.randn(16, 40, device="cuda").to(BF)
    t = torch.full((6,), 7, device="cuda")
    dH, dW, loss = head.cross_entropy_step(W, H, t, head.workspace(6), ignore_index=7)
    assert loss.item() == 0 and (dH == 0).all() and (dW == 0).all()
    i = torch.full((6, 3), -1, device="cuda")
    dH, dW, loss = head.distill_step(W, H, i, torch.zeros(6, 3, device="cuda"), head.workspace(6, top=3))
    assert loss.item() == 0 and (dH == 0).all() and (dW == 0).all()
    i = torch.zeros(6, 1, dtype=torch.int64, device="cuda")
    loss = head.distill(W, H, i, torch.full((6, 1), float("-inf"), device="cuda"), head.workspace(6))
    assert loss.item() == 0
    E = H[:0]
    dH, dW, loss = head.cross_entropy_step(W, E, t[:0], head.workspace(0))
    assert loss.item() == 0 and dH.shape == (0, 16) and (dW == 0).all()


@pytest.mark.parametrize("bad", [40, -1, 1 << 40])
def test_targets_outside_the_vocabulary_are_loud(ffmlp, gpu, bad):
    """No memory outside is touched: the loss and the gradients are NaN."""
    head = ffmlp.SoftmaxHead(16, 40)
    H = torch.randn(6, 16, device="cuda").to(BF)
    W = torch.randn(16, 40, device="cuda").to(BF)
    t = torch.zeros(6, dtype=torch.int64, device="cuda")
    t[2] = bad
    rl = torch.empty(6, device="cuda")
    dH, dW, loss = head.cross_entropy_step(W, H, t, head.workspace(6), row_loss=rl)
    assert loss.isnan().all() and rl.isnan().tolist() == [False, False, True, False, False, False]
    assert dH[2].isnan().all() and dW.isnan().all()
    if bad > 0:
        rl.fill_(0)
        loss = head.distill(W, H, t[:, None].contiguous(), torch.zeros(6, 1, device="cuda"), head.workspace(6), row_loss=rl)
        assert loss.isnan().all() and rl.isnan().tolist() == [False, False, True, False, False, False]


def test_cross_entropy_extreme_logits(ffmlp, gpu):
    """Logits of +-1e4: the running maximum keeps the sums in range."""
    D, V = 8, 700
    H = torch.zeros(3, D, dtype=BF, device="cuda")
    W = torch.zeros(D, V, dtype=BF, device="cuda")
    H[:, 0] = torch.tensor([1.0, -1.0, 0.0])
    W[0, 3], W[0, 600] = 9984.0, -9984.0
    t = torch.tensor([3, 3, 3], device="cuda")
    head = ffmlp.SoftmaxHead(D, V)
    rl = torch.empty(3, device="cuda")
    dH, dW, loss = head.cross_entropy_step(W, H, t, head.workspace(3), row_loss=rl)
    ref = torch.tensor([0.0, 2 * 9984.0, math.log(V)])
    assert torch.allclose(rl.cpu(), ref, rtol=1e-6, atol=1e-3) and torch.isfinite(dH).all() and torch.isfinite(dW).all()


def test_gradients_against_differences(ffmlp, gpu):
    """Central differences of the 64-bit loss along random directions against
    the gradients: of order 1e-2 of their size (bf16 rounding of the delta)."""
    g = gen(21)
    M, D, V = 24, 32, 300
    H, W = randn(g, M, D), randn(g, D, V, std=0.3)
    t = torch.randint(0, V, (M,), generator=g, device="cuda")
    head = ffmlp.SoftmaxHead(D, V)
    dH, dW, _ = head.cross_entropy_step(W, H, t, head.workspace(M))

    def f(h, w):
        return torch.nn.functional.cross_entropy(h @ w, t)

    for k in range(3):
        a, b = torch.randn(M, D, generator=g, device="cuda").double(), torch.randn(D, V, generator=g, device="cuda").double()
        e = 1e-5
        num = (f(H.double() + e * a, W.double() + e * b) - f(H.double() - e * a, W.double() - e * b)) / (2 * e)
        ana = (dH.double() * a).sum() + (dW.double() * b).sum()
        scale = (dH.double().norm() * a.norm() / math.sqrt(M * D) + dW.double().norm() * b.norm() / math.sqrt(D * V))
        assert abs(num - ana) <= 3 * 2.0 ** -8 * scale  # independent roundings, three standard deviations and more


# ------------------------------------------------- streams, graphs, repeats --

def chain(ffmlp, s, ws):
    """Norm, widening layer, narrowing layer onto the residual, then both
    losses, and everything backwards: the operators as one step uses them."""
    norm, up, down, head = s["norm"], s["up"], s["down"], s["head"]
    n = norm.forward(s["X"], s["gamma"], s["beta"], stats=s["stats"], dtype=BF)
    a = up.forward(s["W1"], n, s["b1"], stash=s["stash"], ws=ws["up"])
    y = down.forward(s["W2"], a, s["b2"], residual=s["X"], ws=ws["down"], dtype=F32)
    h = y.to(BF)
    dH, dWh, loss = head.cross_entropy_step(s["Wh"], h, s["target"], ws["head"])
    dHk, dWk, kd = head.distill_step(s["Wh"], h, s["index"], s["logits"], ws["head"], temperature=2.0)
    dy = dH + dHk
    da, dW2, db2 = down.backward(s["W2"], a, dy, ws["down"])
    dn, dW1, db1 = up.backward(s["W1"], n, da, ws["up"], stash=s["stash"])
    dx, dg, db = norm.backward(s["X"], s["gamma"], s["stats"], dn, ws["norm"], dtype=F32)
    return [n, a, y, loss, kd, dWh, dWk, dW2, db2, dW1, db1, dx + dy, dg, db]


def chain_state(ffmlp, M=96, D=128, F=320, V=1500, seed=4):
    g = gen(seed)
    s = {"norm": ffmlp.LayerNorm(D), "up": ffmlp.Dense(D, F, "gelu"), "down": ffmlp.Dense(F, D), "head": ffmlp.SoftmaxHead(D, V),
         "X": randn(g, M, D, dtype=F32), "gamma": 1 + 0.1 * torch.randn(D, generator=g, device="cuda"),
         "beta": 0.1 * torch.randn(D, generator=g, device="cuda"), "W1": randn(g, D, F, std=0.1), "W2": randn(g, F, D, std=0.1),
         "b1": 0.1 * torch.randn(F, generator=g, device="cuda"), "b2": 0.1 * torch.randn(D, generator=g, device="cuda"),
         "Wh": randn(g, D, V, std=0.2), "target": torch.randint(0, V, (M,), generator=g, device="cuda"),
         "index": torch.rand(M, V, generator=g, device="cuda").topk(12, 1).indices,
         "logits": torch.randn(M, 12, generator=g, device="cuda"), "stats": torch.empty(M, 2, device="cuda")}
    s["target"][::7] = -100
    s["stash"] = s["up"].stash(M)
    return s


def chain_ws(s):
    M = s["X"].shape[0]
    ws = {k: s[k].workspace(M) for k in ("norm", "up", "down")}
    ws["head"] = s["head"].workspace(M, top=12)
    return ws


def test_chain_matches_autograd(ffmlp, gpu):
    """The whole step against autograd in 64 bits, at the bf16 rounding of
    six chained tensors (half a step each, independent)."""
    s = chain_state(ffmlp)
    out = chain(ffmlp, s, chain_ws(s))
    p = {k: s[k].double().requires_grad_() for k in ("X", "gamma", "beta", "W1", "b1", "W2", "b2", "Wh")}
    F = torch.nn.functional
    n = F.layer_norm(p["X"], (p["X"].shape[1],), p["gamma"], p["beta"], 1e-5)
    y = F.gelu(n @ p["W1"] + p["b1"]) @ p["W2"] + p["b2"] + p["X"]
    l = y @ p["Wh"]
    ce = F.cross_entropy(l, s["target"])
    q = torch.softmax(s["logits"].double() / 2, 1)
    lp = torch.log_softmax(l / 2, 1).gather(1, s["index"])
    kd = 4 * (torch.xlogy(q, q) - q * lp).sum(1).mean()
    (ce + kd).backward()
    tol = math.sqrt(6) * 2.0 ** -8
    assert abs(out[3].item() - ce.item()) < tol * ce.item() and abs(out[4].item() - kd.item()) < tol * kd.item()
    got = {"Wh": out[5] + out[6], "W2": out[7], "b2": out[8], "W1": out[9], "b1": out[10], "X": out[11], "gamma": out[12],
           "beta": out[13]}
    for k, v in got.items():
        ref = p[k].grad
        rel = ((v.double() - ref).norm() / ref.norm()).item()
        print(f"  {k}: {rel:.2e}")
        assert rel < tol, k


def test_fused_net_between_norm_and_head(ffmlp, gpu):
    """A fused net with a layer norm in front and a vocabulary behind: dH is
    the net's dY, its dX the norm's dY."""
    import datagen
    M, W0 = 700, 64
    g = gen(8)
    net = ffmlp.FusedMLP(64, 2, W0, 48, "relu")
    packed = net.pack(datagen.xavier_weights(3, 64, 2, W0, 48, device=gpu))
    norm, head = ffmlp.LayerNorm(W0), ffmlp.SoftmaxHead(48, 1200)
    X, Wh = randn(g, M, W0), randn(g, 48, 1200, std=0.3)
    t = torch.randint(0, 1200, (M,), generator=g, device="cuda")
    stats, ws = torch.empty(M, 2, device="cuda"), net.workspace(M)
    n = norm.forward(X, stats=stats)
    Y = net.forward(packed, n, stash=ws)
    dH, dWh, loss = head.cross_entropy_step(Wh, Y, t, head.workspace(M))
    G, dn = net.backward_dx(packed, n, dH, ws)
    dX, _, _ = norm.backward(X, None, stats, dn, norm.workspace(M))
    # the head and the norm at their own inputs, in 64 bits
    y = Y.double().requires_grad_()
    ref = torch.nn.functional.cross_entropy(y @ Wh.double(), t)
    ref.backward()
    assert abs(loss.item() - ref.item()) < 1e-5 * ref.item()
    assert (dH.double() - y.grad).norm() < 2.0 ** -8 * y.grad.norm()
    x = X.double().requires_grad_()
    torch.nn.functional.layer_norm(x, (W0,)).backward(dn.double())
    assert (dX.double() - x.grad).norm() < 2.0 ** -8 * x.grad.norm()
    assert torch.isfinite(G).all() and G.norm() > 0


def test_repeats_are_bitwise_equal(ffmlp, gpu):
    s = chain_state(ffmlp, M=333, F=520, V=3001)
    a, b = chain(ffmlp, s, chain_ws(s)), chain(ffmlp, s, chain_ws(s))
    for x, y in zip(a, b):
        assert torch.equal(x, y)


def test_another_stream(ffmlp, gpu):
    s = chain_state(ffmlp)
    ref = chain(ffmlp, s, chain_ws(s))
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ws = chain_ws(s)
        other = chain(ffmlp, s, ws)
    st.synchronize()
    for x, y in zip(ref, other):
        assert torch.equal(x, y)


def test_graph_capture_replays(ffmlp, gpu):
    """Captured and replayed with new inputs and eager work in between."""
    s = chain_state(ffmlp)
    ws = chain_ws(s)
    chain(ffmlp, s, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = chain(ffmlp, s, ws)
    for k in range(3):
        fresh = chain_state(ffmlp, seed=40 + k)
        for name in ("X", "W1", "Wh", "target", "index", "logits"):
            s[name].copy_(fresh[name])
        eager = dict(s, stats=torch.empty_like(s["stats"]), stash=torch.empty_like(s["stash"]))
        torch.cuda.synchronize()
        graph.replay()
        ref = chain(ffmlp, eager, chain_ws(eager))
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(out, ref)):
            assert torch.equal(x, y), (k, i)


# -------------------------------------------------------------------- refusals --

def test_layer_refusals_on_device(ffmlp, gpu):
    d = "cuda"
    ln, de, he = ffmlp.LayerNorm(64), ffmlp.Dense(64, 32, "gelu"), ffmlp.SoftmaxHead(64, 100)
    X = torch.randn(8, 64, device=d).to(BF)
    W, Wh = torch.randn(64, 32, device=d).to(BF), torch.randn(64, 100, device=d).to(BF)
    st, sh = torch.empty(8, 2, device=d), de.stash(8)
    t = torch.zeros(8, dtype=torch.int64, device=d)
    wsd, wsh, wsn = de.workspace(8), he.workspace(8), ln.workspace(8)
    dY = torch.randn(8, 32, device=d)
    i3, l3 = torch.zeros(8, 3, dtype=torch.int64, device=d), torch.zeros(8, 3, device=d)
    bad = [
        lambda: ln.forward(X[:, :32]), lambda: ln.forward(X.half()), lambda: ln.forward(X.t().contiguous().t()),
        lambda: ln.forward(X[:1].expand(8, 64)), lambda: ln.forward(X, torch.ones(63, device=d)),
        lambda: ln.forward(X, torch.ones(64, device=d).double()), lambda: ln.forward(X, stats=st[:4]),
        lambda: ln.forward(X, dtype=torch.float16), lambda: ln.forward(X.cpu()), lambda: ln.forward(X[0]),
        lambda: ln.backward(X, None, st, X[:4], wsn), lambda: ln.backward(X, None, st, X, wsn[:100]),
        lambda: ln.backward(X, None, st, X, None),
        lambda: de.forward(W, X.float()), lambda: de.forward(W.t().contiguous(), X), lambda: de.forward(W.float(), X),
        lambda: de.forward(W, X, torch.zeros(32, device=d).to(BF)),
        lambda: de.forward(W, X, residual=torch.zeros(8, 32, device=d), dtype=BF),
        lambda: de.forward(W, X, stash=torch.empty(8, 32, device=d).half()),
        lambda: de.backward(W, X, dY, wsd), lambda: de.backward(W, X, dY[:, :31], wsd, stash=sh),
        lambda: de.backward(W, X, dY, wsd[:64], stash=sh), lambda: de.backward(W, X, dY.double(), wsd, stash=sh),
        lambda: he.cross_entropy(Wh, X, t.int(), wsh), lambda: he.cross_entropy(Wh, X, t[:4], wsh),
        lambda: he.cross_entropy(Wh, X, None, wsh), lambda: he.cross_entropy(Wh[:, :99], X, t, wsh),
        lambda: he.cross_entropy_step(Wh, X, t, he.workspace(8, mode=ffmlp.MLP_MODE_INFER)),
        lambda: he.cross_entropy_step(Wh, X, t, wsh, dtype=torch.float16),
        lambda: he.distill(Wh, X, i3, l3[:, :2], wsh), lambda: he.distill(Wh, X, i3.int(), l3, wsh),
        lambda: he.distill(Wh, X, i3, l3.half(), wsh), lambda: he.distill(Wh, X, i3, l3, he.workspace(8)[:10]),
    ]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"case {k} was accepted")
    with pytest.raises(ffmlp.FFMLPError):
        he.distill(Wh, X, i3, l3, he.workspace(8, top=3), temperature=0.0)
    with pytest.raises(ffmlp.FFMLPError):
        he.distill(Wh, X, i3, l3, he.workspace(8, top=3), temperature=float("nan"))
    for out_of_range in (1e-5, 1e5, float("inf"), -1.0):
        with pytest.raises(ffmlp.FFMLPError, match="temperature"):
            he.distill(Wh, X, i3, l3, he.workspace(8, top=3), temperature=out_of_range)
    torch.cuda.synchronize()
    assert torch.isfinite(he.cross_entropy(Wh, X, t, wsh)).all()
