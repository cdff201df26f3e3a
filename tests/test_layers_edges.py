"""Layer norm, dense layers and vocabulary losses where their numerics are
tightest, against the same formulas in 64 bits (tolerances: test_layers.py
says how they count).

The losses here are given their logits' own error bound e_l = (D + 8) u sum
|h w| / T per logit, and with d = (max z - z) / T the distance of a teacher's
entry from its row's largest: (z - max) / T is a subtraction and a product by a
rounded 1 / T, so q is off by (3 d + 24) u of itself (exp 2 u, its sum and the
division 20 u), and a q below 2^-126 may be 0.
"""
import math

import pytest
import torch

from test_layers import BF, F32, HALF, U, check_guard, close, close_norm, gen, guarded, norm_case, randn

pytestmark = pytest.mark.gpu


def teacher64(index, logits, T):
    """q, its error bound and which rows count."""
    there = index >= 0
    z = torch.where(there, logits.double(), float("-inf"))
    mx = z.amax(1, keepdim=True)
    live = torch.isfinite(mx)
    d = torch.where(there & live, mx - z, float("inf")) / T
    q = torch.nan_to_num(torch.exp(-d) / torch.exp(-d).sum(1, keepdim=True), nan=0.0)
    return q, torch.where(q > 0, q * (3 * d + 24) * U, 0.0) + 2.0 ** -126, live[:, 0]


def distill_on(ffmlp, H, W, index, logits, T, gt=F32, exact_p=None):
    """distill_step on these inputs: rows' losses, loss, dH and dW, element by
    element and in the norm.  exact_p: softmax(H W / T), where the logits' own
    rounding is too coarse to say."""
    (M, D), V, top = H.shape, W.shape[1], index.shape[1]
    head = ffmlp.SoftmaxHead(D, V)
    ws = head.workspace(M, top=top)
    ws.fill_(255)
    rl = torch.full((M,), float("nan"), device="cuda")
    bufh, dH = guarded(M, D, gt)
    bufw, dW = guarded(D, V, gt)
    _, _, loss = head.distill_step(W, H, index, logits, ws, temperature=T, row_loss=rl, dH=dH, dW=dW)
    check_guard(bufh, dH)
    check_guard(bufw, dW)
    h, w = H.double(), W.double()
    l = h @ w / T
    e_l = (D + 8) * U * (h.abs() @ w.abs()) / T + 4 * U * l.abs()
    e_lse = e_l.amax(1, keepdim=True) + 24 * U  # of a sum of V terms
    lse = torch.logsumexp(l, 1, keepdim=True)
    q, e_q, live = teacher64(index, logits, T)
    ix = index.clamp_min(0)
    lq, lp = torch.log(q.clamp_min(1e-300)), (l - lse).gather(1, ix)
    rows = T * T * (q * (lq - lp)).sum(1) * live
    e_row = T * T * (e_q * ((lq - lp).abs() + 1) + q * (e_l.gather(1, ix) + e_lse + 8 * U * (lq.abs() + lp.abs() + 1))).sum(1)
    close(rl, rows, e_row * live + 100 * U * rows.abs() + 1e-12, "row loss")
    n = max(1, int(live.sum()))
    close(loss, (rows.sum() / n).reshape(1), ((e_row * live).sum() / n + 180 * U * rows.abs().sum() / n).reshape(1) + 1e-12, "loss")
    p = torch.exp(l - lse) if exact_p is None else exact_p
    p = p * live[:, None]
    P = p.scatter_add(1, ix, -q * live[:, None])
    hit = torch.zeros_like(p).scatter_add(1, ix, (index >= 0).double()) > 0
    # p outside the lists passes through fp16 (2^-11, or 2^-40 of a block's
    # largest); where q is subtracted it has only the logits' error
    e_p = p * (e_l + e_lse + 32 * U) if exact_p is None else 32 * U * p
    e_P = e_p + torch.where(hit, 0.0, 2.0 ** -11 * p + 2.0 ** -40)
    e_P = (e_P.scatter_add(1, ix, e_q) + HALF[BF] * P.abs()) * live[:, None]
    # in the norm: roundings of P's elements are independent, and those of a
    # logit's sum too; the error of lse is one for the row
    e_i, e_c = 0.0 * p, 32 * U * p
    if exact_p is None:
        e_i = p * (math.sqrt(D + 8) * U * (h.abs() @ w.abs()) / T + 4 * U * l.abs())
        e_c = p * ((e_i / p.clamp_min(1e-300) * (p > 1e-12)).amax(1, keepdim=True) + 56 * U)
    e_i = e_i + torch.where(hit, 0.0, 2.0 ** -11 * p + 2.0 ** -40)
    e_i = (e_i.scatter_add(1, ix, e_q) + HALF[BF] * P.abs()) * live[:, None]
    a = T / n
    ref, s = a * (P @ w.t()), a * (P.abs() @ w.abs().t())
    close(dH, ref, a * (e_P @ w.abs().t()) + (V + 8) * U * s + HALF[gt] * (ref.abs() + HALF[BF] * s) + 1e-14, "dH")
    close_norm(dH, ref, a * ((e_i.square() @ w.square().t()).sum().sqrt() + (e_c @ w.t()).norm()).item()
               + math.sqrt(V + 8) * U * s.norm().item() + HALF[gt] * ref.norm().item() + 1e-14, "dH norm")
    ref, s = a * (h.t() @ P), a * (h.abs().t() @ P.abs())
    close(dW, ref, a * (h.abs().t() @ e_P) + (M + 8) * U * s + HALF[gt] * (ref.abs() + HALF[BF] * s) + 1e-14, "dW")
    close_norm(dW, ref, a * ((h.square().t() @ e_i.square()).sum().sqrt() + (h.square().t() @ e_c.square()).sum().sqrt()).item()
               + math.sqrt(M + 8) * U * s.norm().item() + HALF[gt] * ref.norm().item() + 1e-14, "dW norm")
    wi = head.workspace(M, mode=ffmlp.MLP_MODE_INFER, top=top)
    wi.fill_(255)
    rl2 = torch.empty_like(rl)
    assert torch.equal(head.distill(W, H, index, logits, wi, temperature=T, row_loss=rl2), loss) and torch.equal(rl, rl2)


# a vocabulary of the pass over whole rows, and one of two passes
WORDS = [900, 3000]


@pytest.mark.parametrize("V", WORDS)
@pytest.mark.parametrize("T", [1.0, 0.1])
def test_teacher_entries_at_the_end_of_the_fp32_range(ffmlp, gpu, V, T):
    """Lists that go down by 80 to 95 units of logit / T in small steps: some
    probabilities are fp32 denormals, others 0."""
    g = gen(31)
    M, D, top = 40, 48, 64
    H, W = randn(g, M, D), randn(g, D, V, std=2 * T / math.sqrt(D))
    index = torch.rand(M, V, generator=g, device="cuda").topk(top, 1).indices
    d = torch.linspace(80.0, 95.0, top - 4, device="cuda").expand(M, top - 4) + 0.2 * torch.rand(M, 1, generator=g, device="cuda")
    logits = torch.cat([torch.rand(M, 4, generator=g, device="cuda"), -d], 1) * T
    distill_on(ffmlp, H, W, index, logits.contiguous(), T)


@pytest.mark.parametrize("V", WORDS)
@pytest.mark.parametrize("zt", [BF, F32])
@pytest.mark.parametrize("T", [0.25, 0.5])
def test_teacher_logits_of_the_lowest_value(ffmlp, gpu, V, zt, T):
    """Lists masked with the type's lowest value, alone (all entries alike),
    beside ordinary logits, and beside the largest value."""
    g = gen(32)
    M, D, top = 33, 40, 6
    H, W = randn(g, M, D), randn(g, D, V, std=2 * T / math.sqrt(D))
    index = torch.rand(M, V, generator=g, device="cuda").topk(top, 1).indices
    logits = torch.randn(M, top, generator=g, device="cuda").to(zt)
    lowest = torch.finfo(zt).min
    logits[0] = lowest
    logits[1, :3] = lowest
    logits[2], logits[2, 4] = lowest, float("-inf")
    logits[3] = -lowest
    logits[4, 0], logits[4, 1] = lowest, -lowest
    logits[5] = float("-inf")  # does not count
    distill_on(ffmlp, H, W, index, logits, T)


@pytest.mark.parametrize("V", WORDS)
@pytest.mark.parametrize("at,T", [(1400.0, 1e-4), (22000.0, 1e-3), (1e5, 1e-4), (-1e5, 1e-4), (1e6, 1e-4)])
def test_distill_of_large_logits(ffmlp, gpu, V, at, T):
    """Logits / T beyond 2^24, of either sign.  Every row has one largest logit,
    or two alike, and the next below by far: the softmax is 1, or 1/2 and 1/2."""
    g = gen(33)
    M, D = 64, 16
    step = 2.0 ** math.floor(math.log2(abs(at)) - 6)  # exact in bf16
    H = torch.zeros(M, D, device="cuda")
    rows = torch.arange(M, device="cuda")
    H[rows, rows % (D - 2)] = 1
    W = torch.full((D, V), math.floor(at / step) * step, device="cuda")
    best, second = torch.randint(0, V // 2, (D,), generator=g, device="cuda"), torch.randint(V // 2, V, (D,), generator=g, device="cuda")
    f = torch.arange(D, device="cuda")
    W -= step * torch.randint(1, 4, (D, V), generator=g, device="cuda")
    W[f, best] = math.floor(at / step) * step
    W[f[::2], second[::2]] = math.floor(at / step) * step
    H, W = H.to(BF), W.to(BF)
    l = H.double() @ W.double()
    top = l.amax(1, keepdim=True)
    assert step / T > 100
    p = (l == top).double()
    p = p / p.sum(1, keepdim=True)
    index = torch.randint(0, V, (M, 1), generator=g, device="cuda")
    index[::3, 0] = best[rows[::3] % (D - 2)]
    distill_on(ffmlp, H, W, index, torch.zeros(M, 1, device="cuda"), T, exact_p=p)


@pytest.mark.parametrize("V", WORDS)
@pytest.mark.parametrize("gt", [F32, BF])
@pytest.mark.parametrize("apart", [0.01, 0.3])
def test_distill_of_a_student_near_its_teacher(ffmlp, gpu, V, gt, apart):
    """p is near q: what is left of p - q is rounded once, to bf16."""
    g = gen(34)
    M, D, top, T = 300, 64, 48, 2.0
    H, W = randn(g, M, D), randn(g, D, V, std=2 / math.sqrt(D))
    words = 101 + torch.arange(top, device="cuda") + 3 * (torch.arange(top, device="cuda") > 30)
    H[:, 0] = 1
    W[0] = -60.0
    W[0, words] = 0.0
    l = (H.double() @ W.double())[:, words]
    logits = (l + apart * T * torch.randn(M, top, generator=g, device="cuda")).float()
    perm = torch.rand(M, top, generator=g, device="cuda").argsort(1)
    distill_on(ffmlp, H, W, words[perm], logits.gather(1, perm), T, gt)
    # one word twice: its probabilities add up
    index = words[perm].clone()
    index[:, 5] = index[:, 9]
    distill_on(ffmlp, H, W, index, logits.gather(1, perm), T, gt)


def test_layer_norm_of_2_23_rows(ffmlp, gpu):
    """Rows of 512 threads each, as many as make a launch of 2^32 threads."""
    M, N = 1 << 23, 2049
    X = torch.empty(M, N, dtype=BF, device="cuda")
    g = gen(35)
    some = randn(g, 4099, N)  # rows m and m + 4099 are alike
    for r in range(0, M, 4099 * 64):
        n = min(4099 * 64, M - r)
        X[r:r + n] = some.repeat(64, 1)[:n]
    want = ffmlp.LayerNorm(N).forward(some)
    x = some.double()
    ref = (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    close(want, ref, (HALF[BF] + 200 * U) * ref.abs() + 200 * U, "Y")
    stats = torch.empty(M, 2, device="cuda")
    assert ffmlp.LayerNorm(N).forward(X, Y=X, stats=stats) is X
    for r in range(0, M, 4099 * 64):
        n = min(4099 * 64, M - r)
        assert torch.equal(X[r:r + n], want.repeat(64, 1)[:n])
    assert torch.equal(stats[:4099], stats[-(M % 4099) - 4099:][:4099]) and torch.isfinite(stats).all()


def test_default_dtype_of_the_program(ffmlp, gpu):
    """Outputs that the layers allocate are fp32 whatever torch's default is."""
    ln, de, he = ffmlp.LayerNorm(32), ffmlp.Dense(32, 24), ffmlp.SoftmaxHead(32, 50)
    g = gen(36)
    X, W, Wh = randn(g, 6, 32), randn(g, 32, 24), randn(g, 32, 50)
    stats = torch.empty(6, 2, dtype=F32, device="cuda")
    t = torch.zeros(6, dtype=torch.int64, device="cuda")
    old = torch.get_default_dtype()
    try:
        for d in (torch.float64, torch.bfloat16):
            torch.set_default_dtype(d)
            ln.forward(X, stats=stats)
            _, dg, db = ln.backward(X, None, stats, X, ln.workspace(6))
            _, _, b = de.backward(W, X, randn(g, 6, 24), de.workspace(6))
            loss = he.cross_entropy(Wh, X, t, he.workspace(6))
            assert dg.dtype == db.dtype == b.dtype == loss.dtype == F32
    finally:
        torch.set_default_dtype(old)


# ------------------------------------------------- more than one round of rows --

@pytest.mark.parametrize("M,N,xt,yt", [(7001, 1000, BF, BF), (2051, 2048, BF, BF), (1101, 3001, BF, F32), (1101, 3000, F32, BF), (601, 5003, F32, BF),
                                       (523, 8192, BF, BF), (300, 16384, BF, BF), (5001, 400, BF, BF), (70001, 24, BF, F32), (33001, 100, F32, F32), (9001, 250, BF, BF)])
def test_layer_norm_of_several_rows_per_workgroup(ffmlp, gpu, M, N, xt, yt):
    """Every way of holding a row, with rows left for a second turn of the
    backward pass's workgroups and a last turn that is not full."""
    norm_case(ffmlp, M, N, xt, yt, seed=M + N)


@pytest.mark.parametrize("M,N,t", [(40003, 24, BF), (20011, 128, F32), (5001, 400, BF), (7001, 1000, BF), (2051, 2048, BF), (1101, 3001, F32), (601, 5003, BF), (300, 16384, F32)])
def test_layer_norm_backward_in_place_over_several_rows(ffmlp, gpu, M, N, t):
    """dX may be dY: the rows asked for ahead are not yet written."""
    g = gen(41)
    ln = ffmlp.LayerNorm(N)
    X, dY, gamma = randn(g, M, N, dtype=t), randn(g, M, N, dtype=t), torch.randn(N, generator=g, device="cuda")
    stats, ws = torch.empty(M, 2, device="cuda"), ln.workspace(M)
    ln.forward(X, gamma, stats=stats)
    dX, dg, db = ln.backward(X, gamma, stats, dY, ws)
    d2 = dY.clone()
    _, dg2, db2 = ln.backward(X, gamma, stats, d2, ws, dX=d2)
    assert torch.equal(d2, dX) and torch.equal(dg2, dg) and torch.equal(db2, db)


@pytest.mark.parametrize("N", [40, 100, 1000, 2049, 20001])
def test_layer_norm_keeps_what_is_not_finite_to_its_row(ffmlp, gpu, N):
    """A row with an infinity or a NaN is NaN; its neighbours, which share its
    wave or workgroup, are as without it."""
    g = gen(42)
    ln = ffmlp.LayerNorm(N)
    X, dY = randn(g, 9, N, dtype=F32), randn(g, 9, N, dtype=F32)
    Xb = X.clone()
    Xb[2, N // 2], Xb[5, N - 1], Xb[7, 0] = float("inf"), float("nan"), float("-inf")
    bad = torch.zeros(9, dtype=torch.bool, device="cuda")
    bad[[2, 5, 7]] = True
    st, stb = torch.empty(9, 2, device="cuda"), torch.empty(9, 2, device="cuda")
    Y, Yb = ln.forward(X, stats=st), ln.forward(Xb, stats=stb)
    assert torch.equal(Y[~bad], Yb[~bad]) and Yb[bad].isnan().all() and stb[bad].isnan().any(1).all()
    dX, _, db = ln.backward(X, None, st, dY, ln.workspace(9))
    dXb, dgb, dbb = ln.backward(Xb, None, stb, dY, ln.workspace(9))
    assert torch.equal(dX[~bad], dXb[~bad]) and dXb[bad].isnan().all() and dgb.isnan().all() and torch.equal(db, dbb)


# ------------------------------------------------------------- several pieces --

def pieces_case(ffmlp, M, D, V, T, gt, seed, rows, words):
    """A step of several pieces, checked at some rows of dH and columns of dW.
    Lists of 4 within the first, a middle and the last words."""
    g = gen(seed)
    H, W = randn(g, M, D), randn(g, D, V, std=2 * T / math.sqrt(D))
    index = torch.randint(0, V, (M, 4), generator=g, device="cuda")
    index[:, 1] = (index[:, 0] + V // 2) % V
    index[::5, 2] = -1
    index[3::50] = -1
    logits = torch.randn(M, 4, generator=g, device="cuda")
    head = ffmlp.SoftmaxHead(D, V)
    ws = head.workspace(M, top=4)
    ws.fill_(255)
    rl = torch.empty(M, device="cuda")
    dH, dW, loss = head.distill_step(W, H, index, logits, ws, temperature=T, row_loss=rl, dtype=gt)
    q, e_q, live = teacher64(index, logits, T)
    n, w = int(live.sum()), W.double()
    a = T / n
    h = H[rows].double()
    l = h @ w / T
    e_l = (D + 8) * U * (h.abs() @ w.abs()) / T
    lse = torch.logsumexp(l, 1, keepdim=True)
    p = torch.exp(l - lse) * live[rows][:, None]
    ix = index[rows].clamp_min(0)
    P = p.scatter_add(1, ix, -q[rows])
    e_P = p * (e_l + e_l.amax(1, keepdim=True) + 56 * U + 2.0 ** -11) + 2.0 ** -40
    e_P = e_P.scatter_add(1, ix, e_q[rows]) + HALF[BF] * P.abs()
    ref, s = a * (P @ w.t()), a * (P.abs() @ w.abs().t())
    close(dH[rows], ref, a * (e_P @ w.abs().t()) + (V + 16) * U * s + HALF[gt] * (ref.abs() + HALF[BF] * s) + 1e-14, "dH")
    close_norm(dH[rows], ref, a * ((e_P.square() @ w.square().t()).sum().sqrt()).item() + math.sqrt(V + 16) * U * s.norm().item()
               + HALF[gt] * ref.norm().item() + 1e-14, "dH norm")
    # columns of dW: over all rows, some at a time
    ref, s, e1, e2 = (torch.zeros(D, len(words), dtype=torch.float64, device="cuda") for _ in range(4))
    wc = w[:, words]
    for r in range(0, M, 4096):
        h = H[r:r + 4096].double()
        lse = torch.cat([torch.logsumexp(h[k:k + 512] @ w / T, 1, keepdim=True) for k in range(0, len(h), 512)])
        e_l = (D + 8) * U * (h.abs() @ w.abs().amax(1))[:, None] / T
        p = torch.exp(h @ wc / T - lse) * live[r:r + 4096, None]
        hit = (index[r:r + 4096, :, None] == words).double()
        P = p - (q[r:r + 4096, :, None] * hit).sum(1)
        e_P = p * (2 * e_l + 56 * U + 2.0 ** -11) + 2.0 ** -40 + (e_q[r:r + 4096, :, None] * hit).sum(1) + HALF[BF] * P.abs()
        ref += a * (h.t() @ P)
        s += a * (h.abs().t() @ P.abs())
        e1 += a * (h.abs().t() @ e_P)
        e2 += a * a * (h.square().t() @ e_P.square())
    close(dW[:, words], ref, e1 + (M + 8) * U * s + HALF[gt] * (ref.abs() + HALF[BF] * s) + 1e-14, "dW")
    close_norm(dW[:, words], ref, e2.sum().sqrt().item() + math.sqrt(M + 8) * U * s.norm().item() + HALF[gt] * ref.norm().item() + 1e-14, "dW norm")
    assert torch.isfinite(dH).all() and torch.isfinite(dW).all() and torch.isfinite(loss).all() and (dH[~live] == 0).all()


@pytest.mark.parametrize("gt", [F32, BF])
def test_three_pieces(ffmlp, gpu, gt):
    """2^20 rows: pieces of 1024 words, the middle one added to and written."""
    M, V = 1 << 20, 2500
    pieces_case(ffmlp, M, 8, V, 1.5, gt, 43, torch.arange(0, M, 1709, device="cuda"),
                torch.tensor([0, 1, 500, 1023, 1024, 1025, 1500, 2047, 2048, 2300, 2499], device="cuda"))


def test_pieces_of_a_wide_hidden_size(ffmlp, gpu):
    """Two pieces and a rest behind them, at a hidden size of several steps."""
    M, D, V = 12345, 328, 90001
    assert M * V > 1 << 30
    words = torch.cat([torch.arange(0, V, 5003), torch.tensor([43263, 43264, 86527, 86528, V - 1])]).to("cuda")
    pieces_case(ffmlp, M, D, V, 2.0, F32, 44, torch.arange(0, M, 63, device="cuda"), words)


# ---------------------------------------------------------------- error norms --

@pytest.mark.parametrize("M,D,V", [(300, 256, 1000), (300, 300, 1000), (257, 130, 5003), (2050, 64, 4101), (1500, 512, 8192)])
@pytest.mark.parametrize("gt", [F32, BF])
def test_losses_in_the_norm(ffmlp, gpu, M, D, V, gt):
    """Errors of dH and dW in the norm, where independent roundings do not add
    up as their absolute values do."""
    g = gen(45)
    H, W = randn(g, M, D), randn(g, D, V, std=2 / math.sqrt(D))
    index = torch.rand(M, V, generator=g, device="cuda").topk(9, 1).indices
    index[::6, 4:] = -1
    distill_on(ffmlp, H, W, index, 2 * torch.randn(M, 9, generator=g, device="cuda"), 1.0, gt)
    distill_on(ffmlp, H, W, index[:, :1].contiguous(), torch.zeros(M, 1, device="cuda"), 1.0, gt)


def test_residual_must_be_a_tensor(ffmlp, gpu):
    de = ffmlp.Dense(32, 24)
    g = gen(46)
    with pytest.raises(ValueError, match="residual"):
        de.forward(randn(g, 32, 24), randn(g, 4, 32), residual=1.0)
