"""The operators that surround a fused MLP in a language model, as measurable cases.

Four of them, named by a case's "op":

  norm     layer norm of the rows of a matrix: Y = (X - mean) / sqrt(var + eps) * gamma + beta
  dense    one layer of any width: Y = act(X W + bias) + R
  ce       softmax cross entropy of the logits H W over a large vocabulary
  distill  T^2 KL(teacher || softmax(H W / T)) where the teacher gives a few top logits of each row

"way" is "forward" (the outputs alone; for a loss, the loss alone) or "step"
(the outputs and every gradient).  Types are "bf16" or "fp32"; the matrix
products take bf16 operands.  Gradients of sums over bf16-rounded operands
are returned in bf16.
"""
import math

import torch

own = False

_T = {"bf16": torch.bfloat16, "fp32": torch.float32}
_EPS = 1e-5
_IGNORE = -100


def _norm(name, way, rows, dim, x, y):
    return {"name": name, "op": "norm", "way": way, "rows": rows, "dim": dim, "x": x, "y": y}


def _dense(name, way, rows, k, n, act, out="bf16", grad="bf16", residual=False):
    return {"name": name, "op": "dense", "way": way, "rows": rows, "k": k, "n": n, "act": act, "out": out,
            "grad": grad, "residual": residual}


def _ce(name, way, rows, dim, vocab):
    return {"name": name, "op": "ce", "way": way, "rows": rows, "dim": dim, "vocab": vocab}


def _distill(name, way, rows, dim, vocab, top, temperature):
    return {"name": name, "op": "distill", "way": way, "rows": rows, "dim": dim, "vocab": vocab, "top": top,
            "temperature": temperature}


def listed():
    return [
        # Eight sequences that each decode one token: the norm of eight rows.
        # Latency is all of it.
        _norm("norm_decode", "forward", 8, 1024, "bf16", "bf16"),
        # A training batch of 16384 tokens of a mid-sized model, forward and backward.
        _norm("norm_step_16k", "step", 16384, 2048, "bf16", "bf16"),
        # An fp32 residual stream of odd width, the next layer reading bf16.
        _norm("norm_step_odd", "step", 3001, 5003, "fp32", "bf16"),
        # One token through a wide layer: the weights are read once.
        _dense("dense_decode", "forward", 1, 4096, 4096, "gelu"),
        # Prefill of 8192 tokens through the widening layer of a block.
        _dense("dense_prefill", "forward", 8192, 2048, 8192, "gelu"),
        # Training the narrowing layer, onto an fp32 residual stream, with fp32
        # weight gradients for the optimizer.
        _dense("dense_step_linear", "step", 8192, 4096, 1024, "linear", "fp32", "fp32", True),
        # A ragged training batch through a layer whose widths suit no tile.
        _dense("dense_step_odd", "step", 1111, 771, 1283, "silu"),
        # A fused net of width 128 as a classifier of a thousand classes.
        _ce("ce_step_classes", "step", 4096, 128, 1000),
        # Training the output layer of a mid-sized model on 8192 tokens.
        _ce("ce_step_vocab", "step", 8192, 2048, 65536),
        # Perplexity of a held-out text: the loss of every token, odd sizes.
        _ce("ce_eval_odd", "forward", 2047, 1000, 50021),
        # A small student trained on 32 stored logits of its teacher per token.
        _distill("distill_step", "step", 4096, 1024, 32768, 32, 2.0),
        # A short ragged batch with few stored logits.
        _distill("distill_step_odd", "step", 513, 200, 10007, 7, 1.0),
    ]


def _size(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.4 and v > 64:
        v = v // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["norm", "dense", "ce", "distill"])
    way = rng.choice(["forward", "step", "step"])
    if op == "norm":
        dim = _size(rng, 16, 16384)
        rows = _size(rng, 1, min(1 << 18, (1 << 25) // dim))
        c = _norm("", way, rows, dim, rng.choice(["bf16", "fp32"]), rng.choice(["bf16", "fp32"]))
    elif op == "dense":
        k, n = _size(rng, 16, 8192), _size(rng, 16, 8192)
        rows = _size(rng, 1, min(16384, (1 << 35) // (k * n)))
        act = rng.choice(["linear", "relu", "sigmoid", "sine", "gelu", "silu"])
        c = _dense("", way, rows, k, n, act, rng.choice(["bf16", "fp32"]),
                   rng.choice(["bf16", "fp32"]) if act == "linear" else "bf16", rng.random() < 0.5)
    else:
        dim, vocab = _size(rng, 16, 2048), _size(rng, 256, 65536)
        rows = _size(rng, 1, 8192)
        if op == "ce":
            c = _ce("", way, rows, dim, vocab)
        else:
            c = _distill("", way, rows, dim, vocab, rng.randint(1, 64), rng.choice([1.0, 2.0, 4.0]))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs --

def _data(case, seed):
    """The inputs of a case, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    op, rows, d = case["op"], case["rows"], {}
    if op == "norm":
        dim = case["dim"]
        # rows of different offset and scale, as in a residual stream
        scale = torch.rand(rows, 1, generator=g, device="cuda") * 3 + 0.2
        d["X"] = ((torch.randn(rows, dim, generator=g, device="cuda") + 0.3) * scale).to(_T[case["x"]])
        d["gamma"] = 1 + 0.2 * torch.randn(dim, generator=g, device="cuda")
        d["beta"] = 0.1 * torch.randn(dim, generator=g, device="cuda")
        if case["way"] == "step":
            d["dY"] = normal(rows, dim, dtype=_T[case["y"]])
    elif op == "dense":
        k, n = case["k"], case["n"]
        d["X"] = normal(rows, k)
        d["W"] = normal(k, n, std=1.0 / math.sqrt(k))
        d["bias"] = 0.1 * torch.randn(n, generator=g, device="cuda")
        if case["residual"]:
            d["R"] = normal(rows, n, dtype=_T[case["out"]])
        if case["way"] == "step":
            d["dY"] = normal(rows, n)
    else:
        dim, vocab = case["dim"], case["vocab"]
        d["H"] = normal(rows, dim)
        d["W"] = normal(dim, vocab, std=2.0 / math.sqrt(dim))
        if op == "ce":
            # frequent words first, as a tokenizer orders them; some tokens of
            # the batch (padding, a prompt) do not count
            u = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64)
            t = (torch.exp(u * math.log(vocab)) - 1).long().clamp_(0, vocab - 1)
            skip = torch.rand(rows, generator=g, device="cuda") < 0.07
            t[skip] = _IGNORE
            t[0] = vocab - 1
            d["target"] = t
        else:
            top = case["top"]
            start = torch.randint(0, vocab, (rows, 1), generator=g, device="cuda")
            step = torch.randint(1, max(2, vocab // top), (rows, 1), generator=g, device="cuda")
            index = (start + step * torch.arange(top, device="cuda")) % vocab
            logits = torch.randn(rows, top, generator=g, device="cuda") * 2 + 8
            # lists of different lengths; some rows have none
            length = torch.randint(1, top + 1, (rows, 1), generator=g, device="cuda")
            length[torch.rand(rows, 1, generator=g, device="cuda") < 0.05] = 0
            length[0] = top
            index[torch.arange(top, device="cuda") >= length] = -1
            d["index"], d["logits"] = index, logits
    return d


def prepare(case, seed):
    s = {"case": dict(case)}
    s.update(_data(case, seed))
    if own:
        import paper_2403_17607_amd as ffmlp
        op, rows, step = case["op"], case["rows"], case["way"] == "step"
        if op == "norm":
            s["layer"] = ffmlp.LayerNorm(case["dim"], eps=_EPS)
        elif op == "dense":
            s["layer"] = ffmlp.Dense(case["k"], case["n"], case["act"])
        else:
            s["layer"] = ffmlp.SoftmaxHead(case["dim"], case["vocab"])
        if op in ("norm", "dense"):
            mode = ffmlp.MLP_MODE_TRAIN if step else ffmlp.MLP_MODE_INFER
            s["ws"] = s["layer"].workspace(rows, mode=mode)
        else:
            mode = ffmlp.MLP_MODE_TRAIN if step else ffmlp.MLP_MODE_INFER
            s["ws"] = s["layer"].workspace(rows, top=case.get("top", 1), mode=mode)
        if op == "norm" and step:
            s["stats"] = torch.empty(rows, 2, device="cuda")
        if op == "dense" and step:
            s["stash"] = s["layer"].stash(rows)
    return s


# --------------------------------------------------------------------- run --

def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    c, layer, ws = s["case"], s["layer"], s["ws"]
    op, step = c["op"], c["way"] == "step"
    if op == "norm":
        Y = layer.forward(s["X"], s["gamma"], s["beta"], stats=s.get("stats"), dtype=_T[c["y"]])
        if not step:
            return {"Y": Y}
        dX, dg, db = layer.backward(s["X"], s["gamma"], s["stats"], s["dY"], ws, dtype=_T[c["x"]])
        return {"Y": Y, "dX": dX, "dgamma": dg, "dbeta": db}
    if op == "dense":
        Y = layer.forward(s["W"], s["X"], s["bias"], residual=s.get("R"), stash=s.get("stash"), ws=ws,
                          dtype=_T[c["out"]])
        if not step:
            return {"Y": Y}
        dX, dW, db = layer.backward(s["W"], s["X"], s["dY"], ws, stash=s["stash"], dtype=_T[c["grad"]])
        return {"Y": Y, "dX": dX, "dW": dW, "dbias": db}
    if op == "ce":
        if not step:
            rl = torch.empty(c["rows"], device="cuda")
            loss = layer.cross_entropy(s["W"], s["H"], s["target"], ws, ignore_index=_IGNORE, row_loss=rl)
            return {"loss": loss, "row_loss": rl}
        dH, dW, loss = layer.cross_entropy_step(s["W"], s["H"], s["target"], ws, ignore_index=_IGNORE,
                                                dtype=torch.bfloat16)
        return {"loss": loss, "dH": dH, "dW": dW}
    if not step:
        rl = torch.empty(c["rows"], device="cuda")
        loss = layer.distill(s["W"], s["H"], s["index"], s["logits"], ws, temperature=c["temperature"], row_loss=rl)
        return {"loss": loss, "row_loss": rl}
    dH, dW, loss = layer.distill_step(s["W"], s["H"], s["index"], s["logits"], ws, temperature=c["temperature"],
                                      dtype=torch.bfloat16)
    return {"loss": loss, "dH": dH, "dW": dW}


def _act(act, z):
    """act(z) and its derivative."""
    if act == "linear":
        return z, torch.ones_like(z)
    if act == "relu":
        on = (z > 0).to(z.dtype)
        return z * on, on
    if act == "sine":
        return torch.sin(z), torch.cos(z)
    if act == "gelu":  # z Phi(z)
        phi = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    p = 1 / (1 + torch.exp(-z))
    if act == "sigmoid":
        return p, p * (1 - p)
    return z * p, p + z * p * (1 - p)  # silu


def _plain(s):
    c = s["case"]
    op, step = c["op"], c["way"] == "step"
    if op == "norm":
        x = s["X"].float()
        xc = x - x.mean(1, keepdim=True)
        r = 1 / torch.sqrt((xc * xc).mean(1, keepdim=True) + _EPS)
        xh = xc * r
        out = {"Y": (xh * s["gamma"] + s["beta"]).to(_T[c["y"]])}
        if step:
            dy = s["dY"].float()
            out["dgamma"] = (dy * xh).sum(0)
            out["dbeta"] = dy.sum(0)
            q = dy * s["gamma"]
            dx = r * (q - q.mean(1, keepdim=True) - xh * (q * xh).mean(1, keepdim=True))
            out["dX"] = dx.to(_T[c["x"]])
        return out
    if op == "dense":
        x, w = s["X"].float(), s["W"].float()
        y, d = _act(c["act"], x @ w + s["bias"])
        if c["residual"]:
            y = y + s["R"].float()
        out = {"Y": y.to(_T[c["out"]])}
        if step:
            dz = s["dY"].float() * d
            out["dX"] = (dz @ w.t()).to(_T[c["grad"]])
            out["dW"] = (x.t() @ dz).to(_T[c["grad"]])
            out["dbias"] = dz.sum(0)
        return out
    h, w = s["H"].float(), s["W"].float()
    t = c.get("temperature", 1.0)
    l = (h @ w) / t
    lse = l.amax(1, keepdim=True)
    lse = lse + torch.log(torch.exp(l - lse).sum(1, keepdim=True))
    if op == "ce":
        index, counts = s["target"][:, None], s["target"][:, None] != _IGNORE
        q = counts.float()
    else:
        index = s["index"]
        counts = index >= 0
        z = torch.where(counts, s["logits"] / t, float("-inf"))
        z = z - z.amax(1, keepdim=True).clamp_min(-3e38)
        q = torch.exp(z)
        q = q / q.sum(1, keepdim=True).clamp_min(1e-30)
    index = index.clamp_min(0)
    terms = lse - l.gather(1, index)
    if op == "distill":
        terms = terms + torch.log(q.clamp_min(1e-38))
    row_loss = t * t * (q * terms).sum(1)
    rows = counts.any(1, keepdim=True).float()
    scale = 1 / rows.sum().clamp_min(1)
    loss = (row_loss.sum() * scale).reshape(1)
    if not step:
        return {"loss": loss, "row_loss": row_loss}
    dl = torch.exp(l - lse) * rows
    dl = dl.scatter_add(1, index, -q) * (t * scale)
    return {"loss": loss, "dH": (dl @ w.t()).to(torch.bfloat16), "dW": (h.t() @ dl).to(torch.bfloat16)}


# ------------------------------------------------------------------- sizes --

def work(case):
    """Bytes that a pass has to move (each input once, each output once) and
    the flops of its products; the norms' few operations per element."""
    op, rows, step = case["op"], case["rows"], case["way"] == "step"
    size = {"bf16": 2, "fp32": 4}
    if op == "norm":
        dim = case["dim"]
        e = rows * dim
        b = e * (size[case["x"]] + size[case["y"]]) + 8 * dim
        f = 8 * e
        if step:
            b += e * (size[case["x"]] + size[case["y"]]) + 8 * dim
            f += 14 * e
        return {"bytes": b, "flops": f}
    if op == "dense":
        k, n = case["k"], case["n"]
        b = 2 * rows * k + 2 * k * n + 4 * n + rows * n * size[case["out"]] * (2 if case["residual"] else 1)
        f = 2 * rows * k * n
        if step:
            b += 2 * rows * n + (rows * k + k * n) * size[case["grad"]] + 4 * n
            f *= 3
        return {"bytes": b, "flops": f}
    dim, vocab = case["dim"], case["vocab"]
    b = 2 * (rows * dim + dim * vocab) + rows * (8 if op == "ce" else 12 * case["top"])
    f = 2 * rows * dim * vocab
    if step:
        b += 2 * (rows * dim + dim * vocab)
        f *= 3
    else:
        b += 4 * rows
    return {"bytes": b, "flops": f}


# -------------------------------------------------------------------- exact --

def exact(case, seed):
    """run()'s answer in 64 bits, from the definitions: the norm's gradients
    from its Jacobian, the losses from log-probabilities."""
    d = {k: (v.double() if v.is_floating_point() else v) for k, v in _data(case, seed).items()}
    op, step = case["op"], case["way"] == "step"
    if op == "norm":
        x, gamma, n = d["X"], d["gamma"], case["dim"]
        var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
        std = (var + _EPS) ** 0.5
        y = (x - mean) / std
        out = {"Y": torch.addcmul(d["beta"], y, gamma)}
        if step:
            dy = d["dY"]
            out["dgamma"], out["dbeta"] = torch.einsum("ij,ij->j", dy, y), dy.sum(0)
            # d y_j / d x_i = (delta_ij - 1/n - y_i y_j / n) / std
            u = dy * gamma
            out["dX"] = (u - (u.sum(1, keepdim=True) + y * (u * y).sum(1, keepdim=True)) / n) / std
        return out
    if op == "dense":
        z = torch.addmm(d["bias"], d["X"], d["W"]).requires_grad_(step)
        f = {"linear": lambda v: v * 1, "relu": torch.relu, "sigmoid": torch.sigmoid, "sine": torch.sin,
             "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[case["act"]]
        y = f(z)
        if step:
            dz, = torch.autograd.grad(y, z, d["dY"])
        y = y.detach() + d["R"] if case["residual"] else y.detach()
        if not step:
            return {"Y": y}
        return {"Y": y, "dX": torch.mm(dz, d["W"].t()), "dW": torch.mm(d["X"].t(), dz), "dbias": dz.sum(0)}
    rows, t = case["rows"], case.get("temperature", 1.0)
    if op == "ce":
        there = (d["target"] != _IGNORE)[:, None]
        index = torch.where(there, d["target"][:, None], 0)
        q = there.double()
    else:
        there = d["index"] >= 0
        index = torch.where(there, d["index"], 0)
        q = torch.nan_to_num(torch.softmax(torch.where(there, d["logits"] / t, -torch.inf), 1))
    live = there.any(1)
    n = max(1, int(live.sum()))
    row_loss = torch.zeros(rows, dtype=torch.float64, device="cuda")
    dH = torch.zeros_like(d["H"]) if step else None
    dW = torch.zeros_like(d["W"]) if step else None
    for r in range(0, rows, 2048):
        sl = slice(r, r + 2048)
        logp = torch.log_softmax(d["H"][sl] @ d["W"] / t, 1)
        qs = q[sl]
        row_loss[sl] = t * t * (torch.xlogy(qs, qs) - qs * logp.gather(1, index[sl])).sum(1)
        if step:
            g = logp.exp_().mul_(live[sl, None])
            g.scatter_add_(1, index[sl], -qs).mul_(t / n)
            dH[sl] = g @ d["W"].t()
            dW += d["H"][sl].t() @ g
    loss = (row_loss.sum() / n).reshape(1)
    return {"loss": loss, "dH": dH, "dW": dW} if step else {"loss": loss, "row_loss": row_loss}
