"""Performance cases of the operators that make a language model of a cascade.

A cascade maps rows of N values to rows of N values. These operators turn
tokens into such rows and rows into a loss over a vocabulary:

* ``vocab``       cross entropy over a vocabulary from hidden rows and a weight
                  [classes, width], without keeping the logits, with the
                  gradients of both; ``vocab_score`` gives the
                  log-probabilities alone.
* ``norm``        layer norm and its backward pass with the gradients of weight
                  and bias; ``norm_forward`` the forward pass alone.
* ``embedding``   rows of a weight looked up by tokens, times a scale, and the
                  gradient of the weight; ``embedding_forward`` the lookup
                  alone.

A negative target or token marks a row that takes no part (a prompt, padding).
"""

import math
import random

import torch

own = False

EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


# ------------------------------------------------------------------ the cases


def _vocab(op, rows, width, classes, dtype="bf16", weighted=False, **more):
    return dict(more, op=op, rows=rows, width=width, classes=classes, dtype=dtype, weighted=weighted)


def _norm(op, rows, width, stride=0, dtype="f32", out="", **more):
    return dict(more, op=op, rows=rows, width=width, stride=stride or width, dtype=dtype, out=out or dtype)


def _embedding(op, tokens, width, classes, dtype="f32", out="", **more):
    return dict(more, op=op, tokens=tokens, width=width, classes=classes, dtype=dtype, out=out or dtype)


def listed():
    return [
        # a narrow cascade's rows over a small set of classes: latency
        _vocab("vocab", 64, 256, 1000, "f32", name="vocab_n256_v1000_r64"),
        # a training step's tokens on a cascade of middle width
        _vocab("vocab", 2048, 1024, 32768, name="vocab_n1024_v32768_r2048_bf16"),
        # the benchmark cascade's batch over a large vocabulary
        _vocab("vocab", 8192, 4096, 65536, name="vocab_n4096_v65536_r8192_bf16"),
        # float32 rows as a cascade leaves them, an odd vocabulary, weighted rows
        _vocab("vocab", 1000, 1024, 20001, "f32", True, name="vocab_n1024_v20001_r1000"),
        # candidates of a few requests scored: few rows, the weight is what is read
        _vocab("vocab_score", 8, 4096, 131072, name="vocab_score_n4096_v131072_r8_bf16"),
        # the smallest layer's rows: latency
        _norm("norm", 64, 256, name="norm_n256_r64"),
        # the benchmark cascade's batch, handed on in bfloat16
        _norm("norm", 8192, 4096, dtype="f32", out="bf16", name="norm_n4096_r8192_f32_bf16"),
        # odd rows inside wider ones
        _norm("norm", 20011, 1000, 1024, "bf16", name="norm_n1000_r20011_bf16"),
        # flattened convolution features, forward
        _norm("norm_forward", 1024, 9216, name="norm_forward_n9216_r1024"),
        # a batch of tokens into float32 rows, the weight in bfloat16
        _embedding("embedding", 8192, 4096, 65536, "bf16", "f32", name="embedding_n4096_v65536_t8192_bf16"),
        # many tokens of a small vocabulary: long runs of one token
        _embedding("embedding", 131072, 257, 1000, name="embedding_n257_v1000_t131072"),
        # one token of each of a few sequences
        _embedding("embedding_forward", 16, 1024, 32768, name="embedding_forward_n1024_v32768_t16"),
    ]


def _spread(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    """Another case of the same ranges: one row to many thousands, a handful of
    classes to 2^17, odd sizes as likely as even ones."""
    op = rng.choice(("vocab", "vocab", "vocab_score", "norm", "norm", "norm_forward", "embedding", "embedding",
                     "embedding_forward"))
    dtype = rng.choice(("f32", "bf16"))
    if op.startswith("vocab"):
        most = 2_000_000_000_000 // (6 if dtype == "f32" else 1)
        classes = _spread(rng, 8, 1 << 17)
        width = _spread(rng, 8, 8192)
        if rng.random() < 0.5:
            width = -(-width // 64) * 64
        rows = _spread(rng, 1, max(1, min(16384, most // (classes * width))))
        return _vocab(op, rows, width, classes, dtype, rng.random() < 0.3)
    out = rng.choice((dtype, dtype, "f32", "bf16"))
    if op.startswith("norm"):
        width = _spread(rng, 2, 1 << 16)
        stride = width + (rng.choice((1, 24, 128)) if rng.random() < 0.3 else 0)
        return _norm(op, _spread(rng, 1, min(1 << 18, 100_000_000 // width)), width, stride, dtype, out)
    width = _spread(rng, 2, 9216)
    return _embedding(op, _spread(rng, 1, min(1 << 18, 100_000_000 // width)), width,
                      _spread(rng, 8, min(1 << 18, 260_000_000 // width)), dtype, out)


def _idle(rows):
    """Rows that take no part."""
    return rows // 10


# ----------------------------------------------------------------- the inputs


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _tokens(count, classes, gen):
    """Tokens by the frequencies of words: the k-th about as often as 1 / k."""
    u = torch.rand(count, generator=gen, device="cuda", dtype=torch.float64)
    t = ((u * math.log(classes + 1)).exp() - 1).long().clamp_(0, classes - 1)
    t[torch.randperm(count, generator=gen, device="cuda")[:_idle(count)]] = -1
    return t


def _normal(rows, width, gen, std=1.0, dtype=torch.float32, stride=0):
    """Normal values in rows ``stride`` apart."""
    stride = stride or width
    full = torch.empty(rows, stride, dtype=dtype, device="cuda")
    step = max(1, (1 << 28) // stride)
    for r in range(0, rows, step):
        full[r:r + step] = torch.randn(min(step, rows - r), stride, generator=gen, device="cuda").mul_(std)
    return full[:, :width]


def prepare(case, seed):
    gen = _generator(seed)
    c, op = case, case["op"]
    dtype = DTYPES[c["dtype"]]
    s = {"case": case}
    if op.startswith("vocab"):
        # rows as a normalisation leaves them, logits of standard deviation 2
        s["hidden"] = _normal(c["rows"], c["width"], gen, 1.0, dtype)
        s["weight"] = _normal(c["classes"], c["width"], gen, 2.0 / math.sqrt(c["width"]), dtype)
        s["targets"] = _tokens(c["rows"], c["classes"], gen)
        s["weights"] = 0.5 + torch.rand(c["rows"], generator=gen, device="cuda") if c["weighted"] else None
    elif op.startswith("norm"):
        # rows with means of their own and a few wide columns
        x = _normal(c["rows"], c["stride"], gen, 1.0)
        x += 0.5 * torch.randn(c["rows"], 1, generator=gen, device="cuda")
        x[:, ::97] *= 8.0
        s["x"] = x.to(dtype)[:, :c["width"]]
        s["weight"] = 1 + 0.1 * torch.randn(c["width"], generator=gen, device="cuda")
        s["bias"] = 0.1 * torch.randn(c["width"], generator=gen, device="cuda")
        if op == "norm":
            s["grad"] = _normal(c["rows"], c["width"], gen, 0.01, DTYPES[c["out"]])
    else:
        s["tokens"] = _tokens(c["tokens"], c["classes"], gen)
        s["weight"] = _normal(c["classes"], c["width"], gen, 0.02, dtype)
        s["scale"] = math.sqrt(c["width"])
        if op == "embedding":
            s["grad"] = _normal(c["tokens"], c["width"], gen, 0.01, DTYPES[c["out"]])
    return s


# ------------------------------------------------ the operators in plain torch


def _plain_vocab(s, train):
    hidden, weight, targets = s["hidden"], s["weight"], s["targets"]
    h, w = hidden.float(), weight.float()
    active = targets >= 0
    t = targets.clamp(min=0).unsqueeze(1)
    x = h @ w.t()
    x -= x.amax(1, keepdim=True)
    xt = x.gather(1, t)
    e = x.exp_()
    total = e.sum(1, keepdim=True)
    logp = torch.where(active, (xt - total.log()).squeeze(1), 0.0)
    if not train:
        return {"logp": logp}
    share = active.float() if s["weights"] is None else torch.where(active, s["weights"], 0.0)
    all_of = share.sum()
    share = torch.where(all_of > 0, share / all_of, 0.0)
    e *= (share / total.squeeze(1)).unsqueeze(1)
    grad = e.scatter_add_(1, t, -share.unsqueeze(1))
    return {"stats": torch.stack([-(share * logp).sum(), all_of]), "logp": logp,
            "grad_hidden": (grad @ w).to(hidden.dtype), "grad_weight": (grad.t() @ h).to(weight.dtype)}


def _plain_norm(s, train):
    x, w = s["x"].float(), s["weight"]
    centred = x - x.mean(1, keepdim=True)
    rstd = (centred.square().mean(1, keepdim=True) + EPS).rsqrt()
    unit = centred * rstd
    y = (unit * w + s["bias"]).to(DTYPES[s["case"]["out"]])
    if not train:
        return {"y": y}
    g = s["grad"].float()
    inner = g * w
    gx = rstd * (inner - inner.mean(1, keepdim=True) - unit * (inner * unit).mean(1, keepdim=True))
    return {"y": y, "grad_x": gx.to(s["x"].dtype), "grad_weight": (g * unit).sum(0), "grad_bias": g.sum(0)}


def _plain_embedding(s, train):
    tokens, weight, scale = s["tokens"], s["weight"], s["scale"]
    active = tokens >= 0
    rows = weight[tokens.clamp(min=0)].float() * scale
    out = {"rows": torch.where(active.unsqueeze(1), rows, 0.0).to(DTYPES[s["case"]["out"]])}
    if train:
        order = torch.argsort(tokens, stable=True)
        order = order[tokens[order] >= 0]
        grad = torch.zeros(weight.shape, device="cuda")
        grad.index_put_((tokens[order],), s["grad"][order].float() * scale, accumulate=True)
        out["grad_weight"] = grad.to(weight.dtype)
    return out


def _plain(s):
    op = s["case"]["op"]
    if op.startswith("vocab"):
        return _plain_vocab(s, op == "vocab")
    if op.startswith("norm"):
        return _plain_norm(s, op == "norm")
    return _plain_embedding(s, op == "embedding")


# ------------------------------------------------------- the framework's calls


def _own(s):
    from paper_1511_05946_amd import layers, losses

    c, op = s["case"], s["case"]["op"]
    if op == "vocab":
        r = losses.vocab_loss(s["hidden"], s["weight"], s["targets"], weights=s["weights"])
        return {"stats": r.stats, "logp": r.logp, "grad_hidden": r.grad_hidden, "grad_weight": r.grad_weight}
    if op == "vocab_score":
        return {"logp": losses.vocab_logprobs(s["hidden"], s["weight"], s["targets"]).logp}
    if op.startswith("norm"):
        train = op == "norm"
        r = layers.layer_norm(s["x"], s["weight"], s["bias"], EPS, dtype=DTYPES[c["out"]], save=train)
        if not train:
            return {"y": r.y}
        gx, gw, gb = layers.layer_norm_backward(s["x"], s["grad"], s["weight"], r.saved)
        return {"y": r.y, "grad_x": gx, "grad_weight": gw, "grad_bias": gb}
    out = {"rows": layers.embedding(s["tokens"], s["weight"], s["scale"], dtype=DTYPES[c["out"]])}
    if op == "embedding":
        out["grad_weight"] = layers.embedding_backward(s["tokens"], s["grad"], c["classes"], s["scale"],
                                                       dtype=s["weight"].dtype)
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------ definitions in 64 bits


def _exact_vocab(c, s):
    train = c["op"] == "vocab"
    W = s["weight"].double()
    on = (s["targets"] >= 0).nonzero().squeeze(1)
    logp = torch.zeros(c["rows"], dtype=torch.float64, device="cuda")
    share = torch.zeros_like(logp)
    share[on] = 1.0 if s["weights"] is None else s["weights"][on].double()
    total = share.sum()
    if train:
        grad_hidden = torch.zeros(c["rows"], c["width"], dtype=torch.float64, device="cuda")
        grad_weight = torch.zeros_like(W)
    for part in on.split(max(1, (1 << 28) // c["classes"])):
        H, t = s["hidden"][part].double(), s["targets"][part]
        logits = torch.mm(H, W.t().contiguous())
        log_p = logits - torch.logsumexp(logits, 1, keepdim=True)
        pick = torch.arange(len(part), device="cuda")
        logp[part] = log_p[pick, t]
        if train:
            p = torch.exp(log_p)
            p[pick, t] -= 1
            p *= (share[part] / total)[:, None]
            grad_hidden[part] = torch.mm(p, W)
            grad_weight += torch.mm(p.t().contiguous(), H)
    if not train:
        return {"logp": logp}
    loss = -(share * logp).sum() / total if len(on) else total
    return {"stats": torch.stack([loss, total]), "logp": logp, "grad_hidden": grad_hidden, "grad_weight": grad_weight}


def _exact_norm(c, s):
    train = c["op"] == "norm"
    w, b, n = s["weight"].double(), s["bias"].double(), c["width"]
    y, gx = [], []
    gw, gb = torch.zeros_like(w), torch.zeros_like(w)
    step = max(1, (1 << 27) // n)
    for r in range(0, c["rows"], step):
        x = s["x"][r:r + step].double()
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        sigma = torch.sqrt(var + EPS)
        xhat = (x - mean) / sigma
        y.append(xhat * w + b)
        if train:
            g = s["grad"][r:r + step].double()
            gb += g.sum(0)
            gw += (g * xhat).sum(0)
            d = g * w / sigma
            gx.append(d - d.sum(1, keepdim=True) / n - xhat * ((d * xhat).sum(1, keepdim=True) / n))
    out = {"y": torch.cat(y)}
    if train:
        out.update(grad_x=torch.cat(gx), grad_weight=gw, grad_bias=gb)
    return out


def _exact_embedding(c, s):
    tokens, W = s["tokens"], s["weight"].double()
    on = (tokens >= 0).nonzero().squeeze(1)
    rows = torch.zeros(c["tokens"], c["width"], dtype=torch.float64, device="cuda")
    rows[on] = W.index_select(0, tokens[on]) * s["scale"]
    out = {"rows": rows}
    if c["op"] == "embedding":
        out["grad_weight"] = torch.zeros_like(W).index_add_(0, tokens[on], s["grad"][on].double()) * s["scale"]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("vocab"):
        return _exact_vocab(case, s)
    return (_exact_norm if case["op"].startswith("norm") else _exact_embedding)(case, s)


# ------------------------------------------------------------- the work at least


def work(case):
    c, op = case, case["op"]
    e = BYTES[c["dtype"]]
    if op.startswith("vocab"):
        rows, n, v = c["rows"], c["width"], c["classes"]
        train = op == "vocab"
        tensors = (rows * n + v * n) * e
        product = 2 * (rows - _idle(rows)) * n * v
        return {"bytes": tensors * (2 if train else 1) + rows * (16 if c["weighted"] else 12),
                "flops": product * (3 if train else 1)}
    o = BYTES[c["out"]]
    if op.startswith("norm"):
        values = c["rows"] * c["width"]
        train = op == "norm"
        return {"bytes": values * (2 * (e + o) if train else e + o) + c["width"] * (16 if train else 8),
                "flops": values * (20 if train else 8)}
    t, n, v = c["tokens"], c["width"], c["classes"]
    on = t - _idle(t)
    train = op == "embedding"
    return {"bytes": 8 * t + min(on, v) * n * e + t * n * o + (on * n * o + v * n * e if train else 0),
            "flops": on * n * (2 if train else 1)}
