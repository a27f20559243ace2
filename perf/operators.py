"""Performance cases of the operators around a cascade's training step.

``acdc.forward`` gives a cascade's rows and ``acdc.backward`` takes a gradient
of them; these operators stand on either side of that pair:

* ``policy``      clipped policy loss with a KL term and an entropy bonus over
                  rows of logits, and its gradient.
* ``preference``  preference loss over pairs of token sequences (log ratios
                  against a reference), and its gradient.
* ``logprobs``    log-probabilities (and entropies) of given tokens;
                  ``logprobs_train`` adds the gradient.
* ``adamw``       AdamW over a list of tensors with moments in 32 or 8 bits,
                  alone or after the global norm of the gradients.

Logits are rows of ``classes`` values, ``stride`` apart (a cascade's width may
exceed the number of classes). A negative target marks a row that takes no
part; its logits need not be read.

8-bit moments are codes in float8 (e4m3) of m and of sqrt(v), with one float32
scale per 256 elements: the block's largest magnitude over 448.
"""

import math
import random

import torch

own = False

BLOCK = 256          # elements that share a scale (8-bit moments)
TOP = 448.0          # largest e4m3 value
TINY = 2.0 ** -9     # smallest positive e4m3 value

LR, BETAS, EPS, DECAY, STEP = 1e-3, (0.9, 0.999), 1e-8, 0.01, 7
CLIP = (0.2, 0.28)
KL, ENTROPY = 0.05, 0.01
BETA, SMOOTHING = 0.1, 0.05

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ the cases


def _rows(op, rows, classes, stride=0, dtype="f32", **more):
    return dict(more, op=op, rows=rows, classes=classes, stride=stride or classes, dtype=dtype)


def _pairs(pairs, longest, classes, stride=0, dtype="f32", **more):
    return dict(more, op="preference", pairs=pairs, longest=longest, classes=classes, stride=stride or classes,
                dtype=dtype)


def _tensors(bits, layout, count, elements, dtype="f32", clip=False, **more):
    return dict(more, op="adamw", bits=bits, layout=layout, count=count, elements=elements, dtype=dtype, clip=clip)


def listed():
    return [
        # the diagonals and the bias of one narrow layer: the smallest step, launches and host
        _tensors(32, "even", 3, 256, name="adamw_n256_k1"),
        # sixteen cascades of twelve 4096-wide layers (A, D, bias each), gradients clipped
        _tensors(32, "even", 48, 12 * 4096, clip=True, name="adamw_clip_n4096_k12_x16"),
        # a mixed-precision network around its structured layers: bf16 tensors of all sizes with float32 masters
        _tensors(32, "ragged", 200, 160_000_000, dtype="bf16_master", clip=True, name="adamw_clip_bf16_200_tensors"),
        # tensors of all sizes, moments in 8 bits
        _tensors(8, "ragged", 300, 20_000_000, name="adamw8_300_tensors"),
        # a few large embeddings and projections, moments in 8 bits to save memory
        _tensors(8, "even", 8, 50_000_001, name="adamw8_8_large"),
        # a bandit policy on the smallest layer: latency
        _rows("policy", 64, 256, name="policy_v256_r64"),
        # the benchmark cascade's rows read as logits
        _rows("policy", 8192, 4096, name="policy_v4096_r8192"),
        # a batch of trajectories over a large vocabulary
        _rows("policy", 8192, 65536, dtype="bf16", name="policy_v65536_r8192_bf16"),
        # short answers over 1000 classes in rows of 1024
        _pairs(12, 48, 1000, 1024, name="preference_v1000_p12"),
        # long answers over a vocabulary
        _pairs(48, 384, 32768, dtype="bf16", name="preference_v32768_p48_bf16"),
        # a few requests, one token each, over a large vocabulary: few rows, long ones
        _rows("logprobs", 8, 131072, name="logprobs_v131072_r8"),
        # flattened convolution features read as logits, with gradient
        _rows("logprobs_train", 1024, 9216, name="logprobs_train_v9216_r1024"),
    ]


def _spread(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    """Another case of the same ranges: one row to thousands, a handful of
    classes to 2^18, one tensor to hundreds, odd sizes as likely as even ones."""
    op = rng.choice(("adamw", "adamw", "policy", "policy", "preference", "logprobs", "logprobs_train"))
    if op == "adamw":
        count = _spread(rng, 1, 400)
        dtype = rng.choice(("f32", "f32", "f32_bf16", "bf16_master", "bf16"))
        if rng.random() < 0.5:
            return _tensors(rng.choice((8, 32)), "even", count, _spread(rng, 1, 200_000_000 // count), dtype,
                            rng.random() < 0.5)
        return _tensors(rng.choice((8, 32)), "ragged", count, _spread(rng, 4 * count, 200_000_000), dtype,
                        rng.random() < 0.5, shape=rng.randrange(1000))
    dtype = rng.choice(("f32", "bf16"))
    classes = _spread(rng, 8, 1 << 18)
    stride = classes + (rng.choice((1, 24, 128)) if rng.random() < 0.3 else 0)
    most = 250_000_000 // classes
    if op == "preference":
        longest = _spread(rng, 1, 512)
        pairs = _spread(rng, 1, max(1, min(256, most // (2 * longest))))
        return _pairs(pairs, min(longest, max(1, most // (2 * pairs))), classes, stride, dtype,
                      shape=rng.randrange(1000))
    return _rows(op, _spread(rng, 1, min(most, 20000)), classes, stride, dtype)


def _sizes(c):
    """Elements of each tensor of an ``adamw`` case."""
    if c["layout"] == "even":
        return [c["elements"]] * c["count"]
    rng = random.Random(c.get("shape", 0))
    share = [math.exp(rng.uniform(0.0, math.log(1e4))) for _ in range(c["count"])]
    total = sum(share)
    return [max(1, int(c["elements"] * s / total)) for s in share]


def _lengths(c):
    """Tokens of each of the 2 * pairs sequences of a ``preference`` case and
    how many of them, at its head, are prompt. Now and then one is empty."""
    rng = random.Random(c.get("shape", 0) + 77)
    got = []
    for _ in range(2 * c["pairs"]):
        n = 0 if rng.random() < 0.02 else rng.randint(max(1, c["longest"] // 2), c["longest"])
        got.append((n, n // 4))
    if not any(n for n, _ in got):
        got[0] = (1, 0)
    return got


def _row_count(c):
    return sum(n for n, _ in _lengths(c)) if c["op"] == "preference" else c["rows"]


def _idle(rows):
    """Rows of a ``policy`` or ``logprobs`` case that take no part."""
    return rows // 10


# ----------------------------------------------------------------- the inputs


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _logits(c, rows, gen):
    """Logits [rows, classes] in rows ``stride`` apart, and one token per row
    drawn from the distribution that they give."""
    V = c["classes"]
    full = torch.empty(rows, c["stride"], dtype=DTYPES[c["dtype"]], device="cuda")
    tokens = torch.empty(rows, dtype=torch.int64, device="cuda")
    step = max(1, (1 << 28) // c["stride"])
    for r in range(0, rows, step):
        x = torch.randn(min(step, rows - r), c["stride"], generator=gen, device="cuda").mul_(2.0)
        full[r:r + step] = x
        noise = torch.rand(x.shape[0], V, generator=gen, device="cuda").clamp_(min=1e-9).log_().neg_().log_().neg_()
        tokens[r:r + step] = (full[r:r + step, :V].float() + noise).argmax(1)
    return full[:, :V], tokens


def _token_logps(logits, tokens):
    out = []
    step = max(1, (1 << 28) // logits.shape[1])
    for r in range(0, logits.shape[0], step):
        out.append(_row_statistics(logits[r:r + step].float(), tokens[r:r + step])[1])
    return torch.cat(out) if out else torch.empty(0, device="cuda")


def _mask_rows(tokens, count, gen):
    tokens[torch.randperm(tokens.numel(), generator=gen, device="cuda")[:count]] = -1
    return tokens


def _prepare_rows(c, seed):
    gen = _generator(seed)
    rows = c["rows"]
    logits, tokens = _logits(c, rows, gen)

    def normal():
        return torch.randn(rows, generator=gen, device="cuda")

    s = {"logits": logits}
    if c["op"] == "policy":
        logp = _token_logps(logits, tokens)
        # policies a few updates apart. Where a ratio stands at a clip bound the gradient
        # jumps, so that rounding would decide: keep off the bounds
        shift = (0.15 * normal()).clamp_(-1.0, 1.0)
        for bound in (math.log(1 - CLIP[0]), math.log(1 + CLIP[1])):
            shift = torch.where((shift - bound).abs() < 2e-3, shift + 5e-3, shift)
        s["old"] = logp - shift
        s["ref"] = logp + 0.1 * normal()
        s["advantages"] = normal()
        s["weights"] = 0.5 + torch.rand(rows, generator=gen, device="cuda")
    else:
        s["grad_logp"], s["grad_entropy"] = normal(), 0.1 * normal()
    s["targets"] = _mask_rows(tokens, _idle(rows), gen)
    return s


def _prepare_pairs(c, seed):
    gen = _generator(seed)
    lengths = _lengths(c)
    rows = sum(n for n, _ in lengths)
    logits, tokens = _logits(c, rows, gen)
    offsets = [0]
    for n, _ in lengths:
        offsets.append(offsets[-1] + n)
    ref = _token_logps(logits, tokens) + 0.05 * torch.randn(rows, generator=gen, device="cuda")
    prompt = torch.tensor([t < k for n, k in lengths for t in range(n)], dtype=torch.bool, device="cuda")
    tokens[prompt] = -1
    return {"logits": logits, "targets": tokens, "ref": ref,
            "offsets": torch.tensor(offsets, dtype=torch.int32, device="cuda")}


def _padded(n):
    return -(-n // BLOCK) * BLOCK


def _prepare_tensors(c, seed):
    """One buffer each for all parameters, gradients and moments, and the
    tensors as parts of it: each starts at a multiple of 256 elements, and
    what lies between two of them is zero."""
    gen = _generator(seed)
    sizes = _sizes(c)
    starts, total = [], 0
    for n in sizes:
        starts.append(total)
        total += _padded(n)

    def parts(flat, unit=1):
        return [flat[a // unit:a // unit + -(-n // unit)] for a, n in zip(starts, sizes)]

    inside = torch.zeros(total, device="cuda")
    for part in parts(inside):
        part.fill_(1.0)

    def normal(std, mean=0.0):
        return torch.randn(total, generator=gen, device="cuda").mul_(std).add_(mean).mul_(inside)

    p_type = torch.bfloat16 if c["dtype"].startswith("bf16") else torch.float32
    g_type = torch.bfloat16 if "bf16" in c["dtype"] else torch.float32
    weights = normal(0.1, 1.0)
    s = {"param": weights.to(p_type), "grad": normal(0.02).to(g_type)}
    s["params"], s["grads"] = parts(s["param"]), parts(s["grad"])
    if c["dtype"] == "bf16_master":
        s["master"] = weights
        s["masters"] = parts(weights)
    m, root = normal(0.01), normal(0.02).abs_()  # root: the square root of v
    if c["bits"] == 32:
        s["m"], s["v"] = m, root.square_()
        s["moments"] = list(zip(parts(s["m"]), parts(s["v"])))
    else:
        s["m"], s["m_scale"] = _encode(m, False)
        s["v"], s["v_scale"] = _encode(root, True)
        s["moments"] = list(zip(parts(s["m"]), parts(s["v"]), parts(s["m_scale"], BLOCK), parts(s["v_scale"], BLOCK)))
    return s


def prepare(case, seed):
    make = {"adamw": _prepare_tensors, "preference": _prepare_pairs}.get(case["op"], _prepare_rows)
    return dict(make(case, seed), case=case)


# ------------------------------------------------ the operators in plain torch


def _row_statistics(x, targets):
    """(p, logp, entropy, safe targets) of rows of float32 logits."""
    t = targets.clamp(min=0).unsqueeze(1)
    top = x.amax(1, keepdim=True)
    shifted = x - top
    e = shifted.exp()
    total = e.sum(1, keepdim=True)
    p = e / total
    logp = shifted.gather(1, t) - total.log()
    entropy = total.log() - (p * shifted).sum(1, keepdim=True)
    return p, logp.squeeze(1), entropy.squeeze(1), t


def _row_gradient(p, logp_target, entropy, t, g, h):
    """dL/dlogits from g = dL/dlogp and h = dL/dentropy of each row."""
    log_p = torch.where(p > 0, p, torch.ones_like(p)).log()
    grad = p * (-g.unsqueeze(1) - h.unsqueeze(1) * (log_p + entropy.unsqueeze(1)))
    return grad.scatter_add(1, t, g.unsqueeze(1))


def _plain_logprobs(s, train):
    logits, targets = s["logits"], s["targets"]
    active = targets >= 0
    p, logp, entropy, t = _row_statistics(logits.float(), targets)
    out = {"logp": torch.where(active, logp, 0.0), "entropy": torch.where(active, entropy, 0.0)}
    if train:
        g, h = torch.where(active, s["grad_logp"], 0.0), torch.where(active, s["grad_entropy"], 0.0)
        out["grad"] = _row_gradient(p, logp, entropy, t, g, h).to(logits.dtype)
    return out


def _plain_policy(s):
    logits, targets, a = s["logits"], s["targets"], s["advantages"]
    active = targets >= 0
    w = torch.where(active, s["weights"], 0.0)
    total = w.sum()
    w = torch.where(total > 0, w / total, 0.0)
    p, logp, entropy, t = _row_statistics(logits.float(), targets)
    logp = torch.where(active, logp, 0.0)
    ratio = torch.where(active, (logp - s["old"]).exp(), 1.0)
    free, bounded = ratio * a, ratio.clamp(1 - CLIP[0], 1 + CLIP[1]) * a
    kept = free <= bounded
    policy = -torch.where(kept, free, bounded)
    gap = torch.where(active, s["ref"] - logp, 0.0)
    kl = gap.expm1() - gap
    loss = policy + KL * kl - ENTROPY * entropy
    stats = torch.stack([(w * v).sum() for v in (loss, policy, kl, entropy, (~kept).float(), ratio)])
    g = w * (torch.where(kept, -free, 0.0) - KL * gap.expm1())
    return {"stats": stats, "logp": logp,
            "grad": _row_gradient(p, logp, entropy, t, g, -ENTROPY * w).to(logits.dtype)}


def _plain_preference(s):
    logits, targets, offsets = s["logits"], s["targets"], s["offsets"].long()
    rows, sequences = logits.shape[0], offsets.numel() - 1
    active = targets >= 0
    p, logp, entropy, t = _row_statistics(logits.float(), targets)
    logp = torch.where(active, logp, 0.0)
    sequence = (torch.arange(rows, device=logits.device).unsqueeze(1) >= offsets[1:]).sum(1)
    member = sequence == torch.arange(sequences, device=logits.device).unsqueeze(1)
    excess = torch.where(active, logp - s["ref"], 0.0)
    reward = BETA * torch.where(member, excess, 0.0).sum(1)
    margin = reward[0::2] - reward[1::2]

    def softplus(z):  # log(1 + exp(z))
        return z.clamp(min=0) + (-z.abs()).exp().log1p()

    loss = (1 - SMOOTHING) * softplus(-margin) + SMOOTHING * softplus(margin)
    stats = torch.stack([v.mean() for v in (loss, (margin > 0).float(), margin, reward[0::2], reward[1::2])])
    slope = SMOOTHING / (1 + (-margin).exp()) - (1 - SMOOTHING) / (1 + margin.exp())
    slope = slope * (BETA / margin.numel())
    slope = torch.stack([slope, -slope], 1).view(-1)
    g = torch.where(active, slope[sequence.clamp(max=sequences - 1)], 0.0)
    return {"stats": stats, "logp": logp,
            "grad": _row_gradient(p, logp, entropy, t, g, torch.zeros_like(g)).to(logits.dtype)}


def _encode(x, positive):
    """(codes, scales) of values of which 256 in a row share a scale;
    ``positive`` values never become zero."""
    x = x.view(-1, BLOCK)
    scale = x.abs().amax(1, keepdim=True) / TOP
    q = torch.where(scale > 0, x / scale, 0.0)
    if positive:
        q = torch.where((x > 0) & (q < TINY), TINY, q)
    return q.to(torch.float8_e4m3fn).view(-1), scale.view(-1)


def _decode(codes, scale):
    return (codes.float().view(-1, BLOCK) * scale.unsqueeze(1)).view(-1)


def _plain_adamw(s):
    """The step of all tensors at once, in the buffers that they are parts of:
    what is zero between them stays zero."""
    c = s["case"]
    out = {}
    g = s["grad"].float()
    if c["clip"]:
        norm = g.square().sum().sqrt()
        scale = (1.0 / (norm + 1e-6)).clamp(max=1.0)
        out["norm"] = torch.stack([norm, scale])
        g = g * scale
    if c["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m, v = _decode(s["m"], s["m_scale"]), _decode(s["v"], s["v_scale"]).square()
    m = BETAS[0] * m + (1 - BETAS[0]) * g
    v = BETAS[1] * v + (1 - BETAS[1]) * g * g
    root = v.sqrt()
    w = s["master"] if "master" in s else s["param"].float()
    step = m / (root / math.sqrt(1 - BETAS[1] ** STEP) + EPS)
    w = w * (1 - LR * DECAY) - LR / (1 - BETAS[0] ** STEP) * step
    if "master" in s:
        s["master"].copy_(w)
    s["param"].copy_(w)
    if c["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        for name, x in (("m", m), ("v", root)):
            codes, scales = _encode(x, name == "v")
            s[name].copy_(codes)
            s[name + "_scale"].copy_(scales)
    return dict(out, **_adamw_state(s))


def _adamw_state(s):
    return {k: s[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale") if k in s}


def _plain(s):
    op = s["case"]["op"]
    if op == "adamw":
        return _plain_adamw(s)
    if op == "policy":
        return _plain_policy(s)
    if op == "preference":
        return _plain_preference(s)
    return _plain_logprobs(s, op == "logprobs_train")


# ------------------------------------------------- the framework's own calls


def _own(s):
    from paper_1511_05946_amd import losses, optim

    c = s["case"]
    op = c["op"]
    if op == "adamw":
        out, scale = {}, None
        if c["clip"]:
            out["norm"] = optim.grad_norm(s["grads"], max_norm=1.0)
            scale = out["norm"][1:]
        optim.adamw_step(s["params"], s["grads"], s["moments"], STEP, lr=LR, betas=BETAS, eps=EPS,
                         weight_decay=DECAY, masters=s.get("masters"), grad_scale=scale)
        return dict(out, **_adamw_state(s))
    if op == "policy":
        r = losses.policy_loss(s["logits"], s["targets"], s["old"], s["advantages"], logp_ref=s["ref"],
                               weights=s["weights"], clip=CLIP, kl_coef=KL, entropy_coef=ENTROPY)
        return {"stats": r.stats, "logp": r.logp, "grad": r.grad_logits}
    if op == "preference":
        r = losses.preference_loss(s["logits"], s["targets"], s["offsets"], s["ref"], beta=BETA,
                                   label_smoothing=SMOOTHING)
        return {"stats": r.stats, "logp": r.logp, "grad": r.grad_logits}
    train = op == "logprobs_train"
    r = losses.token_logprobs(s["logits"], s["targets"], entropy=True, save=train)
    out = {"logp": r.logp, "entropy": r.entropy}
    if train:
        out["grad"] = losses.token_logprobs_backward(s["logits"], s["targets"], r.saved, s["grad_logp"],
                                                     s["grad_entropy"])
    return out


def run(state):
    return _own(state) if own else _plain(state)


# --------------------------------------------------------- what a pass needs


def work(case):
    op = case["op"]
    if op == "adamw":
        n = sum(_sizes(case))
        p, g = (2 if case["dtype"].startswith("bf16") else 4), (2 if "bf16" in case["dtype"] else 4)
        master = case["dtype"] == "bf16_master"
        # parameters are read unless masters stand for them; moments are read and written
        params = 8 + p if master else 2 * p
        moments = 16 if case["bits"] == 32 else 4 * (1 + 4 / BLOCK)
        return {"bytes": n * (g + params + moments), "flops": 14 * n + (2 * n if case["clip"] else 0)}
    size = 2 if case["dtype"] == "bf16" else 4
    rows, V = _row_count(case), case["classes"]
    idle = sum(k for _, k in _lengths(case)) if op == "preference" else _idle(rows)
    used = rows - idle
    if op == "logprobs":
        return {"bytes": used * V * size + rows * 16, "flops": used * V * 5}
    return {"bytes": (used + rows) * V * size + rows * 28, "flops": used * V * 9}


# ------------------------------------------------------- the values in 64 bits


def _exact_log_softmax(s):
    """(logits that autograd follows, log-probabilities, entropies)."""
    x = s["logits"].double().requires_grad_(True)
    log_p = x - torch.logsumexp(x, 1, keepdim=True)
    p = log_p.exp()
    return x, log_p, -(p * log_p).sum(1)


def _exact_rows(s):
    c = s["case"]
    x, log_p, entropy = _exact_log_softmax(s)
    on = (s["targets"] >= 0).double()
    rows = torch.arange(x.shape[0], device=x.device)
    logp = log_p[rows, s["targets"].clamp(min=0)]
    out = {"logp": (logp * on).detach()}
    if c["op"].startswith("logprobs"):
        out["entropy"] = (entropy * on).detach()
        if c["op"] == "logprobs":
            return out
        objective = (on * (logp * s["grad_logp"].double() + entropy * s["grad_entropy"].double())).sum()
    elif c["op"] == "policy":
        a, w = s["advantages"].double(), on * s["weights"].double()
        w = w / w.sum() if float(w.sum()) > 0 else w * 0
        ratio = torch.exp(logp - s["old"].double())
        policy = -torch.minimum(ratio * a, torch.clamp(ratio, 1 - CLIP[0], 1 + CLIP[1]) * a)
        kl = torch.exp(s["ref"].double() - logp) - (s["ref"].double() - logp) - 1
        cut = (torch.clamp(ratio, 1 - CLIP[0], 1 + CLIP[1]) * a < ratio * a).double()
        means = [(w * v).sum() for v in (policy + KL * kl - ENTROPY * entropy, policy, kl, entropy, cut, ratio)]
        out["stats"] = torch.stack(means).detach()
        objective = means[0]
    else:
        lengths = [n for n, _ in _lengths(c)]
        reward = torch.stack([BETA * v.sum() for v in ((logp - s["ref"].double()) * on).split(lengths)])
        good, bad = reward[0::2], reward[1::2]
        margin = good - bad
        loss = -(1 - SMOOTHING) * torch.nn.functional.logsigmoid(margin) \
            - SMOOTHING * torch.nn.functional.logsigmoid(-margin)
        means = [v.mean() for v in (loss, (margin > 0).double(), margin, good, bad)]
        out["stats"] = torch.stack(means).detach()
        objective = means[0]
    out["grad"], = torch.autograd.grad(objective, x)
    return out


def _exact_adamw(s):
    c = s["case"]
    out = {}
    g = s["grad"].double()
    if c["clip"]:
        norm = torch.linalg.vector_norm(g)
        factor = min(1.0, 1.0 / (float(norm) + 1e-6))
        out["norm"] = torch.tensor([float(norm), factor], dtype=torch.float64)
        g *= factor
    m, v = s["m"].double(), s["v"].double()
    if c["bits"] == 8:
        m *= s["m_scale"].double().repeat_interleave(BLOCK)
        v *= s["v_scale"].double().repeat_interleave(BLOCK)
        v *= v
    (b1, b2), w = BETAS, s.get("master", s["param"]).double()
    m.lerp_(g, 1 - b1)
    v.lerp_(g * g, 1 - b2)
    w -= LR * DECAY * w + LR * (m / (1 - b1 ** STEP)) / ((v / (1 - b2 ** STEP)).sqrt() + EPS)
    out["param"] = w
    if "master" in s:
        out["master"] = w
    if c["bits"] == 32:
        return dict(out, m=m, v=v)
    for name, x in (("m", m), ("v", v.sqrt())):
        x = x.view(-1, BLOCK)
        scale = x.abs().max(dim=1).values / TOP
        q = x / torch.where(scale == 0, torch.ones_like(scale), scale).unsqueeze(1)
        if name == "v":
            q[(x > 0) & (q < TINY)] = TINY
        out[name], out[name + "_scale"] = q.view(-1).to(torch.float8_e4m3fn).double(), scale
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_adamw(s) if case["op"] == "adamw" else _exact_rows(s)
