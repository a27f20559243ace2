"""Losses over rows of logits on the GPU against their definitions in 64 bits."""

import numpy as np
import pytest

import train_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1511_05946_amd import losses
    return torch, losses


# rows, classes, distance of rows, type, bits of the targets: one class to more than a
# workgroup holds, odd and even, one row and more rows than a workgroup has threads
SHAPES = [(1, 1, 1, "float32", 64), (3, 7, 7, "float32", 32), (300, 8, 8, "float32", 64), (64, 256, 256, "float32", 64),
          (37, 1000, 1024, "float32", 64), (5, 1023, 1025, "bfloat16", 32), (9, 4096, 4096, "bfloat16", 64),
          (130, 33, 40, "bfloat16", 64), (6, 9216, 9216, "float32", 64), (2, 16387, 16387, "float32", 32),
          (3, 50001, 50001, "bfloat16", 64), (2, 131073, 131073, "float32", 64), (1, 262144, 262144, "bfloat16", 64),
          (700, 513, 513, "float32", 64), (1100, 2048, 2056, "bfloat16", 32), (600, 20000, 20000, "bfloat16", 64),
          (520, 40001, 40001, "float32", 64), (4, 300001, 300001, "float32", 64),
          # more than a workgroup's registers hold, with rows enough for one pass; rows in parts, more than 16
          (130, 66001, 66003, "float32", 64), (128, 132001, 132001, "bfloat16", 32), (40, 20001, 20001, "float32", 64),
          # tiles of short rows: several of them, each number of chunks a lane
          (5000, 9, 9, "bfloat16", 64), (300, 400, 401, "float32", 64), (200, 1500, 1504, "bfloat16", 64),
          (150, 4000, 4001, "bfloat16", 64)]


def make(torch, shape, seed=0, spread=2.0, idle=0.2):
    """Logits (NaN and infinities in idle rows) and targets on the GPU, and both on the CPU."""
    rows, V, stride, dtype, bits = shape
    print(f"[case] {shape} seed={seed}", flush=True)
    gen = torch.Generator().manual_seed(1000 * seed + rows + V)
    full = (spread * torch.randn(rows, stride, generator=gen)).to(getattr(torch, dtype))
    t = torch.randint(0, V, (rows,), generator=gen)
    off = torch.rand(rows, generator=gen) < idle
    if rows > 1:
        off[0], off[1] = False, True
    else:
        off[:] = False
    t[off] = -1 - torch.randint(0, 100, (int(off.sum()),), generator=gen)
    x = full[:, :V].double().numpy()
    full[off] = torch.tensor([float("nan"), float("inf"), -float("inf")]).to(full.dtype).repeat(stride)[:stride]
    return (full.cuda()[:, :V], t.to(getattr(torch, f"int{bits}")).cuda(), x, t.numpy(), ~off.numpy())


def close(got, ref, tol, what):
    got = got.double().cpu().numpy()
    assert got.shape == ref.shape
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[:3], got[bad][:3], ref[bad][:3], np.broadcast_to(tol, ref.shape)[bad][:3])


def check_gradient(got, x, t, on, g, h, bf16):
    tt = np.clip(t, 0, x.shape[1] - 1)
    p, logp, ent, spread = R.rows(x, t)
    g, h = np.where(on, g, 0.0), np.where(on, h, 0.0)
    ref = R.gradient(p, ent, tt, g, h)
    close(got, ref, R.gradient_tolerance(p, ref, ent, spread, tt, g, h, bf16), "gradient")


@pytest.mark.parametrize("shape", SHAPES)
def test_token_logprobs_and_gradient(env, shape):
    torch, losses = env
    logits, targets, x, t, on = make(torch, shape)
    rows = len(t)
    r = losses.token_logprobs(logits, targets, entropy=True, save=True)
    p, logp, ent, spread = R.rows(x, t)
    tol = R.logp_tolerance(logp, spread)
    close(r.logp, np.where(on, logp, 0.0), tol, "logp")
    close(r.entropy, np.where(on, ent, 0.0), tol * 2, "entropy")
    rng = np.random.RandomState(3)
    g, h = rng.randn(rows).astype(np.float32), rng.randn(rows).astype(np.float32)
    gt, ht = torch.from_numpy(g).cuda(), torch.from_numpy(h).cuda()
    grad = losses.token_logprobs_backward(logits, targets, r.saved, gt, ht)
    check_gradient(grad, x, t, on, g.astype(float), h.astype(float), logits.dtype is torch.bfloat16)
    # in place of the logits (their neighbours in wider rows stay), and again: bit for bit
    again = losses.token_logprobs_backward(logits, targets, r.saved, gt, ht, out=logits)
    assert again.data_ptr() == logits.data_ptr() and torch.equal(again, grad)
    # without the entropies
    logits2, targets2, *_ = make(torch, shape)
    assert torch.equal(losses.token_logprobs(logits2, targets2).logp, r.logp)
    scale = torch.tensor([0.5], device="cuda")
    half = losses.token_logprobs_backward(logits2, targets2, r.saved, gt, scale=scale)
    check_gradient(half, x, t, on, 0.5 * g.astype(float), np.zeros(rows), logits.dtype is torch.bfloat16)


def policy_inputs(torch, logp, rows, seed):
    rng = np.random.RandomState(seed)
    shift = np.clip(0.3 * rng.randn(rows), -1, 1)
    for b in (np.log(0.8), np.log(1.3)):   # off the clip bounds, where rounding would decide
        shift = np.where(np.abs(shift - b) < 1e-3, shift + 3e-3, shift)
    f = np.float32
    old, ref, adv, w = (logp - shift).astype(f), (logp + 0.2 * rng.randn(rows)).astype(f), rng.randn(rows).astype(f), \
        rng.rand(rows).astype(f) + f(0.5)
    if rows > 3:
        w[2] = 0.0
    return old, ref, adv, w


def check_stats(got, ref, size):
    """A weighted mean of values that carry the rounding of logp."""
    got = got.double().cpu().numpy()
    assert np.all(np.abs(got - ref) <= size), (got, ref)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("options", ["full", "plain", "sum"])
def test_policy_loss(env, shape, options):
    torch, losses = env
    logits, targets, x, t, on = make(torch, shape, 1)
    rows, bf16 = len(t), logits.dtype is torch.bfloat16
    p, logp, ent, spread = R.rows(x, t)
    old, ref, adv, w = policy_inputs(torch, logp, rows, 5)
    old[~on] = np.nan      # nothing of an idle row is looked at
    adv[~on] = np.inf
    kw = {"full": dict(logp_ref=ref, weights=w, clip=(0.2, 0.3), kl_coef=0.1, entropy_coef=0.02),
          "plain": dict(clip=(0.2, 0.3)),
          "sum": dict(weights=w, clip=(0.2, 0.3), entropy_coef=-0.05, mean=False, grad_scale=0.25)}[options]
    dev = {k: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for k, v in kw.items()}
    r = losses.policy_loss(logits, targets, torch.from_numpy(old).cuda(), torch.from_numpy(adv).cuda(), save=True, **dev)
    weights = np.where(on, kw.get("weights", np.ones(rows)).astype(float), 0.0)
    part = weights != 0
    safe = lambda v: np.where(part, v, 0.0).astype(float)  # noqa: E731
    stats, g, h = R.policy(p, logp, ent, part, safe(old), safe(ref) if "logp_ref" in kw else None, safe(adv), weights,
                           kw["clip"], kw.get("kl_coef", 0.0), kw.get("entropy_coef", 0.0), kw.get("mean", True))
    tol = R.logp_tolerance(logp, spread)
    close(r.logp, np.where(part, logp, 0.0), tol, "logp")
    # every value of a row moves by at most its logp's error times (|a| ratio + kl_coef exp(k) + 2) and some units
    norm = weights / weights.sum() if kw.get("mean", True) and weights.sum() else weights
    ratio = np.where(part, np.exp(logp - safe(old)), 0.0)
    k = np.where(part, np.abs(np.expm1(safe(ref) - logp)), 0.0)
    move = (2 * tol + 8 * R.EPS) * (np.abs(safe(adv)) * ratio + ratio + 2 * k + np.abs(ent) + 2)
    check_stats(r.stats, stats, (np.abs(norm) * move).sum() + 16 * R.EPS * np.abs(stats))
    c = kw.get("grad_scale", 1.0)
    gtol = np.abs(norm) * move
    got = r.row_grads.double().cpu().numpy()
    assert np.all(np.abs(got[0] - g) <= gtol + 8 * R.EPS * np.abs(g)) and np.all(np.abs(got[1] - h) <= 8 * R.EPS * np.abs(h))
    # the gradient of the logits follows from the row gradients
    check_gradient(r.grad_logits, x, t, part, c * got[0], c * got[1], bf16)
    values = losses.policy_loss(logits, targets, torch.from_numpy(old).cuda(), torch.from_numpy(adv).cuda(), grad=False,
                                **dev)
    assert values.grad_logits is None
    check_stats(values.stats, stats, (np.abs(norm) * move).sum() + 16 * R.EPS * np.abs(stats))
    # in place
    inplace = losses.policy_loss(logits, targets, torch.from_numpy(old).cuda(), torch.from_numpy(adv).cuda(),
                                 out=logits, **dev)
    assert torch.equal(inplace.grad_logits, r.grad_logits) and torch.equal(inplace.stats, r.stats)


def lengths_for(rows, seed):
    """Offsets of an even number of sequences over part of the rows, some of them empty."""
    rng = np.random.RandomState(seed)
    first, last = (1, rows - 1) if rows > 4 else (0, rows)
    count = 2 * max(1, min(40, (last - first) // 3))
    cuts = np.sort(rng.randint(first, last + 1, count - 1))
    return np.concatenate([[first], cuts, [last]])


@pytest.mark.parametrize("shape", SHAPES)
def test_preference_loss(env, shape):
    torch, losses = env
    logits, targets, x, t, on = make(torch, shape, 2)
    rows, bf16 = len(t), logits.dtype is torch.bfloat16
    p, logp, ent, spread = R.rows(x, t)
    ref = (logp + 0.3 * np.random.RandomState(1).randn(rows)).astype(np.float32)
    ref[~on] = np.nan
    offsets = lengths_for(rows, rows)
    beta, e = 0.3, 0.1
    r = losses.preference_loss(logits, targets, torch.from_numpy(offsets.astype(np.int32 if rows % 2 else np.int64)).cuda(),
                               torch.from_numpy(ref).cuda(), beta=beta, label_smoothing=e, grad_scale=2.0, save=True)
    stats, g = R.preference(logp, on, offsets, ref.astype(float), beta, e)
    tol = R.logp_tolerance(logp, spread)
    close(r.logp, np.where(on, logp, 0.0), tol, "logp")
    # a reward moves by beta times the errors of its rows' logp and a few units of its size
    move = beta * tol.sum() + 8 * R.EPS * beta * np.abs(np.where(on, logp - ref, 0.0)).sum()
    got = r.stats.double().cpu().numpy()
    assert got[1] == pytest.approx(stats[1], abs=1e-6)
    assert np.all(np.abs(got - stats)[[0, 2, 3, 4]] <= 2 * move + 8 * R.EPS * np.abs(stats[[0, 2, 3, 4]])), (got, stats)
    rows_g = r.row_grads.double().cpu().numpy()
    assert np.all(np.abs(rows_g[0] - g) <= (2 * move + 16 * R.EPS) * beta) and not rows_g[1].any()
    assert not rows_g[0][g == 0].any()
    check_gradient(r.grad_logits, x, t, on, 2.0 * rows_g[0], np.zeros(rows), bf16)
    inplace = losses.preference_loss(logits, targets, torch.from_numpy(offsets).cuda(), torch.from_numpy(ref).cuda(),
                                     beta=beta, label_smoothing=e, grad_scale=2.0, out=logits)
    assert torch.equal(inplace.grad_logits, r.grad_logits) and torch.equal(inplace.stats, r.stats)


@pytest.mark.parametrize("V", [5, 300, 5000, 70000])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_masked_classes(env, V, dtype):
    """-inf and the type's lowest value in most classes; rows of them alone."""
    torch, losses = env
    print(f"[case] masked V={V} {dtype}", flush=True)
    dt = getattr(torch, dtype)
    gen = torch.Generator().manual_seed(V)
    low = float(torch.finfo(dt).min)
    x = (2 * torch.randn(6, V, generator=gen)).to(dt)
    hide = torch.rand(6, V, generator=gen) < 0.8
    hide[:, 1] = False
    x[0:2][hide[0:2]] = -float("inf")
    x[2:4][hide[2:4]] = low
    x[4] = -float("inf")      # nothing is left
    x[5] = low                # all alike
    t = torch.full((6,), 1)
    t[1] = int(hide[1].nonzero()[0]) if hide[1].any() else 0   # a class of probability 0
    logits, targets = x.cuda(), t.cuda()
    r = losses.token_logprobs(logits, targets, entropy=True, save=True)
    xd = x.double().numpy()
    p, logp, ent, spread = R.rows(xd, t.numpy())
    keep = [0, 2, 3, 5]
    tol = R.logp_tolerance(logp, spread)
    close(r.logp[keep], logp[keep], tol[keep], "logp")
    close(r.entropy[[0, 1, 2, 3, 5]], ent[[0, 1, 2, 3, 5]], 2 * tol[[0, 1, 2, 3, 5]], "entropy")
    if hide[1].any():
        assert r.logp[1].item() == -float("inf")
    assert torch.isnan(r.logp[4]) and torch.isnan(r.entropy[4])
    g, h = torch.ones(6, device="cuda"), torch.full((6,), 0.5, device="cuda")
    grad = losses.token_logprobs_backward(logits, targets, r.saved, g, h)
    assert torch.isnan(grad[4]).all()
    one = np.ones(5)
    check_gradient(grad[[0, 1, 2, 3, 5]], xd[[0, 1, 2, 3, 5]], t.numpy()[[0, 1, 2, 3, 5]], one > 0, one, 0.5 * one,
                   dt is torch.bfloat16)
    assert (grad[0].cpu()[hide[0]] == 0).all()
    # the policy loss meets the same rows: what is left of them is finite, an idle empty row is not looked at
    w = torch.ones(6, device="cuda")
    w[4] = 0
    old = torch.where(torch.isfinite(r.logp), r.logp, torch.zeros_like(r.logp))
    q = losses.policy_loss(logits, targets, old, g, weights=w, entropy_coef=0.1)
    assert torch.isfinite(q.stats).all() and torch.isfinite(q.grad_logits).all() and not q.grad_logits[4].any()
    bad = losses.policy_loss(logits, targets, old, g)
    assert torch.isnan(bad.stats[0])


@pytest.mark.parametrize("V,dtype", [(9, "float32"), (1000, "bfloat16"), (33000, "bfloat16"), (90000, "float32")])
def test_not_a_number_and_targets_past_the_classes(env, V, dtype):
    torch, losses = env
    print(f"[case] nan V={V} {dtype}", flush=True)
    dt = getattr(torch, dtype)
    x = torch.randn(5, V, generator=torch.Generator().manual_seed(V)).to(dt).cuda()
    x[1, V - 1] = float("nan")
    x[2, V // 2] = float("inf")
    t = torch.tensor([0, 0, 0, V, 1 << 40], device="cuda")
    r = losses.token_logprobs(x, t, entropy=True, save=True)
    assert torch.isfinite(r.logp[0]) and torch.isnan(r.logp[1:]).all()
    g = torch.ones(5, device="cuda")
    grad = losses.token_logprobs_backward(x, t, r.saved, g)
    assert torch.isfinite(grad[0]).all() and torch.isnan(grad[1:]).all()
    q = losses.policy_loss(x, t, torch.zeros(5, device="cuda"), g)
    assert torch.isnan(q.stats[0]) and torch.isfinite(q.grad_logits[0]).all() and torch.isnan(q.grad_logits[1:]).all()


def test_nothing_to_do(env):
    torch, losses = env
    z = torch.empty(0, 16, device="cuda")
    t = torch.empty(0, dtype=torch.int64, device="cuda")
    f = torch.empty(0, device="cuda")
    r = losses.token_logprobs(z, t, entropy=True, save=True)
    assert r.logp.shape == (0,) and losses.token_logprobs_backward(z, t, r.saved, f).shape == (0, 16)
    q = losses.policy_loss(z, t, f, f)
    assert q.stats.tolist() == [0.0] * 6 and q.grad_logits.shape == (0, 16)
    s = losses.preference_loss(z, t, torch.zeros(5, dtype=torch.int32, device="cuda"), f)
    # two pairs of empty sequences: every margin is 0
    assert s.stats.tolist() == pytest.approx([float(np.log(2)), 0, 0, 0, 0], rel=1e-6)
    s = losses.preference_loss(z, t, torch.zeros(1, dtype=torch.int64, device="cuda"), f)
    assert s.stats.tolist() == [0.0] * 5
    # rows, but none of them takes part
    x = torch.full((4, 33), float("nan"), device="cuda")
    idle = torch.full((4,), -1, device="cuda")
    v = torch.full((4,), float("nan"), device="cuda")
    q = losses.policy_loss(x, idle, v, v, logp_ref=v, weights=v, kl_coef=0.1, entropy_coef=0.1)
    assert q.stats.tolist() == [0.0] * 6 and not q.grad_logits.any() and not q.logp.any()
    one = torch.zeros(4, dtype=torch.int64, device="cuda")
    q = losses.policy_loss(x, one, v, v, weights=torch.zeros(4, device="cuda"))
    assert q.stats.tolist() == [0.0] * 6 and not q.grad_logits.any()


@pytest.mark.parametrize("V", [6, 700])
def test_gradients_against_differences(env, V):
    """The kernels' gradient along a direction against central differences of
    the loss's definition in 64 bits: O(step^2) = 1e-8 and rounding."""
    torch, losses = env
    rows = 7
    rng = np.random.RandomState(V)
    x = (1.5 * rng.randn(rows, V)).astype(np.float32)
    t = rng.randint(0, V, rows)
    t[3] = -1
    on = t >= 0
    tt = np.clip(t, 0, None)
    _, logp, _, _ = R.rows(x.astype(float), tt)
    old, ref, adv, w = policy_inputs(torch, logp, rows, 9)
    offsets = np.array([0, 2, 3, 3, 7])

    def policy(z):
        p, lp, ent, _ = R.rows(z, tt)
        return R.policy(p, lp, ent, on & (w != 0), old.astype(float), ref.astype(float), adv.astype(float), w.astype(float),
                        (0.2, 0.3), 0.1, 0.02, True)[0][0]

    def preference(z):
        _, lp, _, _ = R.rows(z, tt)
        return R.preference(lp, on, offsets, ref.astype(float), 0.5, 0.1)[0][0]

    c = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    pol = losses.policy_loss(c(x), c(t), c(old), c(adv), logp_ref=c(ref), weights=c(w), clip=(0.2, 0.3), kl_coef=0.1,
                             entropy_coef=0.02).grad_logits
    pre = losses.preference_loss(c(x), c(t), c(offsets), c(ref), beta=0.5, label_smoothing=0.1).grad_logits
    for f, grad in ((policy, pol), (preference, pre)):
        grad = grad.double().cpu().numpy()
        for k in range(4):
            u = rng.randn(rows, V)
            step = 1e-4 / np.sqrt(V)
            diff = (f(x + step * u) - f(x - step * u)) / (2 * step)
            assert diff == pytest.approx((grad * u).sum(), rel=1e-4, abs=2e-5)


def test_autograd(env):
    torch, losses = env
    rng = np.random.RandomState(0)
    rows, V = 12, 50
    base = torch.from_numpy(rng.randn(rows, 64).astype(np.float32)).cuda()
    t = torch.from_numpy(rng.randint(0, V, rows)).cuda()
    t[4] = -1
    old = torch.full((rows,), -4.0, device="cuda")
    adv = torch.from_numpy(rng.randn(rows).astype(np.float32)).cuda()
    full = base.clone().requires_grad_(True)
    loss, stats, logp = losses.policy_loss_autograd(full[:, :V], t, old, adv, logp_ref=old, kl_coef=0.1, entropy_coef=0.01)
    (3.0 * loss).backward()
    r = losses.policy_loss(base[:, :V], t, old, adv, logp_ref=old, kl_coef=0.1, entropy_coef=0.01)
    assert torch.allclose(full.grad[:, :V], 3.0 * r.grad_logits, rtol=1e-5, atol=1e-9) and not full.grad[:, V:].any()
    assert loss.item() == pytest.approx(r.stats[0].item(), rel=1e-5) and not stats.requires_grad and not logp.requires_grad
    offsets = torch.tensor([0, 3, 6, 9, 12], device="cuda")
    leaf = base.clone().requires_grad_(True)
    loss, _, _ = losses.preference_loss_autograd(leaf, t, offsets, old, beta=0.2)
    loss.backward()
    s = losses.preference_loss(base, t, offsets, old, beta=0.2)
    assert torch.allclose(leaf.grad, s.grad_logits, rtol=1e-5, atol=1e-9)
    # broadcast upstream gradients, one output unused
    leaf = base.clone().requires_grad_(True)
    logp, entropy = losses.token_logprobs_autograd(leaf, t)
    logp.sum().backward()
    u = losses.token_logprobs(base, t, save=True)
    want = losses.token_logprobs_backward(base, t, u.saved, torch.ones(rows, device="cuda"))
    assert torch.equal(leaf.grad, want)
    assert entropy.shape == (rows,)


def test_other_streams_and_workspaces(env):
    """Calls on another stream, into a workspace full of NaN, alternating shapes."""
    torch, losses = env
    got = {}
    side = torch.cuda.Stream()
    ws = torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
    for k, shape in enumerate([(37, 1000, 1024, "float32", 64), (4, 70001, 70001, "bfloat16", 64), (3, 7, 7, "float32", 32)] * 2):
        logits, targets, _, t, _ = make(torch, shape, 4)
        rows = len(t)
        ref, off = torch.full((rows,), -3.0, device="cuda"), torch.tensor([0, rows // 2, rows], device="cuda")
        adv = torch.ones(rows, device="cuda")
        assert losses.workspace_bytes(logits, 1) <= ws.numel()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            a = losses.policy_loss(logits, targets, ref, adv, workspace=ws)
            b = losses.preference_loss(logits, targets, off, ref, workspace=ws)
            c = losses.token_logprobs(logits, targets, workspace=ws)
        side.synchronize()
        now = [a.stats, a.grad_logits, b.stats, b.grad_logits, c.logp]
        for x, y in zip(now, got.setdefault(shape, now)):
            assert torch.equal(x, y)


def test_rows_past_32_bit_offsets(env):
    """The last rows of logits that hold more than 2^31 values."""
    torch, losses = env
    rows, V = 32770, 65600
    print(f"[case] {rows} x {V} bfloat16", flush=True)
    full = torch.empty(rows, V, dtype=torch.bfloat16, device="cuda")
    x = (2 * torch.randn(3, V, generator=torch.Generator().manual_seed(1))).to(torch.bfloat16)
    full[-3:] = x.cuda()
    t = torch.full((rows,), -1, device="cuda")
    t[-3:] = torch.tensor([5, V - 1, 40000], device="cuda")
    tail = t[-3:].cpu().numpy()
    p, logp, ent, spread = R.rows(x.double().numpy(), tail)
    old, adv = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    old[-3:] = torch.from_numpy(logp).float().cuda() - 0.01
    r = losses.policy_loss(full, t, old, adv, out=full, save=True)
    close(r.logp[-3:], logp, R.logp_tolerance(logp, spread), "logp")
    got = r.row_grads.double().cpu().numpy()[:, -3:]
    check_gradient(full[-3:], x.double().numpy(), tail, np.ones(3, bool), got[0], got[1], True)
    assert not full[-4].any() and not full[0].any()


def test_wrong_arguments_on_the_gpu(env):
    """What the native part of the binding does not take is refused as on the CPU."""
    torch, losses = env
    x, t, f = torch.zeros(4, 10, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    saved, off = torch.zeros(4, 4, device="cuda"), torch.tensor([0, 2, 4], device="cuda")
    for call in (lambda: losses.token_logprobs(x.double(), t), lambda: losses.token_logprobs(x, t[:3]),
                 lambda: losses.token_logprobs(x, t.float()), lambda: losses.token_logprobs(x, t.cpu()),
                 lambda: losses.token_logprobs(torch.zeros(10, 4, device="cuda").t(), t),
                 lambda: losses.token_logprobs(x, t, workspace=torch.zeros(1, dtype=torch.uint8, device="cuda")),
                 lambda: losses.token_logprobs_backward(x, t, saved[:3], f),
                 lambda: losses.token_logprobs_backward(x, t, saved, f[:1].expand(4)),
                 lambda: losses.token_logprobs_backward(x, t, saved, f, out=x.bfloat16()),
                 lambda: losses.policy_loss(x, t, f, f.cpu()), lambda: losses.policy_loss(x, t, f, f, kl_coef=0.1),
                 lambda: losses.policy_loss(x, t, f, f, clip=(-1, 0.2)), lambda: losses.policy_loss(x, t, f, f.double()),
                 lambda: losses.preference_loss(x, t, off[:2], f), lambda: losses.preference_loss(x, t, off.float(), f),
                 lambda: losses.preference_loss(x, t, off, f, label_smoothing=2.0)):
        with pytest.raises(ValueError):
            call()
    from paper_1511_05946_amd.acdc import ACDCError
    with pytest.raises(ACDCError, match="invalid argument"):   # memory that overlaps the logits': seen by the library
        wide = torch.zeros(64, device="cuda")
        losses.token_logprobs_backward(wide[:40].view(4, 10), t, saved, f, out=wide[2:42].view(4, 10))
    with pytest.raises(ValueError):
        losses.token_logprobs(x.cpu(), t.cpu())


def test_more_rows_than_a_grid_has_workgroups(env):
    """Over 2^22 rows: the streaming kernels take several each."""
    torch, losses = env
    rows, V = (1 << 22) + 1000, 8
    print(f"[case] {rows} x {V}", flush=True)
    x = 2 * torch.randn(rows, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    t = torch.arange(rows, device="cuda") % V
    t[::7] = -1
    r = losses.token_logprobs(x, t, entropy=True, save=True)
    g = torch.ones(rows, device="cuda")
    grad = losses.token_logprobs_backward(x, t, r.saved, g)
    pick = torch.cat([torch.arange(2000), torch.arange(rows - 3000, rows)])
    xs, ts = x.cpu()[pick].double().numpy(), t.cpu()[pick].numpy()
    on = ts >= 0
    p, logp, ent, spread = R.rows(xs, np.clip(ts, 0, None))
    close(r.logp[pick.cuda()], np.where(on, logp, 0.0), R.logp_tolerance(logp, spread), "logp")
    check_gradient(grad[pick.cuda()], xs, ts, on, np.ones(len(ts)), np.zeros(len(ts)), False)
    q = losses.policy_loss(x, t, r.logp, g, grad=False)
    # every ratio is 1 and every advantage 1
    assert q.stats[:2].tolist() == pytest.approx([-1.0, -1.0], rel=1e-6) and q.stats[5].item() == pytest.approx(1.0, rel=1e-6)


# around the chunks that 16 lanes, a wave and a workgroup take a row at, a chunk being 16 bytes;
# rows that fill no whole workgroup, on and off their chunks' alignment
WIDTHS = [(dtype, per * chunks + more) for dtype, per in (("float32", 4), ("bfloat16", 8))
          for chunks, more in ((0, 2), (16, 1), (48, 0), (63, 1), (64, 0), (65, 0), (192, 3), (256, 1), (512, 0), (513, 0))]


@pytest.mark.parametrize("dtype,classes", WIDTHS)
@pytest.mark.parametrize("apart", [0, 3])
def test_rows_that_share_a_workgroup(env, dtype, classes, apart):
    for rows in (1, 3, 18, 133):
        shape = rows, classes, classes + apart, dtype, 64
        test_token_logprobs_and_gradient(env, shape)
        if rows > 3:
            test_preference_loss(env, shape)


def test_more_short_rows_than_a_grid_has_lanes_for(env):
    """Over 2^26 rows, 16 to a workgroup: each workgroup takes several lots."""
    torch, losses = env
    rows, V = (1 << 26) + 1000, 2
    print(f"[case] {rows} x {V}", flush=True)
    x = torch.randn(rows, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    t = torch.arange(rows, device="cuda", dtype=torch.int32) % V
    t[::7] = -1
    r = losses.token_logprobs(x, t, entropy=True, save=True)
    g = torch.ones(rows, device="cuda")
    grad = losses.token_logprobs_backward(x, t, r.saved, g)
    pick = torch.cat([torch.arange(2000), torch.arange(rows - 3000, rows)]).cuda()
    xs, ts = x[pick].double().cpu().numpy(), t[pick].cpu().numpy()
    on = ts >= 0
    p, logp, ent, spread = R.rows(xs, np.clip(ts, 0, None))
    close(r.logp[pick], np.where(on, logp, 0.0), R.logp_tolerance(logp, spread), "logp")
    check_gradient(grad[pick], xs, ts, on, np.ones(len(ts)), np.zeros(len(ts)), False)
