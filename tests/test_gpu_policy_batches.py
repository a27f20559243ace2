"""The policy loss's one pass over large batches, against its definition in 64
bits: every lane's class as the target, workgroups that take several lots of
rows, weights summed by a launch of their own."""

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


@pytest.mark.parametrize("dtype,V,apart", [("float32", 300, 0), ("float32", 700, 1), ("float32", 1024, 0), ("bfloat16", 600, 3),
                                           ("bfloat16", 1500, 0), ("bfloat16", 2048, 1)])
@pytest.mark.parametrize("rows", [16, 0])
def test_targets_of_every_lane(env, dtype, V, apart, rows):
    """A row's target is loaded by one lane and read by all: every class once, in one
    workgroup (rows at a time) and in many."""
    torch, losses = env
    print(f"[case] every target, {V} {dtype} + {apart}, {rows} rows a call", flush=True)
    x = torch.randn(V, V + apart, generator=torch.Generator().manual_seed(V)).to(getattr(torch, dtype)).cuda()[:, :V]
    t = torch.arange(V, device="cuda")
    old, adv = torch.full((V,), -6.0, device="cuda"), torch.linspace(-1, 1, V, device="cuda")
    p, logp, ent, spread = R.rows(x.double().cpu().numpy(), np.arange(V))
    for k in range(0, V, rows or V):
        at = slice(k, min(V, k + (rows or V)))
        r = losses.policy_loss(x[at], t[at], old[at], adv[at], save=True)
        got = r.logp.double().cpu().numpy()
        assert np.all(np.abs(got - logp[at]) <= R.logp_tolerance(logp, spread)[at]), k
        g, h = r.row_grads.double().cpu().numpy()
        want = R.gradient(p[at], ent[at], np.arange(V)[at], g, h)
        tol = R.gradient_tolerance(p[at], want, ent[at], spread[at], np.arange(V)[at], g, h, dtype == "bfloat16")
        assert np.all(np.abs(r.grad_logits.double().cpu().numpy() - want) <= tol), k


def definition(torch, x, t, old, ref, adv, w, clip, kl_coef, entropy_coef):
    """(stats, g, h, gradient) of the mean loss in 64 bits on the GPU, and how far 32 bits may be from each."""
    on = (t >= 0) & (w != 0)
    x, old, ref, adv, w = (v.double() for v in (x, old, ref, adv, w))
    tt = t.clamp(min=0).unsqueeze(1)
    d = x - x.amax(1, keepdim=True)
    e = d.exp()
    s = e.sum(1, keepdim=True)
    p = e / s
    logp = (d.gather(1, tt) - s.log()).squeeze(1)
    ent = (s.log() - (p * d).sum(1, keepdim=True)).squeeze(1)
    spread = torch.where(e > 1e-12, -d, 0.0).amax(1)
    w = torch.where(on, w, 0.0)
    w = w / w.sum()
    ratio, k = (logp - old).exp(), ref - logp
    free, bound = ratio * adv, ratio.clamp(1 - clip[0], 1 + clip[1]) * adv
    cut = bound < free
    pol, kl = -torch.minimum(free, bound), k.expm1() - k
    values = [pol + kl_coef * kl - entropy_coef * ent, pol, kl, ent, cut.double(), ratio]
    stats = torch.stack([(w * v).sum() for v in values])
    g, h = w * (torch.where(cut, 0.0, -free) - kl_coef * k.expm1()), -entropy_coef * w
    grad = -p * (g.unsqueeze(1) + h.unsqueeze(1) * (d - s.log() + ent.unsqueeze(1)))
    grad.scatter_add_(1, tt, g.unsqueeze(1))
    # a row's values move by its logp's error times their slopes, and some units
    lp_tol = R.EPS * (32 + 4 * spread + 2 * logp.abs())
    move = (2 * lp_tol + 8 * R.EPS) * (adv.abs() * ratio + ratio + 2 * k.expm1().abs() + ent.abs() + 2)
    # sums: 9 roundings of a weight over the weights' sum, 4 of a value, 7 over a wave and a workgroup, 10 over all
    stats_tol = (w * move).sum() + 40 * R.EPS * torch.stack([(w * v).abs().sum() for v in values])
    g_tol = w * move + 16 * R.EPS * g.abs()
    return stats, g, h, grad, p, spread, ent, stats_tol, g_tol


# several rows for a workgroup: 16 lanes a row, a wave with two rows and with one, a wave and four
# rows a workgroup, a workgroup a row, and rows longer than its registers, in both types
@pytest.mark.parametrize("rows,V,dtype", [(270000, 9, "float32"), (263000, 129, "bfloat16"), (140000, 301, "float32"),
                                          (70000, 601, "float32"), (33500, 1100, "float32"), (9000, 4097, "float32"),
                                          (8300, 66001, "bfloat16"), (8200, 66002, "float32")])
def test_large_batches(env, rows, V, dtype):
    torch, losses = env
    print(f"[case] policy {rows} x {V} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    make = lambda: torch.randn(rows, device="cuda", generator=gen)  # noqa: E731
    x = torch.empty(rows, V, dtype=getattr(torch, dtype), device="cuda").normal_(generator=gen).mul_(2)
    t = torch.randint(0, V, (rows,), device="cuda", generator=gen)
    logp = losses.token_logprobs(x, t).logp
    shift = (0.3 * make()).clamp(-1, 1)
    clip = (0.2, 0.3)
    for b in (np.log(1 - clip[0]), np.log(1 + clip[1])):   # off the clip bounds, where rounding would decide
        shift = torch.where((shift - b).abs() < 1e-3, shift + 3e-3, shift)
    old, ref, adv = logp - shift, logp + 0.2 * make(), make()
    w = torch.rand(rows, device="cuda", generator=gen) * 3 + 0.1
    w[::50] = 0
    t[torch.rand(rows, device="cuda", generator=gen) < 0.15] = -3
    kw = dict(logp_ref=ref, weights=w, clip=clip, kl_coef=0.1, entropy_coef=0.02)
    r = losses.policy_loss(x, t, old, adv, save=True, grad_scale=0.5, **kw)
    stats, g, h, grad, p, spread, ent, stats_tol, g_tol = definition(torch, x, t, old, ref, adv, w, clip, 0.1, 0.02)
    assert torch.all((r.stats.double() - stats).abs() <= stats_tol), (r.stats.tolist(), stats.tolist(), stats_tol.tolist())
    got = r.row_grads.double()
    assert torch.all((got[0] - g).abs() <= g_tol) and torch.all((got[1] - h).abs() <= 16 * R.EPS * h.abs())
    # the logits' gradient carries the row gradients' errors and its own
    size = g.abs() + h.abs() * (spread + ent.abs() + 1)
    tol = R.EPS * (32 + 4 * spread).unsqueeze(1) * p * size.unsqueeze(1) + g_tol.unsqueeze(1) * p + \
        16 * R.EPS * (h.abs() * (spread + ent.abs() + 1)).unsqueeze(1) * p
    tol.scatter_add_(1, t.clamp(min=0).unsqueeze(1), (4 * R.EPS * g.abs() + g_tol).unsqueeze(1))
    tol += (R.BF16 * grad.abs() if dtype == "bfloat16" else 0.0) + 1e-38
    bad = (2 * r.grad_logits.double() - grad).abs() > tol
    assert not bad.any(), bad.nonzero()[:3].tolist()
    again = losses.policy_loss(x, t, old, adv, save=True, grad_scale=0.5, **kw)
    assert all(torch.equal(a, b) for a, b in zip(again, r))
    # the values alone, by the passes that the rows' statistics stand between
    values = losses.policy_loss(x, t, old, adv, grad=False, **kw)
    assert torch.all((values.stats.double() - stats).abs() <= stats_tol)
