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
