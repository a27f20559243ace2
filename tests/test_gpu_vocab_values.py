"""Logits of every size in the losses over a vocabulary, in calls of few tiles and of many,
of one piece of the vocabulary and of several, on the GPU, against the definitions in 64 bits."""

import numpy as np
import pytest

import lm_reference as R
from test_gpu_vocab import check_gradients, close, env, make  # noqa: F401 (env: a fixture)

pytestmark = pytest.mark.gpu

# few tiles; small tiles that keep their exponentials or not (few rows); large tiles; more than
# one piece of the vocabulary
SIZES = [(90, 40, 100), (100, 30, 1500), (8, 40, 5000), (300, 16, 8300), (1100, 512, 16500)]
CASES = [(*s, dtype) for s in SIZES for dtype in ("float32", "bfloat16")] + [(16384, 8, 14000, "float32")]
# small tiles of logits and large ones of gradients, of 8 bits of dL/dlogits and of 16
CASES += [(1100, 8200, 1030, "bfloat16"), (40, 33000, 100, "bfloat16")]


def switched_off(torch, case, seed):
    """A column of ones beside hidden, and beside the weight one that is 0, or the type's
    lowest value for each third class: hidden, weight, targets among the others, those classes."""
    rows, width, classes, dtype = case
    h, w, t, h64, w64, t64, share = make(torch, (rows, width, classes, dtype, 64, 0, 0), seed=seed, idle=0.97 if rows > 10000 else 0.25)
    off = torch.arange(classes, device="cuda") % 3 == 1
    t64 = np.where(t64 < 0, t64, t64 - (t64 % 3 == 1))
    column = torch.where(off, torch.finfo(w.dtype).min, 0.0).to(w.dtype)
    h = torch.cat((h, torch.ones(rows, 1, dtype=h.dtype, device="cuda")), 1)
    w = torch.cat((w, column[:, None]), 1)
    h64 = np.concatenate((h64, np.ones((rows, 1))), 1)
    w64 = np.concatenate((w64, np.zeros((classes, 1))), 1)
    return h, w, torch.from_numpy(t64).cuda(), h64, w64, t64, off


@pytest.mark.parametrize("case", CASES)
def test_classes_switched_off(env, case):  # noqa: F811
    """Classes whose logit is the type's lowest value: as if they were not there."""
    torch, losses = env
    h, w, t, h64, w64, t64, off = switched_off(torch, case, 11)
    on, rows = (~off).cpu().numpy(), t64 >= 0
    # the definition over the other classes, and their numbers among themselves
    number = np.cumsum(on) - 1
    ref = R.Vocab(h64[rows], w64[on], number[t64[rows]])
    there = torch.from_numpy(rows).cuda()

    def check(logp, gh, gw):
        close(logp[there], ref.logp, ref.logp_tol, "logp")
        check_gradients(ref, -ref.share, gh[there], gw[~off], case[3] == "bfloat16")
        assert (gw[off] == 0).all() and (gh[~there] == 0).all()

    r = losses.vocab_loss(h, w, t, save=True)
    assert abs(r.stats[0].item() - ref.loss) <= ref.loss_tol
    check(r.logp, r.grad_hidden, r.grad_weight)
    s = losses.vocab_logprobs(h, w, t, save=True)
    close(s.logp[there], ref.logp, ref.logp_tol, "logp")
    check(s.logp, *losses.vocab_logprobs_backward(h, w, t, s.saved, r.row_grads))
    # one of them as a target: its log-probability is as low, and no row is NaN
    t[torch.nonzero(there)[0]] = 1
    r = losses.vocab_loss(h, w, t)
    assert r.logp.min().item() <= torch.finfo(h.dtype).min and not torch.isnan(r.logp).any()
    assert torch.isfinite(r.grad_weight[~off]).all()


@pytest.mark.parametrize("case", CASES)
def test_what_is_not_a_number(env, case):  # noqa: F811
    """A target past the classes and hidden values that are not finite: NaN for their own
    row and the weight's gradient, and no other row."""
    torch, losses = env
    rows, width, classes, dtype = case
    h, w, t, h64, w64, t64, _ = make(torch, (rows, width, classes, dtype, 64, 0, 0), seed=12, idle=0.97 if rows > 10000 else 0.25)
    t64 = np.where(np.arange(rows) < 3, 7, t64)
    t = torch.from_numpy(t64).cuda()
    t[0], h[1, 3], h[2, 0] = classes, float("inf"), float("nan")
    h[1, :3] = 1.0
    on = t64 >= 0
    on[:3] = False
    ref = R.Vocab(h64[on], w64, t64[on])
    there, idle = torch.from_numpy(on).cuda(), torch.from_numpy(t64 < 0).cuda()
    r = losses.vocab_loss(h, w, t, mean=False, save=True)
    s = losses.vocab_logprobs(h, w, t, save=True)
    again = losses.vocab_logprobs_backward(h, w, t, s.saved, r.row_grads.nan_to_num(-1.0))
    assert torch.isnan(r.stats[0])
    for logp, gh, gw in ((r.logp, r.grad_hidden, r.grad_weight), (s.logp, *again)):
        close(logp[there], ref.logp, ref.logp_tol, "logp")
        assert torch.isnan(logp[:3]).all() and torch.isnan(gh[:3]).all() and torch.isnan(gw).all()
        assert torch.isfinite(gh[there]).all() and (gh[idle] == 0).all() and (logp[idle] == 0).all()


@pytest.mark.parametrize("case", CASES)
def test_far_logits(env, case):  # noqa: F811
    """Rows whose softmax is one class: logits up to thousands apart."""
    torch, losses = env
    rows, width, classes, dtype = case
    h, w, t, h64, w64, t64, _ = make(torch, (rows, width, classes, dtype, 64, 0, 0), seed=13, idle=0.97 if rows > 10000 else 0.25)
    on = t64 >= 0
    w = (w.float() * 1000.0).to(w.dtype)
    ref = R.Vocab(h64[on], w.double().cpu().numpy(), t64[on])
    there = torch.from_numpy(on).cuda()
    r = losses.vocab_loss(h, w, t, save=True)
    close(r.logp[there], ref.logp, ref.logp_tol, "logp")
    again = losses.vocab_logprobs_backward(h, w, t, r.saved, r.row_grads)
    for g in (r.grad_hidden, r.grad_weight, *again):
        assert torch.isfinite(g).all()


@pytest.mark.parametrize("case", CASES)
def test_likely_targets(env, case):  # noqa: F811
    """Targets of a probability near 1, whose 1 - p has few digits left: of the loss, which may take it
    from kept exponentials, and of the backward call, which computes the logits again."""
    torch, losses = env
    rows, width, classes, dtype = case
    h, w, t, h64, w64, t64, _ = make(torch, (rows, width, classes, dtype, 64, 0, 0), seed=17, idle=0.97 if rows > 10000 else 0.25)
    on = t64 >= 0
    w = (w.float() * 6.0).to(w.dtype)
    w64 = w.double().cpu().numpy()
    t64 = np.where(on, (np.where(on[:, None], h64, 0.0) @ w64.T).argmax(1), t64)
    t.copy_(torch.from_numpy(t64))
    ref = R.Vocab(h64[on], w64, t64[on])
    there = torch.from_numpy(on).cuda()
    r = losses.vocab_loss(h, w, t, save=True)
    close(r.logp[there], ref.logp, ref.logp_tol, "logp")
    check_gradients(ref, -ref.share, r.grad_hidden[there], r.grad_weight, dtype == "bfloat16")
    gh, gw = losses.vocab_logprobs_backward(h, w, t, r.saved, r.row_grads)
    check_gradients(ref, -ref.share, gh[there], gw, dtype == "bfloat16")


# sums of few terms, in products of large tiles: few rows for the weight's gradient, few classes for hidden's
# (the last one: two pieces of the vocabulary)
@pytest.mark.parametrize("case", [(1, 4096, 8192), (8, 1024, 33000), (64, 1024, 8192), (200, 520, 16500), (1000, 520, 16500),
                                  (20000, 512, 700), (1000, 8, 300000)])
def test_few_terms_of_bfloat16(env, case):  # noqa: F811
    """Gradients of bfloat16 inputs whose sums have few terms: dL/dlogits keeps 16 bits, and only the
    rounding of the gradient itself is seen."""
    torch, losses = env
    h, w, t, h64, w64, t64, share = make(torch, (*case, "bfloat16", 64, 0, 0), seed=14, idle=0.985 if case[2] > 100000 else 0.25)
    on = t64 >= 0
    there = torch.from_numpy(on).cuda()
    ref = R.Vocab(h64[on], w64, t64[on], share.double().numpy()[on])
    rows = np.arange(on.sum())

    def check(g, gh, gw):
        G = -g[:, None] * ref.p
        G[rows, t64[on]] += g
        # two roundings to 8 bits one of what the other leaves: 2^-16 of every value
        for got, (want, tol), left, right in ((gh[there], ref.gradients(g, False, True, True)[0], G, w64),
                                              (gw, ref.gradients(g, False, True, True)[1], G.T, h64[on])):
            close(got, want, tol + R.BF16 ** 2 * (np.abs(left) @ np.abs(right)), "gradient")

    r = losses.vocab_loss(h, w, t, weights=share.cuda(), save=True)
    check(-ref.share, r.grad_hidden, r.grad_weight)
    g = torch.randn(case[0], generator=torch.Generator().manual_seed(3))
    check(g.double().numpy()[on], *losses.vocab_logprobs_backward(h, w, t, r.saved, g.cuda()))
    # the weight's gradient in float32: no rounding but that one
    full = torch.zeros(w.shape, device="cuda")
    losses.vocab_loss(h, w, t, weights=share.cuda(), grad_weight=full)
    want, tol = ref.gradients(-ref.share, False, False, False)[1]
    G = ref.share[:, None] * ref.p
    G[rows, t64[on]] -= ref.share
    close(full, want, tol + R.BF16 ** 2 * (np.abs(G).T @ np.abs(h64[on])), "float32 gradient")


# products of 8 bits of dL/dlogits, of 16 in large and in small tiles, of few tiles, and float32
@pytest.mark.parametrize("case", [(5500, 256, 16640, "bfloat16"), (300, 512, 16640, "bfloat16"), (300, 16, 8300, "bfloat16"),
                                  (90, 40, 100, "bfloat16"), (50, 40, 100, "bfloat16"), (300, 16, 8300, "float32")])
def test_factor_of_all_rows(env, case):  # noqa: F811
    """dL/dlogp of -1 / W in every row is -1 under a scale of 1 / W, bit for bit: the factor is not
    rounded with each target's value, where it would be off the same way in all of them."""
    torch, losses = env
    rows, width, classes, dtype = case
    h, w, t, h64, w64, t64, share = make(torch, (*case, 64, 0, 0), seed=15)
    s = losses.vocab_logprobs(h, w, t, save=True)
    inverse = torch.tensor([1.0 / rows], device="cuda")
    ones = torch.full((rows,), -1.0, device="cuda")
    want = losses.vocab_logprobs_backward(h, w, t, s.saved, ones, scale=inverse)
    got = losses.vocab_logprobs_backward(h, w, t, s.saved, ones * inverse)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # the same with rows of both signs and sizes, an infinite one among them
    g = torch.randn(rows, generator=torch.Generator().manual_seed(4)).cuda()
    g[0], t[0] = float("inf"), 0
    gh, gw = losses.vocab_logprobs_backward(h, w, t, s.saved, g)
    assert not torch.isfinite(gh[0]).any() and torch.isfinite(gh[1:]).all() and not torch.isfinite(gw[0]).any()


def test_many_rows_of_one_class(env):  # noqa: F811
    """The gradient of a class that thousands of rows have as their target, of rows alike: errors of
    the same sign add up."""
    torch, losses = env
    rows, width, classes = 5500, 256, 16640
    h, w, t, h64, w64, t64, _ = make(torch, (rows, width, classes, "bfloat16", 64, 0, 0), seed=16, idle=0.0)
    h[:] = (torch.ones(width, device="cuda") + 0.1 * torch.randn(rows, width, device="cuda", generator=torch.Generator("cuda").manual_seed(6))).to(h.dtype)
    t[:] = 3
    h64, t64 = h.double().cpu().numpy(), t.cpu().numpy()
    ref = R.Vocab(h64, w64, t64)
    want, tol = ref.gradients(-ref.share, True, True, False)[1]
    # rows alike have a p alike: 1 - p, of class 3 in every row, is rounded the same way in all of
    # them, so that these roundings are not of mean 0, as the tolerance has it, and their sizes
    # add up.  (p is 0.001 to 0.004 or so; in [1/2, 1] bfloat16 values are 2^-8 apart.)
    q = 1 - ref.p[:, 3]
    tol[3] += (ref.share * np.abs(np.round(q * 256) / 256 - q)) @ np.abs(h64)
    r = losses.vocab_loss(h, w, t, save=True, grad_weight=torch.zeros(classes, width, device="cuda"))
    close(r.grad_weight, want, tol, "vocab_loss")
    full = torch.zeros(classes, width, device="cuda")
    losses.vocab_logprobs_backward(h, w, t, r.saved, r.row_grads, grad_weight=full)
    close(full, want, tol, "vocab_logprobs_backward")
    # the differentiable form
    b = w.clone().requires_grad_(True)
    losses.vocab_loss_autograd(h, b, t)[0].backward()
    close(b.grad, want, tol + R.out_rounding(want, True), "vocab_loss_autograd")
