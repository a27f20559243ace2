"""Losses over a vocabulary without its logits, on the GPU, against their
definitions in 64 bits."""

import struct

import numpy as np
import pytest

import lm_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1511_05946_amd import losses
    return torch, losses


# rows, width, classes, type, bits of the targets, distance of hidden's and of the weight's rows beyond the width:
# one of each, sizes around a step of 64 k and a tile of 64 or 256, odd ones, more than one tile of each
SHAPES = [(1, 1, 1, "float32", 64, 0, 0), (1, 1, 1, "bfloat16", 32, 0, 0), (2, 3, 5, "bfloat16", 64, 1, 2),
          (3, 8, 7, "bfloat16", 32, 0, 0), (64, 64, 64, "bfloat16", 64, 0, 0), (65, 65, 65, "bfloat16", 64, 0, 0),
          (63, 63, 257, "float32", 32, 3, 5), (64, 256, 1000, "float32", 64, 0, 0), (256, 128, 256, "bfloat16", 64, 8, 8),
          (257, 72, 513, "bfloat16", 64, 8, 16), (300, 200, 777, "float32", 64, 0, 1), (70, 264, 2049, "bfloat16", 64, 4, 8),
          (130, 520, 300, "bfloat16", 64, 0, 0), (1000, 96, 1500, "bfloat16", 32, 0, 0), (5, 1000, 4100, "float32", 64, 0, 0),
          (20, 4096, 130, "bfloat16", 64, 0, 0), (520, 31, 90, "float32", 64, 1, 0), (8, 136, 33000, "bfloat16", 64, 0, 0),
          (2100, 40, 50, "bfloat16", 64, 0, 0), (40, 1, 300, "float32", 64, 0, 0),
          # few tiles of many steps
          (3, 8128, 10, "float32", 64, 0, 0), (70, 5000, 100, "bfloat16", 64, 0, 8), (300, 2500, 70, "float32", 32, 1, 0),
          (2, 20000, 3, "bfloat16", 64, 0, 0), (5, 8192, 4000, "bfloat16", 64, 0, 0)]


def values(torch, gen, rows, width, extra, dtype, std):
    full = (std * torch.randn(rows, width + extra, generator=gen)).to(getattr(torch, dtype))
    return full


def make(torch, shape, seed=0, idle=0.25):
    """hidden (NaN in idle rows), weight and targets on the GPU, and in 64 bits."""
    rows, width, classes, dtype, bits, more_h, more_w = shape
    print(f"[case] {shape} seed={seed}", flush=True)
    gen = torch.Generator().manual_seed(31 * seed + rows + width + classes)
    h = values(torch, gen, rows, width, more_h, dtype, 1.0)
    w = values(torch, gen, classes, width, more_w, dtype, 2.0 / width ** 0.5)
    t = torch.randint(0, classes, (rows,), generator=gen)
    off = torch.rand(rows, generator=gen) < idle
    off[0] = False
    t[off] = -1 - torch.randint(0, 100, (int(off.sum()),), generator=gen)
    h64, w64 = h[:, :width].double().numpy().copy(), w[:, :width].double().numpy()
    h[off] = float("nan")
    return (h.cuda()[:, :width], w.cuda()[:, :width], t.to(getattr(torch, f"int{bits}")).cuda(), h64, w64, t.numpy(),
            torch.rand(rows, generator=gen) + 0.5)


def close(got, ref, tol, what):
    got = got.double().cpu().numpy()
    assert got.shape == ref.shape
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3], got[bad][:3], ref[bad][:3],
                           np.broadcast_to(tol, ref.shape)[bad][:3])


def check_gradients(ref, g, gh, gw, bf16):
    (rh, th), (rw, tw) = ref.gradients(g, bf16, gh.element_size() == 2, gw.element_size() == 2)
    close(gh, rh, th, "grad_hidden")
    close(gw, rw, tw, "grad_weight")


@pytest.mark.parametrize("shape", SHAPES)
def test_loss_and_gradients(env, shape):
    torch, losses = env
    h, w, t, h64, w64, t64, share = make(torch, shape)
    bf16 = h.dtype is torch.bfloat16
    for weights in (None, share):
        ref = R.Vocab(h64, w64, t64, None if weights is None else weights.double().numpy())
        r = losses.vocab_loss(h, w, t, weights=None if weights is None else weights.cuda(), save=True)
        close(r.logp, ref.logp, ref.logp_tol, "logp")
        assert abs(r.stats[0].item() - ref.loss) <= ref.loss_tol
        assert abs(r.stats[1].item() - ref.total) <= 2 * R.EPS * ref.total
        close(r.row_grads, -ref.share, 2 * R.EPS * ref.share, "row_grads")
        check_gradients(ref, -ref.share, r.grad_hidden, r.grad_weight, bf16)
        # idle rows: exact zeros; the same call again: bit for bit
        off = torch.from_numpy(~ref.on).cuda()
        assert (r.grad_hidden[off] == 0).all() and (r.logp[off] == 0).all()
        again = losses.vocab_loss(h, w, t, weights=None if weights is None else weights.cuda())
        assert torch.equal(again.grad_hidden, r.grad_hidden) and torch.equal(again.grad_weight, r.grad_weight)
        assert torch.equal(again.stats, r.stats)


@pytest.mark.parametrize("shape", SHAPES[::2])
def test_logprobs_and_gradients(env, shape):
    torch, losses = env
    h, w, t, h64, w64, t64, _ = make(torch, shape, seed=1)
    ref = R.Vocab(h64, w64, t64)
    r = losses.vocab_logprobs(h, w, t, save=True)
    close(r.logp, ref.logp, ref.logp_tol, "logp")
    assert torch.equal(losses.vocab_logprobs(h, w, t).logp, r.logp)
    g = torch.randn(len(t64), generator=torch.Generator().manual_seed(5))
    if len(g) > 2:
        g[1] = 0.0
    scale = torch.tensor([0.375], device="cuda")
    gh, gw = losses.vocab_logprobs_backward(h, w, t, r.saved, g.cuda(), scale=scale)
    check_gradients(ref, 0.375 * g.double().numpy(), gh, gw, h.dtype is torch.bfloat16)
    # one of the two alone, and into given tensors: the same
    one, none = losses.vocab_logprobs_backward(h, w, t, r.saved, g.cuda(), scale=scale, grad="hidden")
    assert none is None and torch.equal(one, gh)
    none, one = losses.vocab_logprobs_backward(h, w, t, r.saved, g.cuda(), scale=scale, grad="weight")
    assert none is None and torch.equal(one, gw)
    wide = torch.full((h.shape[0], h.shape[1] + 5), 3.0, dtype=h.dtype, device="cuda")
    tall = torch.full((w.shape[0], w.shape[1] + 3), 5.0, dtype=w.dtype, device="cuda")
    losses.vocab_logprobs_backward(h, w, t, r.saved, g.cuda(), scale=scale, out=wide[:, 2:-3], grad_weight=tall[:, 1:-2])
    assert torch.equal(wide[:, 2:-3], gh) and torch.equal(tall[:, 1:-2], gw)
    assert (wide[:, :2] == 3).all() and (wide[:, -3:] == 3).all() and (tall[:, :1] == 5).all() and (tall[:, -2:] == 5).all()


@pytest.mark.parametrize("dtype,given", [("bfloat16", "float32"), ("bfloat16", "bfloat16"), ("float32", "float32")])
def test_weight_gradient_is_added(env, dtype, given):
    torch, losses = env
    h, w, t, h64, w64, t64, _ = make(torch, (200, 100, 300, dtype, 64, 0, 0), seed=2)
    start = torch.randn(300, 100, generator=torch.Generator().manual_seed(8)).to(getattr(torch, given)).cuda()
    total = start.clone()
    r = losses.vocab_loss(h, w, t, grad_weight=total, accumulate=True, grad_scale=4.0, mean=False)
    assert r.grad_weight is total
    ref = R.Vocab(h64, w64, t64, mean=False)
    (_, _), (rw, tw) = ref.gradients(-4.0 * ref.share, dtype == "bfloat16", False, False)
    rw = rw + start.double().cpu().numpy()
    close(total, rw, tw + 4 * R.EPS * np.abs(rw) + R.out_rounding(rw, given == "bfloat16"), "grad_weight")


@pytest.mark.parametrize("shape", [(16384, 16, 20000, "bfloat16", 64, 0, 0), (16384, 8, 70000, "bfloat16", 64, 0, 0),
                                   (16384, 16, 20000, "float32", 64, 0, 0), (30000, 7, 7000, "float32", 64, 0, 0),
                                   (3, 131072, 1600, "float32", 64, 0, 0)])
def test_pieces_of_the_vocabulary(env, shape):
    """16384 rows leave 65536 classes of bfloat16 and 13056 of float32 a piece of 2 GiB: one piece, whose exponentials
    are kept, and more."""
    torch, losses = env
    h, w, t, h64, w64, t64, _ = make(torch, shape, seed=3, idle=0.985)
    on = t64 >= 0
    ref = R.Vocab(h64[on], w64, t64[on])
    r = losses.vocab_loss(h, w, t)
    close(r.logp[torch.from_numpy(on).cuda()], ref.logp, ref.logp_tol, "logp")
    check_gradients(ref, -ref.share, r.grad_hidden[torch.from_numpy(on).cuda()], r.grad_weight, h.dtype is torch.bfloat16)
    assert (r.grad_hidden[torch.from_numpy(~on).cuda()] == 0).all()


def test_no_row_takes_part(env):
    torch, losses = env
    h = torch.full((70, 24), float("nan"), device="cuda")
    w = torch.randn(300, 24, device="cuda")
    t = torch.full((70,), -1, device="cuda")
    for kw in ({}, dict(weights=torch.ones(70, device="cuda"))):
        r = losses.vocab_loss(h, w, t, **kw)
        assert r.stats.tolist() == [0, 0] and (r.logp == 0).all() and (r.grad_hidden == 0).all() and (r.grad_weight == 0).all()
    r = losses.vocab_loss(h, w, torch.zeros_like(t), weights=torch.zeros(70, device="cuda"), grad_weight=w.clone(), accumulate=True)
    assert r.stats.tolist() == [0, 0] and torch.equal(r.grad_weight, w)
    # no row at all
    r = losses.vocab_loss(h[:0], w, t[:0], save=True)
    assert r.stats.tolist() == [0, 0] and r.logp.numel() == 0 and (r.grad_weight == 0).all()
    s = losses.vocab_logprobs(h[:0], w, t[:0], save=True)
    gh, gw = losses.vocab_logprobs_backward(h[:0], w, t[:0], s.saved, s.logp)
    assert gh.shape == (0, 24) and (gw == 0).all()
    # the C call with no row and a pointer to where its gradient would go
    from paper_1511_05946_amd import acdc
    from paper_1511_05946_amd._lib import lib
    spare, stats, gw = torch.full((24,), 3.0, device="cuda"), torch.ones(2, device="cuda"), torch.ones_like(w)
    ws = torch.empty(losses.vocab_workspace_bytes(h[:0], w), dtype=torch.uint8, device="cuda")
    head = struct.pack("3Q3q4i", h.data_ptr(), w.data_ptr(), t.data_ptr(), 24, 24, 0, 24, 300, 0, 64)
    record = struct.pack("2Q2q2i", spare.data_ptr(), gw.data_ptr(), 24, 24, 0, 0)
    rc = acdc._call(lib().acdc_vocab_loss, h.device, head, None, struct.pack("fi", 1.0, 1), stats.data_ptr(), None, None, None, record,
                    ws.data_ptr(), ws.numel())
    assert rc == 0 and stats.tolist() == [0, 0] and (spare == 3).all() and (gw == 0).all()


@pytest.mark.parametrize("rows", [2, 64, 300])
def test_weights_that_cancel(env, rows):
    """The mean over weights whose sum is 0: a loss and gradients of 0."""
    torch, losses = env
    h, w = torch.randn(rows, 24, device="cuda"), torch.randn(50, 24, device="cuda")
    t = torch.arange(rows, device="cuda") % 50
    weights = torch.ones(rows, device="cuda")
    weights[1::2] = -1
    r = losses.vocab_loss(h, w, t, weights=weights, save=True)
    assert r.stats.tolist() == [0, 0] and all((x == 0).all() for x in (r.grad_hidden, r.grad_weight, r.row_grads))
    assert (r.logp < 0).all()
    want = -(weights.double() * r.logp.double()).sum().item()
    r = losses.vocab_loss(h, w, t, weights=weights, mean=False, save=True)
    # one rounding of each product and one of the sum
    assert abs(r.stats[0].item() - want) <= 2 ** -24 * (r.logp.abs().double().sum().item() + abs(want)) and r.stats[1].item() == 0
    assert torch.equal(r.row_grads, -weights) and (r.grad_weight != 0).any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_what_is_not_a_number(env, dtype):
    """A target past the classes and hidden values that are not finite give NaN for their
    own row and the weight's gradient, and no other row."""
    torch, losses = env
    h, w, t, h64, w64, t64, _ = make(torch, (90, 40, 100, dtype, 64, 0, 0), seed=4)
    t64 = np.where(np.arange(90) < 3, 7, t64)
    ref = R.Vocab(h64, w64, t64)
    t = torch.from_numpy(t64).cuda()
    t[0], h[1, 3], h[2, 0] = 100, float("inf"), float("nan")
    r = losses.vocab_loss(h, w, t, mean=False)
    close(r.logp[3:], ref.logp[3:], ref.logp_tol[3:], "logp")
    assert torch.isnan(r.logp[:3]).all() and torch.isnan(r.stats[0]) and torch.isnan(r.grad_hidden[:3]).all()
    assert torch.isfinite(r.grad_hidden[3:]).all() and torch.isnan(r.grad_weight).all()
    # a scale of NaN leaves the rows that take no part at 0
    s = losses.vocab_logprobs(h, w, t, save=True)
    gh, _ = losses.vocab_logprobs_backward(h, w, t, s.saved, torch.ones(90, device="cuda"),
                                           scale=torch.full((1,), float("nan"), device="cuda"))
    assert (gh[t < 0] == 0).all() and torch.isnan(gh[t >= 0]).all()


@pytest.mark.parametrize("dtype,spread", [("float32", 60.0), ("bfloat16", 60.0), ("float32", 1e4)])
def test_far_logits(env, dtype, spread):
    """Rows whose softmax is one class, and classes of probability 0."""
    torch, losses = env
    h, w, t, h64, w64, t64, _ = make(torch, (33, 16, 70, dtype, 64, 0, 0), seed=5)
    w = (w.float() * spread).to(w.dtype)
    w64 = w.double().cpu().numpy()
    ref = R.Vocab(h64, w64, t64)
    r = losses.vocab_loss(h, w, t)
    close(r.logp, ref.logp, ref.logp_tol, "logp")
    assert torch.isfinite(r.grad_hidden).all() and torch.isfinite(r.grad_weight).all()
    if spread < 100:
        check_gradients(ref, -ref.share, r.grad_hidden, r.grad_weight, dtype == "bfloat16")


def test_floats_of_every_size(env):
    """float32 values are three bfloat16 planes: small, large, and the largest."""
    torch, losses = env
    h = torch.tensor([[1.0, 1e-30, 3.4e38], [2.0 ** -100, 1.0, 0.0], [1 + 2.0 ** -23, 1.0, 0.0]], device="cuda")
    w = torch.tensor([[1.0, 1e30, 0.0], [0.5, 0.25, 2.0 ** -130], [1.0, -1.0, 0.0]], device="cuda")
    t = torch.tensor([0, 1, 2], device="cuda")
    ref = R.Vocab(h.double().cpu().numpy(), w.double().cpu().numpy(), t.cpu().numpy())
    # products below 2^-126 may come out as 0
    close(losses.vocab_logprobs(h, w, t).logp, ref.logp, ref.logp_tol + 1e-37, "logp")


def test_gradients_against_differences(env):
    torch, losses = env
    h, w, t, *_ = make(torch, (6, 10, 20, "float32", 64, 0, 0), seed=6, idle=0.0)
    r = losses.vocab_loss(h, w, t)

    def loss(hh, ww):
        return torch.nn.functional.nll_loss((hh @ ww.T).log_softmax(1), t).item()

    d = 1e-5
    hd, wd = h.double(), w.double()
    for which, got in ((0, r.grad_hidden), (1, r.grad_weight)):
        x = (hd, wd)[which]
        for i in range(0, x.numel(), 7):
            vals = []
            for sign in (1, -1):
                y = x.clone()
                y.view(-1)[i] += sign * d
                vals.append(loss(y, wd) if which == 0 else loss(hd, y))
            diff = (vals[0] - vals[1]) / (2 * d)
            # the differences' own error: third derivative (below 10) d^2 / 6, and 1e-15 / d
            assert abs(got.reshape(-1)[i].item() - diff) <= 1e-8 + 1e-5 * abs(diff) + 64 * R.EPS


def test_autograd(env):
    torch, losses = env
    h, w, t, h64, w64, t64, share = make(torch, (50, 30, 80, "float32", 64, 2, 0), seed=7)
    want = losses.vocab_loss(h, w, t, weights=share.cuda(), grad_scale=0.5)
    a, b = h.clone().requires_grad_(True), w.clone().requires_grad_(True)
    loss, stats, logp = losses.vocab_loss_autograd(a, b, t, weights=share.cuda(), grad_scale=0.5)
    assert torch.equal(loss, want.stats[0]) and torch.equal(logp, want.logp)
    loss.backward()
    # the explicit form rounds share / W after the product, the differentiable one before
    for got, ref in ((a.grad, want.grad_hidden), (b.grad, want.grad_weight)):
        assert (got - ref).abs().max().item() <= 1e-5 * ref.abs().max().item()
    # one input alone, and an upstream gradient
    b2 = w.clone().requires_grad_(True)
    (3 * losses.vocab_loss_autograd(h, b2, t, weights=share.cuda())[0]).backward()
    assert (b2.grad - 6 * want.grad_weight).abs().max().item() <= 1e-5 * b2.grad.abs().max().item()
    a3, b3 = h.clone().requires_grad_(True), w.clone().requires_grad_(True)
    g = torch.randn(50, device="cuda")
    losses.vocab_logprobs_autograd(a3, b3, t).backward(g)
    s = losses.vocab_logprobs(h, w, t, save=True)
    gh, gw = losses.vocab_logprobs_backward(h, w, t, s.saved, g)
    assert torch.equal(a3.grad, gh) and torch.equal(b3.grad, gw)
    # a second derivative is an error
    a4 = torch.nan_to_num(h).requires_grad_(True)
    first, = torch.autograd.grad(losses.vocab_loss_autograd(a4, w, t)[0], a4, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiated again"):
        first.square().sum().backward()


@pytest.mark.parametrize("shape", [(300, 72, 700, "bfloat16", 64, 0, 0), (40, 65, 300, "float32", 64, 0, 0)])
def test_captured_and_on_another_stream(env, shape):
    torch, losses = env
    h, w, t, *_ = make(torch, shape, seed=8)
    ws = torch.empty(losses.vocab_workspace_bytes(h, w), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = losses.vocab_loss(h, w, t, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = losses.vocab_loss(h, w, t, workspace=ws)
    for k in range(4):
        if k == 2:   # other rows take part, other values
            t.copy_(t.flip(0))
            h.copy_(torch.randn(h.shape, device="cuda"))
        ws.fill_(255)
        graph.replay()
        want = losses.vocab_loss(h, w, t)
        torch.cuda.synchronize()
        for a, b in ((r.stats, want.stats), (r.logp, want.logp), (r.grad_hidden, want.grad_hidden), (r.grad_weight, want.grad_weight)):
            assert torch.equal(a, b), k
        if k == 0:
            assert torch.equal(first.grad_weight, want.grad_weight)
        junk = torch.randn(1 << 20, device="cuda").sum().item()
        assert junk == junk
