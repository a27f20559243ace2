"""Arguments of the losses and the optimiser on the GPU whose memory is not what
their values say, and what autograd has to know of the calls."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1511_05946_amd import losses, optim
    return torch, losses, optim


def test_step_of_a_conjugate_gradient(env):
    torch, _, optim = env
    gen = torch.Generator().manual_seed(1)
    start, a = (torch.randn(3, 70, dtype=torch.complex64, generator=gen).cuda() for _ in range(2))
    w = start.clone().requires_grad_(True)
    (w.conj() * a).real.sum().backward()
    assert w.grad.is_conj()
    got = []
    for g in (w.grad, w.grad.resolve_conj().clone()):
        p = start.clone()
        state = optim.moments(p)
        for step in (1, 2):
            optim.adamw_step([p], [g], [state], step)
        got.append((p, *state))
    assert all(torch.equal(x, y) for x, y in zip(*got))


def test_step_of_negative_views(env):
    torch, _, optim = env
    g = torch.randn(300, generator=torch.Generator().manual_seed(2)).cuda()
    got = []
    for grad, scale in ((torch._neg_view(g), torch._neg_view(torch.full((1,), -0.5, device="cuda"))),
                        (-g, torch.full((1,), 0.5, device="cuda"))):
        p = torch.ones(300, device="cuda")
        state = optim.moments(p, 8)
        optim.adamw_step([p], [grad], [state], 1, grad_scale=scale)
        got.append([x.view(torch.uint8) for x in (p, *state)])
    assert all(torch.equal(x, y) for x, y in zip(*got))
    assert torch.equal(optim.grad_norm([torch._neg_view(g)]), optim.grad_norm([g]))
    p = torch.ones(300, device="cuda")
    with pytest.raises(ValueError, match="view"):
        optim.adamw_step([torch._neg_view(p)], [g], [optim.moments(p)], 1)
    assert (p == 1).all()


def test_losses_of_negative_views(env):
    torch, losses, _ = env
    x, t, f = torch.randn(4, 10, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.ones(4, device="cuda")
    off, saved = torch.tensor([0, 2, 4], device="cuda"), torch.ones(4, 4, device="cuda")
    n = torch._neg_view
    for call in (lambda: losses.token_logprobs(n(x), t), lambda: losses.policy_loss(x, t, f, n(f)),
                 lambda: losses.preference_loss(x, t, off, n(f)), lambda: losses.policy_loss(x, t, f, f, out=n(x)),
                 lambda: losses.token_logprobs_backward(x, t, n(saved), f)):
        with pytest.raises(ValueError, match="negative"):
            call()
    assert torch.equal(losses.token_logprobs(n(x).resolve_neg(), t).logp, losses.token_logprobs(-x, t).logp)


def losses_of(torch, losses, **options):
    """Per loss: its logits, its gradient by the differentiable form, and by the call itself."""
    gen = torch.Generator().manual_seed(3)
    x, a = torch.randn(12, 50, generator=gen).cuda(), torch.randn(12, generator=gen).cuda()
    t, off = torch.arange(12, device="cuda"), torch.tensor([0, 3, 6, 9, 12], device="cuda")
    old = torch.full((12,), -4.0, device="cuda")
    for auto, plain, args in ((losses.policy_loss_autograd, losses.policy_loss, (t, old, a)),
                              (losses.preference_loss_autograd, losses.preference_loss, (t, off, old))):
        leaf = x.clone().requires_grad_(True)
        loss, stats, _ = auto(leaf, *args, **options)
        loss.backward()
        yield leaf.grad, plain(x, *args, **options).grad_logits, loss.detach(), plain(x, *args).stats[0]


def test_differentiable_losses_take_a_gradient_scale(env):
    """As the calls themselves: 0.25 is a power of two, so that the scaled gradient is a
    quarter of the unscaled one to the bit; the two forms differ by roundings of the row's factors."""
    torch, losses, _ = env
    unscaled = list(losses_of(torch, losses))
    for (got, want, loss, value), (full, *_) in zip(losses_of(torch, losses, grad_scale=0.25), unscaled):
        assert torch.equal(got, 0.25 * full)
        assert torch.allclose(got, want, rtol=1e-5, atol=1e-9) and loss == value


def test_differentiable_losses_refuse_a_tensor_for_the_gradient(env):
    torch, losses, _ = env
    x, t, f = torch.randn(4, 10, device="cuda", requires_grad=True), torch.zeros(4, dtype=torch.int64, device="cuda"), \
        torch.zeros(4, device="cuda")
    off, out = torch.tensor([0, 2, 4], device="cuda"), torch.full((4, 10), 7.0, device="cuda")
    with pytest.raises(ValueError, match="out"):
        losses.policy_loss_autograd(x, t, f, f, out=out)
    with pytest.raises(ValueError, match="out"):
        losses.preference_loss_autograd(x, t, off, f, out=out)
    assert (out == 7).all()


def test_step_between_the_passes_of_a_cascade_is_noticed(env):
    """The backward pass needs A and D as they were."""
    torch, losses, optim = env
    from paper_1511_05946_amd import acdc
    A, D = (torch.ones(2, 64, device="cuda", requires_grad=True) for _ in range(2))
    x = torch.randn(8, 64, device="cuda")
    for k in range(2):
        loss = acdc.acdc_cascade(x, A, D).square().sum()
        p = [A.detach(), D.detach()][k:k + 1]
        optim.adamw_step(p, [torch.ones(2, 64, device="cuda")], [optim.moments(p[0])], 1)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()


def test_gradient_over_saved_logits_is_noticed(env):
    torch, losses, _ = env
    x, t, f = torch.randn(4, 10, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    off = torch.tensor([0, 2, 4], device="cuda")
    saved = losses.token_logprobs(x, t, save=True).saved
    for over in (lambda y: losses.policy_loss(y, t, f, f, out=y), lambda y: losses.preference_loss(y, t, off, f, out=y),
                 lambda y: losses.token_logprobs_backward(y, t, saved, f, out=y)):
        leaf = x.clone().requires_grad_(True)
        y = leaf * 1.0
        logp, _ = losses.token_logprobs_autograd(y, t)
        over(y.detach()[:, :10])
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            logp.sum().backward()


def test_versions_of_the_optimisers_tensors(env):
    torch, _, optim = env
    p, g, w = torch.ones(600, device="cuda").bfloat16(), torch.ones(600, device="cuda"), torch.ones(600, device="cuda")
    for bits in (32, 8):
        state = optim.moments(p, bits)
        out = torch.zeros(2, device="cuda")
        watched = [p, w, *state, out]
        before = [t._version for t in watched]
        optim.adamw_step([p], [g], [state], 1, masters=[w])
        optim.grad_norm([g], out=out)
        assert all(t._version > b for t, b in zip(watched, before)) and g._version == 0
    with torch.inference_mode():   # tensors without a version
        q = torch.ones(600, device="cuda")
        optim.adamw_step([q], [g], [optim.moments(q)], 1)
        optim.grad_norm([q], out=torch.zeros(2, device="cuda"))


def test_second_derivatives_are_refused(env):
    """A gradient penalty beside another term: an error, not the other term's gradient alone."""
    torch, losses, _ = env
    x, t, f = torch.randn(4, 10, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    off = torch.tensor([0, 2, 4], device="cuda")
    for form in (lambda y: losses.token_logprobs_autograd(y, t)[0].sum(), lambda y: losses.policy_loss_autograd(y, t, f - 2, f + 1)[0],
                 lambda y: losses.preference_loss_autograd(y, t, off, f)[0]):
        leaf = x.clone().requires_grad_(True)
        loss = form(leaf)
        grad, = torch.autograd.grad(loss, leaf, create_graph=True)
        with pytest.raises(RuntimeError, match="cannot be differentiated again"):
            (grad.square().sum() + form(leaf)).backward()
        first = x.clone().requires_grad_(True)
        form(first).backward()
        assert torch.equal(first.grad, grad.detach())


def test_second_derivatives_of_a_cascade_are_refused(env):
    torch, *_ = env
    from paper_1511_05946_amd import acdc
    for bias in (None, torch.ones(2, 64, device="cuda", requires_grad=True)):
        x, A, D = (torch.randn(n, 64, device="cuda").requires_grad_(True) for n in (8, 2, 2))
        leaves = [t for t in (x, A, D, bias) if t is not None]
        first = torch.autograd.grad(acdc.acdc_cascade(x, A, D, bias=bias).square().sum(), leaves)
        for k, leaf in enumerate(leaves):
            y = acdc.acdc_cascade(x, A, D, bias=bias).square().sum()
            grad = torch.autograd.grad(y, leaves, create_graph=True)
            assert all(torch.equal(u, v.detach()) for u, v in zip(first, grad))
            with pytest.raises(RuntimeError, match="cannot be differentiated again"):
                (grad[k].square().sum() + y).backward()


@pytest.mark.parametrize("part", [False, True])
def test_tensors_without_memory_are_refused(env, part):
    """Nothing is launched: the library would take a null address for an argument left out
    (8-bit moments without scales for 32-bit ones), and another for memory."""
    torch, losses, optim = env

    def gone(t):
        t = torch.stack([t, t])[1] if part else t.clone()
        t.untyped_storage().resize_(0)
        return t

    x, t, f = torch.randn(4, 10, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    saved, off = torch.zeros(4, 4, device="cuda"), torch.tensor([0, 2, 4], device="cuda")
    ws = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    for call in (lambda: losses.token_logprobs(gone(x), t), lambda: losses.token_logprobs(x, gone(t)),
                 lambda: losses.token_logprobs(x, t, workspace=gone(ws)),
                 lambda: losses.token_logprobs_backward(x, t, gone(saved), f),
                 lambda: losses.token_logprobs_backward(x, t, saved, f, gone(f)),
                 lambda: losses.token_logprobs_backward(x, t, saved, f, scale=gone(f[:1])),
                 lambda: losses.token_logprobs_backward(x, t, saved, f, out=gone(x)),
                 lambda: losses.policy_loss(x, t, f, f, weights=gone(f)), lambda: losses.policy_loss(x, t, f, f, logp_ref=gone(f)),
                 lambda: losses.policy_loss(x, t, f, f, out=gone(x)), lambda: losses.preference_loss(x, t, gone(off), f)):
        with pytest.raises(ValueError, match="without memory"):
            call()
    p, g = torch.ones(300, device="cuda"), torch.ones(300, device="cuda")
    half = p.bfloat16()
    s32, s8 = optim.moments(p), optim.moments(p, 8)
    for args, kw in ((([gone(p)], [g], [s32]), {}), (([p], [gone(g)], [s32]), {}), (([p], [g], [(gone(g), g)]), {}),
                     (([p], [g], [(*s8[:2], gone(s8[2]), gone(s8[3]))]), {}),
                     (([half], [g], [s32]), dict(masters=[gone(p)])), (([p], [g], [s32]), dict(grad_scale=gone(p[:1])))):
        with pytest.raises(ValueError):
            optim.adamw_step(*args, 1, **kw)
    for kw in (dict(grads=[gone(p)]), dict(grads=[p], out=gone(p[:2]))):
        with pytest.raises(ValueError):
            optim.grad_norm(**kw)
    assert (p == 1).all() and (half == 1).all() and not s32[0].any()


def test_options_without_a_truth_value(env):
    torch, losses, _ = env
    x, t, f = torch.randn(4, 10, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    off, two = torch.tensor([0, 2, 4], device="cuda"), torch.ones(2)
    for call in (lambda: losses.token_logprobs(x, t, entropy=two), lambda: losses.token_logprobs(x, t, save=two),
                 lambda: losses.policy_loss(x, t, f, f, mean=two), lambda: losses.policy_loss(x, t, f, f, grad=two),
                 lambda: losses.preference_loss(x, t, off, f, save=two)):
        with pytest.raises(RuntimeError, match="[Bb]oolean"):
            call()


@pytest.mark.parametrize("rows,V,dtype", [(1, 1 << 18, "float32"), (8, 131072, "bfloat16"), (40, 100000, "float32"), (63, 20000, "bfloat16"),
                                          (3000, 40, "float32")])
def test_log_probabilities_stay_in_their_workspace(env, rows, V, dtype):
    torch, losses, _ = env
    print(f"[case] workspace of {rows} x {V} {dtype}", flush=True)
    x = torch.randn(rows, V, generator=torch.Generator().manual_seed(rows)).to(getattr(torch, dtype)).cuda()
    t = torch.arange(rows, device="cuda") % V
    need = losses._logprob_bytes(rows, V, 0 if dtype == "float32" else 1)
    room = torch.full((need + 8192,), 77, dtype=torch.uint8, device="cuda")
    r = losses.token_logprobs(x, t, entropy=True, workspace=room[4096:4096 + need])
    assert (room[:4096] == 77).all() and (room[4096 + need:] == 77).all()
    want = x.double().log_softmax(1)[torch.arange(rows, device="cuda"), t]
    # x_t - M, log S and their difference rounded, S's terms and sums: under 100 units of these sizes
    assert ((r.logp.double() - want).abs() <= 100 * 2.0 ** -24 * want.abs().clamp(min=1)).all()
    with pytest.raises(ValueError, match="workspace"):
        losses.token_logprobs(x, t, workspace=room[4096:4096 + need - 1])


def test_gradient_beside_the_logits_in_wider_rows(env):
    """Rows of one buffer that hold logits and gradients next to each other overlap nowhere."""
    torch, losses, _ = env
    from paper_1511_05946_amd.acdc import ACDCError
    rows, V = 20, 30
    x = torch.randn(rows, V, generator=torch.Generator().manual_seed(5)).cuda()
    t, f = torch.arange(rows, device="cuda"), torch.full((rows,), -3.0, device="cuda")
    for first, second, wide in ((0, 30, 60), (33, 2, 64), (1, 31, 61)):
        room = torch.full((rows + 1, wide), 7.0, device="cuda")
        logits, out = room[:rows, first:first + V], room[:rows, second:second + V]
        logits.copy_(x)
        want = losses.policy_loss(logits, t, f, f + 4)   # (the same logits: a row's sums follow its alignment)
        r = losses.policy_loss(logits, t, f, f + 4, out=out)
        assert torch.equal(out, want.grad_logits) and torch.equal(r.stats, want.stats) and torch.equal(logits, x)
        rest = torch.ones(rows + 1, wide, dtype=torch.bool, device="cuda")
        rest[:rows, first:first + V] = rest[:rows, second:second + V] = False
        assert (room[rest] == 7).all()
        # and of rows further on, which stand a whole number of rows away besides
        room[:rows - 2, first:first + V].copy_(x[:rows - 2])
        below = losses.policy_loss(room[:rows - 2, first:first + V], t[:-2], f[:-2], f[:-2] + 4, out=room[2:rows, second:second + V])
        assert torch.equal(room[:rows - 2, first:first + V], x[:rows - 2])
        want = losses.policy_loss(room[:rows - 2, first:first + V], t[:-2], f[:-2], f[:-2] + 4)
        assert torch.equal(below.grad_logits, want.grad_logits) and torch.equal(below.stats, want.stats)
    room = torch.zeros(rows, 2 * V, device="cuda")
    for second in (1, V - 1, 0):   # columns in common, or the same ones a row further on
        with pytest.raises(ACDCError, match="invalid argument"):
            losses.policy_loss(room[:rows - 1, :V], t[:-1], f[:-1], f[:-1], out=room[1 if second == 0 else 0:][:rows - 1, second:second + V])
    assert not room.any()


@pytest.mark.parametrize("kind,bits,most", [("f32", 32, 156), ("master", 32, 133), ("f32", 8, 116), ("master", 8, 103)])
def test_lists_around_a_full_launch_of_offsets(env, kind, bits, most):
    """The first list that a launch does not hold, and twice that: to the bit as one by one."""
    torch, _, optim = env
    import test_gpu_optim as T
    for count in (most - 1, most, most + 1, 2 * most, 2 * most + 1):
        print(f"[case] adamw list of {count} {kind} {bits} bits", flush=True)
        T.same_as_one_by_one(torch, optim, lambda: T.problem(torch, optim, [1 + 53 * k % 900 for k in range(count)], kind, bits,
                                                             count)[:4])
