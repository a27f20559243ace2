"""Arguments of the losses and the optimiser whose memory is not what their
values say, or that no call may take (CPU: the binding's own checks)."""

import ctypes

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def calls(monkeypatch):
    """The binding on CPU tensors: the arguments of its library calls instead of the calls."""
    from paper_1511_05946_amd import losses, optim
    made = []

    def call(fn, device, *args):
        made.append(args)
        return 0

    monkeypatch.setattr(losses, "_call", call)
    monkeypatch.setattr(optim, "_call", call)
    return made


def conjugate_gradient(n=6):
    """A parameter and its gradient as autograd hands it out where the loss takes the conjugate."""
    w = torch.randn(n, dtype=torch.complex64).requires_grad_(True)
    (w.conj() * torch.randn(n, dtype=torch.complex64)).real.sum().backward()
    assert w.grad.is_conj()
    return w.detach(), w.grad


def test_step_takes_the_values_of_a_conjugate_gradient(calls, monkeypatch):
    from paper_1511_05946_amd import optim
    seen = []

    def call(fn, device, records, count, *rest):
        grad = ctypes.c_void_p.from_address(records + 16).value
        seen.extend((ctypes.c_float * 12).from_address(grad))
        return 0

    monkeypatch.setattr(optim, "_call", call)
    p, g = conjugate_gradient()
    optim.adamw_step([p], [g], [optim.moments(p)], 1)
    assert seen == torch.view_as_real(g.resolve_conj()).reshape(-1).tolist()


def test_step_refuses_views_that_it_would_write_wrongly(calls):
    from paper_1511_05946_amd import optim
    p, g = conjugate_gradient()
    r = torch.ones(6)
    half, neg = r.bfloat16(), torch._neg_view(r)
    for args, kw in ((([p.conj()], [g], [optim.moments(p)]), {}), (([neg], [r], [optim.moments(r)]), {}),
                     (([r], [r.clone()], [(neg, r.clone())]), {}), (([half], [r], [optim.moments(r)]), dict(masters=[neg]))):
        with pytest.raises(ValueError, match="view"):
            optim.adamw_step(*args, 1, **kw)
    with pytest.raises(ValueError):
        optim.grad_norm([r], out=torch._neg_view(torch.zeros(2)))
    assert not calls


def test_losses_refuse_negative_views(calls):
    from paper_1511_05946_amd import losses
    x, t, f, saved = torch.randn(4, 10), torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(4, 4)
    off = torch.tensor([0, 2, 4])
    n = torch._neg_view
    one = torch.randn(1, 1, dtype=torch.complex64).conj().imag   # one that torch makes by itself
    assert one.is_neg()
    for call in (lambda: losses.token_logprobs(n(x), t), lambda: losses.token_logprobs(one, t[:1]),
                 lambda: losses.token_logprobs_backward(x, t, n(saved), f),
                 lambda: losses.token_logprobs_backward(x, t, saved, n(f)),
                 lambda: losses.token_logprobs_backward(x, t, saved, f, scale=n(f[:1])),
                 lambda: losses.token_logprobs_backward(x, t, saved, f, out=n(x)),
                 lambda: losses.policy_loss(x, t, n(f), f), lambda: losses.policy_loss(x, t, f, n(f)),
                 lambda: losses.policy_loss(x, t, f, f, logp_ref=n(f)), lambda: losses.policy_loss(x, t, f, f, weights=n(f)),
                 lambda: losses.preference_loss(x, t, off, n(f))):
        with pytest.raises(ValueError, match="negative"):
            call()
    assert not calls


def test_torch_is_told_what_is_written(calls):
    from paper_1511_05946_amd import losses, optim
    x, t, f, saved = torch.randn(4, 10), torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(4, 4)
    off = torch.tensor([0, 2, 4])
    for call in (lambda o: losses.token_logprobs_backward(x, t, saved, f, out=o), lambda o: losses.policy_loss(x, t, f, f, out=o),
                 lambda o: losses.preference_loss(x, t, off, f, out=o)):
        out = torch.zeros(4, 10)
        call(out)
        assert out._version > 0 and x._version == f._version == saved._version == 0
    p, g, w = torch.ones(6).bfloat16(), torch.ones(6), torch.ones(6)
    state = optim.moments(p, 8)
    before = [s._version for s in state]
    optim.adamw_step([p], [g], [state], 1, masters=[w])
    assert p._version > 0 and w._version > 0 and g._version == 0 and all(s._version > b for s, b in zip(state, before))
    out = torch.zeros(2)
    optim.grad_norm([g], out=out)
    assert out._version > 0 and g._version == 0
    with torch.inference_mode():   # tensors without a version
        p = torch.ones(6)
        optim.adamw_step([p], [torch.ones(6)], [optim.moments(p)], 2)
        losses.policy_loss(torch.zeros(4, 10), t, f, f, out=torch.zeros(4, 10))


def freed(t):
    t = t.clone()
    t.untyped_storage().resize_(0)
    return t


def freed_part(t):
    """A part of a larger tensor whose storage was freed: its address is not even null."""
    t = torch.stack([t, t])[1]
    t.untyped_storage().resize_(0)
    return t


@pytest.mark.parametrize("gone", [freed, freed_part])
def test_tensors_without_memory_are_refused(calls, gone):
    from paper_1511_05946_amd import losses, optim
    x, t, f, saved = torch.randn(4, 10), torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(4, 4)
    off, ws = torch.tensor([0, 2, 4]), torch.zeros(1 << 16, dtype=torch.uint8)
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
    p, half = torch.ones(300), torch.ones(300).bfloat16()
    s32, s8 = optim.moments(p), optim.moments(p, 8)
    for args, kw in ((([gone(p)], [p], [s32]), {}), (([p], [gone(p)], [s32]), {}), (([p], [p], [(gone(p), p)]), {}),
                     (([p], [p], [(*s8[:2], gone(s8[2]), gone(s8[3]))]), {}),
                     (([half], [half], [s32]), dict(masters=[gone(p)])), (([p], [p], [s32]), dict(grad_scale=gone(p[:1])))):
        with pytest.raises(ValueError):
            optim.adamw_step(*args, 1, **kw)
    for kw in (dict(grads=[gone(p)]), dict(grads=[p], out=gone(p[:2]))):
        with pytest.raises(ValueError):
            optim.grad_norm(**kw)
    assert not calls


def test_workspaces_that_do_not_hold_their_size_are_refused(calls):
    """One byte read as many: the kernels write bytes next to each other."""
    from paper_1511_05946_amd import losses
    x, t = torch.randn(4, 10), torch.zeros(4, dtype=torch.int64)
    byte, apart = torch.zeros(1, dtype=torch.uint8).expand(1 << 16), torch.zeros(1 << 17, dtype=torch.uint8)[::2]
    for ws in (byte, apart):
        with pytest.raises(ValueError, match="workspace"):
            losses.token_logprobs(x, t, workspace=ws)
    assert not calls


def test_any_iterable_of_tensors(calls):
    """Generators, as modules give their parameters, and views of dictionaries."""
    from paper_1511_05946_amd import optim
    layer = torch.nn.Linear(4, 3)
    for p in layer.parameters():
        p.grad = torch.ones_like(p)
    state = {name: optim.moments(p) for name, p in layer.named_parameters()}
    optim.adamw_step(layer.parameters(), (p.grad for p in layer.parameters()), state.values(), 1)
    optim.grad_norm(p.grad for p in layer.parameters())
    half = {k: torch.ones(4).bfloat16() for k in "ab"}
    full = {k: torch.ones(4) for k in "ab"}
    optim.adamw_step(half.values(), full.values(), [optim.moments(p) for p in full.values()], 1,
                     masters=(full[k].clone() for k in "ab"))
    assert len(calls) == 3 and [c[1] for c in calls if len(c) == 7] == [2, 2]
    with pytest.raises(ValueError, match="one length"):
        optim.adamw_step(layer.parameters(), iter([]), state.values(), 1)
    with pytest.raises(ValueError, match="a tensor at least"):
        optim.grad_norm(iter([]))


def test_log_probabilities_ask_for_what_they_use():
    """Rows whole take no workspace to speak of, however many; few long ones the 16 bytes of
    each part, at least 4096 values long."""
    from paper_1511_05946_amd import _lib
    size = _lib.lib().acdc_logprob_workspace_size
    for dtype in (0, 1):
        for rows, classes in ((1 << 26, 2), (1 << 20, 1000), (64, 4096), (8, 4000), (0, 10)):
            assert 0 < size(rows, classes, dtype) <= 256
        for rows, classes in ((1, 1 << 18), (8, 131072), (40, 100000), (63, 20000)):
            assert 256 < size(rows, classes, dtype) <= 256 + 16 * rows * (classes // 4096)
