"""The losses, the cascade's passes and the step together, as the example runs
them: a policy that follows a teacher's preferences and then its rewards."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


@pytest.mark.parametrize("bits", [8, 32])
def test_example_improves_in_both_phases(env, bits):
    from paper_1511_05946_amd import policy
    print(f"[case] cascade policy, moments in {bits} bits", flush=True)
    start, preference, final = policy.train(bits=bits)
    print([start, preference, final], flush=True)
    # a reward is a rank in [0, 1): 0.5 is chance; each phase closes a tenth of what is left at least
    assert preference[1] > start[1] + 0.1 * (1 - start[1])
    assert final[1] > preference[1] + 0.1 * (1 - preference[1])


def test_step_through_the_cascade_matches_autograd(env):
    """dL/dA, dL/dD, dL/dbias of the loss through the cascade: the explicit calls
    against the differentiable ones. Both run the same kernels on the same row
    gradients; the autograd form computes the logits' gradient in another pass."""
    torch = env
    from paper_1511_05946_amd import acdc, losses, policy
    torch.manual_seed(3)
    N, V, rows = 64, 50, 40
    p = policy.CascadePolicy(N, 3, V, torch.device("cuda:0"))
    x = torch.randn(rows, N, device="cuda")
    a = torch.randint(0, V, (rows,), device="cuda")
    old, adv = torch.full((rows,), -4.0, device="cuda"), torch.randn(rows, device="cuda")
    logits, saved = p.logits(x)
    grad_y = torch.zeros_like(x)
    losses.policy_loss(logits, a, old, adv, entropy_coef=0.01, out=grad_y[:, :V])
    A, D, bias = p.params
    _, *want = acdc.backward(x, grad_y, A, D, saved=saved, bias=bias)
    leaves = [t.clone().requires_grad_(True) for t in p.params]
    y = acdc.acdc_cascade(x, leaves[0], leaves[1], None, 0, leaves[2])
    loss, _, _ = losses.policy_loss_autograd(y[:, :V], a, old, adv, entropy_coef=0.01)
    loss.backward()
    for leaf, w in zip(leaves, want):
        # sums of 40 rows of terms that differ by a few units in the last place
        assert (leaf.grad - w).abs().max().item() <= 1e-5 * w.abs().max().item()


def test_step_in_a_graph(env):
    """The whole step captured once and replayed, with eager work between: each
    replay equals the eager step on the same values."""
    torch = env
    from paper_1511_05946_amd import acdc, losses, optim
    torch.manual_seed(5)
    N, K, V, rows = 256, 2, 200, 96
    x = torch.randn(rows, N, device="cuda")
    a = torch.randint(0, V, (rows,), device="cuda")
    old, adv = torch.full((rows,), -5.0, device="cuda"), torch.randn(rows, device="cuda")
    start = [1 + 0.1 * torch.randn(K, N, device="cuda") for _ in range(2)]
    acdc.prepare(N)

    def fresh():
        p = [t.clone() for t in start]
        return p, [optim.moments(t, 8) for t in p], torch.zeros(rows, N, device="cuda")

    def step(p, m, grad_y):
        y, saved = acdc.forward(x, p[0], p[1], save=True)
        r = losses.policy_loss(y[:, :V], a, old, adv, out=grad_y[:, :V])
        _, *g = acdc.backward(x, grad_y, p[0], p[1], saved=saved)
        clip = optim.grad_norm(g, max_norm=0.5)
        optim.adamw_step(p, g, m, 1, lr=1e-2, grad_scale=clip[1:])
        return r.stats, clip

    eager = fresh()
    warm = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*warm)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    captured = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stats, clip = step(*captured)
    for k in range(4):
        graph.replay()
        want, want_clip = step(*eager)
        torch.cuda.synchronize()
        assert torch.equal(stats, want) and torch.equal(clip, want_clip), k
        assert all(torch.equal(u, v) for u, v in zip(captured[0], eager[0])), k
        junk = torch.randn(1 << 20, device="cuda").sum().item()
        assert junk == junk
