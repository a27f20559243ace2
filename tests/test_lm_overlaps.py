"""No output of the language-model operators may share memory with what its call reads, with
another output, or with the workspace: refused by the C entry points and in words by the
binding, before any HIP call (no GPU needed)."""

import struct

import pytest

from paper_1511_05946_amd import _lib
from test_lm_refusals import N, R, V, f, grads, h, head, host, saved, t, u, vocab_calls, w, workspace  # noqa: F401 (host: a fixture)
from test_train_refusals import EINVAL

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def L():
    return _lib.lib()


class Far:
    """Host addresses a MiB apart, that no case below gets dereferenced."""

    def __init__(self):
        self.base = 1 << 40

    def __call__(self, i):
        return self.base + (i << 20)


WS = 1 << 19   # the workspace: more than any call here needs, less than the next address


def test_vocab_calls(L):
    p = Far()
    logp, saved, stats, rg, g, scale, weights, ws = (p(i) for i in range(5, 13))

    def logprob(logp=logp, saved=saved, ws=ws):
        return L.acdc_vocab_logprob(head(p), logp, saved, ws, WS, None)

    def backward(out=None, saved=saved, g=g, scale=scale, ws=ws):
        return L.acdc_vocab_backward(head(p), saved, g, scale, out or grads(p), ws, WS, None)

    def loss(out=None, weights=weights, stats=stats, logp=logp, saved=saved, rg=rg, ws=ws):
        return L.acdc_vocab_loss(head(p), weights, struct.pack("fi", 1.0, 1), stats, logp, saved, rg, out or grads(p), ws, WS, None)

    inputs = (p(0), p(1), p(2))   # hidden, weight, targets
    gh, gw = p(3), p(4)
    bad = [(logprob, dict(logp=a)) for a in (*inputs, saved + 28)] + [(logprob, dict(saved=a)) for a in (p(0) + 152, p(1), p(2) + 24)]
    bad += [(logprob, dict(ws=a)) for a in (*inputs, logp, saved, p(0) - 4096)]
    for call in (backward, loss):
        bad += [(call, dict(out=grads(p, h=a))) for a in (*inputs, gw + 476, saved, saved + 28)]
        bad += [(call, dict(out=grads(p, w=a))) for a in (*inputs, gh + 156, saved)]
        bad += [(call, dict(ws=a)) for a in (*inputs, gh, gw, saved, p(1) - 2048)]
    bad += [(backward, dict(out=grads(p, **{k: a}))) for k in "hw" for a in (g, scale, g + 12)] + [(backward, dict(ws=a)) for a in (g, scale)]
    bad += [(loss, dict(out=grads(p, **{k: a}))) for k in "hw" for a in (weights, stats, logp, rg)]
    bad += [(loss, {k: a}) for k in ("stats", "logp", "rg", "saved") for a in (*inputs, weights, weights + 8, gh, gw, gh + 152)]
    bad += [(loss, dict(ws=a)) for a in (weights, stats, logp, rg)]
    bad += [(loss, dict(stats=logp)), (loss, dict(logp=rg + 12)), (loss, dict(rg=saved)), (loss, dict(saved=stats)), (loss, dict(stats=saved + 24))]
    for call, kw in bad:
        assert call(**kw) == EINVAL, (call.__name__, kw)


def test_norm_calls(L):
    p = Far()
    x, weight, b, y, saved, gx, gw, gb, ws = (p(i) for i in range(9))

    def forward(x=x, w=weight, b=b, y=y, saved=saved):
        return L.acdc_norm_forward(x, 0, 10, w, b, 0, 1e-5, y, 0, 10, saved, 65, 10, None)

    def backward(x=x, gy=y, w=weight, saved=saved, gx=gx, gw=gw, gb=gb, ws=ws):
        return L.acdc_norm_backward(x, 0, 10, gy, 0, 10, w, 0, saved, gx, 10, gw, gb, 0, 0, 65, 10, ws, WS, None)

    bad = [(forward, dict(y=a)) for a in (x, weight, b, saved, x + 2596, saved + 512)]
    bad += [(forward, dict(saved=a)) for a in (x, weight, b, y, y + 2592)]
    bad += [(backward, dict(gx=a)) for a in (x, y + 40, weight, saved, gw, gb, saved + 512)]
    bad += [(backward, {k: a}) for k in ("gw", "gb") for a in (x, y, weight, saved, gx, x + 2560, y + 2596, saved + 516)]
    bad += [(backward, dict(gw=gb + 36)), (backward, dict(gx=y, gw=y)), (backward, dict(gx=y, ws=y))]
    bad += [(backward, dict(ws=a)) for a in (x, y, weight, saved, gx, gw, gb, saved - 256)]
    for call, kw in bad:
        assert call(**kw) == EINVAL, (call.__name__, kw)


def test_embedding_calls(L):
    p = Far()
    t, weight, y, ws = (p(i) for i in range(4))

    def forward(t=t, bits=64, w=weight, y=y):
        return L.acdc_embedding_forward(t, bits, w, 0, 10, 1.0, y, 0, 10, 4, 10, 12, None)

    def backward(t=t, bits=64, g=y, w=weight, ws=ws):
        return L.acdc_embedding_backward(t, bits, g, 0, 10, 1.0, w, 0, 10, 0, 4, 10, 12, ws, WS, None)

    bad = [(forward, dict(y=a)) for a in (t, t + 28, weight, weight + 476)] + [(forward, dict(t=y + 152)), (forward, dict(t=y + 156, bits=32))]
    bad += [(backward, dict(w=a)) for a in (t, t + 28, y, y + 156)] + [(backward, dict(ws=a)) for a in (t, y, weight, weight - 1024)]
    for call, kw in bad:
        assert call(**kw) == EINVAL, (call.__name__, kw)


def test_binding(host):  # noqa: F811
    losses, layers, made = host
    loss, _, back = vocab_calls(losses)
    room = torch.zeros(4096)   # one memory for two arguments

    def rows(n, width=N):
        return room[:n * width].view(n, width)

    vector, targets = room[4:4 + R], room[:2 * R].view(torch.int64)
    bad = [lambda: loss(t=targets, out=rows(R)), lambda: loss(t=targets, grad_weight=rows(V)),
           lambda: loss(weights=vector, out=rows(R)), lambda: loss(weights=vector, grad_weight=rows(V)),
           lambda: back(t=targets, out=rows(R)), lambda: back(g=vector, out=rows(R)), lambda: back(g=vector, grad_weight=rows(V)),
           lambda: back(saved=rows(R, 2), out=rows(R)), lambda: back(saved=rows(R, 2), grad_weight=rows(V)),
           lambda: back(scale=room[:1], out=rows(R)), lambda: back(scale=room[:1], grad_weight=rows(V)),
           lambda: layers.layer_norm_backward(h, h, u, rows(R, 2), out=rows(R)),
           lambda: layers.layer_norm_backward(h, h, u, rows(R, 2), grads=(room[:N], None)),
           lambda: layers.layer_norm_backward(h, h, u, rows(R, 2), grads=(None, room[:N])),
           lambda: layers.layer_norm_backward(h, rows(R), u, saved, out=rows(R), grads=(room[N:2 * N], None)),
           lambda: layers.embedding(targets, w, out=rows(R)), lambda: layers.embedding_backward(targets, h, V, grad_weight=rows(V))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError, match="overlaps"):
            call()
            pytest.fail(f"call {i} went through")
    assert not made
    # grad_y's own memory for grad_x, the sums beside it
    layers.layer_norm_backward(h, rows(R), u, saved, out=rows(R), grads=(room[1024:1024 + N], room[2048:2048 + N]))
    assert len(made) == 1
