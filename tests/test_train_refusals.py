"""What the training operators refuse, on the host and before any HIP call (no
GPU needed): the C entry points' checks and the binding's."""

import ctypes
import os
import re
import struct

import pytest

from paper_1511_05946_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EUNSUP, EWS = 0, -1, -2, -3
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    return _lib.lib()


def test_every_declared_symbol_is_exported(L):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "acdc_train.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(acdc_[a-z_]+)\s*\(", src)))
    assert len(names) == 10
    for n in names:
        assert hasattr(L, n) and n in _lib.SIGNATURES, n


class Memory:
    """Host addresses that no case below gets dereferenced."""

    def __init__(self):
        self.buf = ctypes.create_string_buffer(1 << 16)
        self.base = (ctypes.addressof(self.buf) + 255) & ~255

    def __call__(self, i):
        return self.base + 2048 * i


def test_logprob_forward(L):
    p = Memory()
    x, t, logp, ent, saved, ws = (p(i) for i in range(6))

    def call(x=x, dtype=0, stride=10, t=t, bits=64, rows=4, V=10, logp=logp, ent=ent, saved=saved, ws=ws, wsb=1 << 20):
        return L.acdc_logprob_forward(x, dtype, stride, t, bits, rows, V, logp, ent, saved, ws, wsb, None)

    assert call(rows=0) == OK
    for bad in (dict(dtype=2), dict(dtype=-1), dict(stride=9), dict(bits=16), dict(rows=-1), dict(rows=1 << 31), dict(V=0),
                dict(x=None), dict(t=None), dict(x=x + 1), dict(x=x + 2), dict(t=t + 4), dict(logp=None), dict(logp=logp + 2),
                dict(ent=ent + 1), dict(saved=saved + 8), dict(stride=1 << 41)):
        assert call(**bad) == EINVAL, bad
    assert L.acdc_logprob_workspace_size(4, 10, 0) > 0
    assert call(ws=None) == EWS and call(wsb=L.acdc_logprob_workspace_size(4, 10, 0) - 1) == EWS
    for size in ((-1, 10, 0), (4, 0, 0), (4, 10, 5)):
        assert L.acdc_logprob_workspace_size(*size) == 0


def test_logprob_backward(L):
    p = Memory()
    x, t, saved, g, h, out = (p(i) for i in range(6))

    def call(x=x, dtype=0, stride=10, t=t, bits=32, saved=saved, g=g, h=h, scale=None, out=out, os_=10, rows=4, V=10):
        return L.acdc_logprob_backward(x, dtype, stride, t, bits, saved, g, h, scale, out, os_, rows, V, None)

    assert call(rows=0) == OK
    # the gradient's memory: the logits' own, row by row, or none of it
    for bad in (dict(saved=None), dict(saved=saved + 4), dict(g=None), dict(out=None), dict(os_=9), dict(out=out + 2),
                dict(h=h + 1), dict(scale=g + 2), dict(out=x, os_=11), dict(out=x + 4), dict(out=x + 40), dict(out=x - 40),
                dict(dtype=1, out=x + 2)):
        assert call(**bad) == EINVAL, bad


def test_policy_loss(L):
    p = Memory()
    x, t, old, ref, adv, w, stats, logp, grad, saved, rg, ws = (p(i) for i in range(12))

    def call(x=x, dtype=1, stride=10, t=t, bits=64, old=old, ref=ref, adv=adv, w=w, rows=4, V=10, params=(.2, .2, 0, 0, 1, 1),
             stats=stats, logp=logp, grad=grad, gs=10, saved=saved, rg=rg, ws=ws, wsb=1 << 20):
        return L.acdc_policy_loss(x, dtype, stride, t, bits, old, ref, adv, w, rows, V,
                                  None if params is None else struct.pack("5fi", *params), stats, logp, grad, gs, saved, rg,
                                  ws, wsb, None)

    for bad in (dict(params=None), dict(params=(-.1, .2, 0, 0, 1, 1)), dict(params=(.1, NAN, 0, 0, 1, 1)),
                dict(params=(.1, .2, INF, 0, 1, 1)), dict(params=(.1, .2, 0, NAN, 1, 1)), dict(params=(.1, .2, 0, 0, INF, 1)),
                dict(params=(.1, .2, .1, 0, 1, 1), ref=None), dict(stats=None), dict(old=None), dict(adv=None),
                dict(logp=None), dict(stats=stats + 2), dict(w=w + 1), dict(rg=rg + 2), dict(grad=x, gs=12), dict(grad=x + 2),
                dict(saved=saved + 4), dict(bits=8), dict(stride=3)):
        assert call(**bad) == EINVAL, bad
    assert call(ws=None) == EWS and call(wsb=8) == EWS


def test_preference_loss(L):
    p = Memory()
    x, t, off, ref, stats, logp, grad, saved, rg, ws = (p(i) for i in range(10))

    def call(x=x, dtype=0, stride=10, t=t, bits=64, off=off, ob=32, ref=ref, rows=4, V=10, pairs=2, params=(.1, 0, 1),
             stats=stats, logp=logp, grad=grad, gs=10, saved=saved, rg=rg, ws=ws, wsb=1 << 20):
        return L.acdc_preference_loss(x, dtype, stride, t, bits, off, ob, ref, rows, V, pairs,
                                      None if params is None else struct.pack("3f", *params), stats, logp, grad, gs, saved,
                                      rg, ws, wsb, None)

    for bad in (dict(params=None), dict(params=(NAN, 0, 1)), dict(params=(.1, -.1, 1)), dict(params=(.1, 1.1, 1)),
                dict(params=(.1, 0, INF)), dict(off=None), dict(off=off + 2), dict(ob=64, off=off + 4), dict(ob=16),
                dict(pairs=-1), dict(pairs=1 << 30), dict(ref=None), dict(logp=None), dict(stats=None), dict(grad=x + 8)):
        assert call(**bad) == EINVAL, bad
    assert call(ws=None) == EWS and call(wsb=8) == EWS
    assert L.acdc_preference_workspace_size(4, 10, 0, -1) == 0


def record(p, **kw):
    v = dict(param=p(0), master=0, grad=p(1), m=p(2), v=p(3), ms=0, vs=0, n=10, lr=1e-3, wd=0.0, pt=0, gt=0)
    v.update(kw)
    return struct.pack("=7Qqffii", *v.values())


def test_adamw_step(L):
    p = Memory()

    def call(rec=None, count=1, b1=.9, b2=.999, eps=1e-8, step=1, scale=None):
        return L.acdc_adamw_step(record(p) if rec is None else rec, count, b1, b2, eps, step, scale, None)

    assert call(count=0) == OK
    assert call(rec=record(p, n=0, param=0, grad=0, m=0, v=0)) == OK
    for bad in (dict(count=-1), dict(b1=1.0), dict(b1=-.1), dict(b2=NAN), dict(eps=-1.0), dict(eps=INF), dict(step=0),
                dict(scale=p(5) + 1)):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(param=0), dict(grad=0), dict(m=0), dict(v=0), dict(n=-1), dict(n=1 << 41), dict(lr=NAN), dict(wd=INF),
                dict(pt=2), dict(gt=-1), dict(master=p(4)), dict(pt=1, master=p(4) + 2), dict(ms=p(5)), dict(vs=p(5)),
                dict(m=p(2) + 1), dict(param=p(0) + 2), dict(ms=p(5) + 1, vs=p(6)), dict(m=p(3)), dict(grad=p(0)),
                dict(pt=1, master=p(0))):
        assert call(rec=record(p, **bad)) == EINVAL, bad
    # a bad tensor anywhere in the list: nothing is launched for the good ones before it
    assert call(rec=record(p) + record(p, m=0), count=2) == EINVAL


def test_grad_norm(L):
    p = Memory()

    def call(ptrs=(p(0), p(1)), sizes=(10, 20), types=(0, 1), count=2, most=1.0, out=p(2), ws=p(3), wsb=1 << 12):
        return L.acdc_grad_norm(struct.pack("2Q", *ptrs), struct.pack("2q", *sizes), struct.pack("2i", *types), count, most,
                                out, ws, wsb, None)

    for bad in (dict(ptrs=(0, p(1))), dict(ptrs=(p(0) + 2, p(1))), dict(ptrs=(p(0), p(1) + 1)), dict(sizes=(10, -1)),
                dict(types=(0, 2)), dict(count=-1), dict(most=NAN), dict(out=None), dict(out=p(2) + 2), dict(ws=p(3) + 4)):
        assert call(**bad) == EINVAL, bad
    assert call(ws=None) == EWS and call(wsb=8) == EWS
    assert L.acdc_grad_norm_workspace_size(struct.pack("2q", 10, 20), 2) > 0
    assert L.acdc_grad_norm_workspace_size(struct.pack("2q", 10, -20), 2) == 0


# ---------------------------------------------------------------- the binding


@pytest.fixture
def host(monkeypatch):
    """The binding on CPU tensors, with its calls counted instead of made."""
    torch = pytest.importorskip("torch")
    from paper_1511_05946_amd import losses, optim
    made = []

    def call(fn, device, *args):
        made.append(fn)
        return 0

    monkeypatch.setattr(losses, "_call", call)
    monkeypatch.setattr(optim, "_call", call)
    return torch, losses, optim, made


def test_binding_of_the_losses(host):
    torch, losses, _, made = host
    R, V = 6, 10
    x, t, f = torch.zeros(R, V), torch.zeros(R, dtype=torch.int64), torch.zeros(R)
    saved = torch.zeros(R, 4)
    off = torch.tensor([0, 2, 6])

    def logprobs(x=x, t=t, ws=None):
        return losses.token_logprobs(x, t, entropy=True, save=True, workspace=ws)

    def back(x=x, t=t, saved=saved, g=f, h=None, scale=None, out=None):
        return losses.token_logprobs_backward(x, t, saved, g, h, scale=scale, out=out)

    def policy(x=x, t=t, old=f, adv=f, **kw):
        return losses.policy_loss(x, t, old, adv, **kw)

    def preference(x=x, t=t, off=off, ref=f, **kw):
        return losses.preference_loss(x, t, off, ref, **kw)

    logprobs(), back(), policy(), preference()
    logprobs(x=torch.zeros(R, 16)[:, :V]), back(out=x), policy(x=x.bfloat16(), logp_ref=f, kl_coef=0.1, weights=f)
    good = len(made)
    assert good == 7
    wide, part = torch.zeros(R, 2 * V), torch.zeros(2 * R)[::2]
    bad = [(logprobs, dict(x=x.half())), (logprobs, dict(x=x.double())), (logprobs, dict(x=x[0])),
           (logprobs, dict(x=torch.zeros(R, 0))), (logprobs, dict(x=wide[:, ::2])), (logprobs, dict(x=x[:1].expand(R, V))),
           (logprobs, dict(x=torch.zeros(V, R).t())), (logprobs, dict(t=t[:-1])), (logprobs, dict(t=t.float())),
           (logprobs, dict(t=torch.zeros(2 * R, dtype=torch.int64)[::2])), (logprobs, dict(ws=torch.zeros(4, dtype=torch.uint8))),
           (logprobs, dict(ws=torch.zeros(4096))), (back, dict(saved=saved[:-1])), (back, dict(saved=saved.double())),
           (back, dict(saved=torch.zeros(4, R).t())), (back, dict(g=f[:-1])), (back, dict(g=part)), (back, dict(g=f[:1].expand(R))),
           (back, dict(h=f.double())), (back, dict(scale=f)), (back, dict(out=wide)), (back, dict(out=x.bfloat16())),
           (back, dict(out=x[:1].expand(R, V))), (policy, dict(old=f[:-1])), (policy, dict(adv=part)),
           (policy, dict(weights=f.bfloat16())), (policy, dict(kl_coef=0.1)), (policy, dict(clip=(-0.1, 0.2))),
           (policy, dict(clip=(NAN, 0.2))), (policy, dict(logp_ref=f[1:])), (preference, dict(off=off[:2])),
           (preference, dict(off=off.float())), (preference, dict(off=off.view(1, 3))), (preference, dict(ref=f[1:])),
           (preference, dict(label_smoothing=1.5)), (preference, dict(label_smoothing=NAN))]
    for fn, kw in bad:
        with pytest.raises(ValueError):
            fn(**kw)
    assert len(made) == good   # none of them reached the library
    # a shape that the meta device gives: tensors on different devices
    with pytest.raises(ValueError):
        logprobs(t=torch.zeros(R, dtype=torch.int64, device="meta"))
    with pytest.raises(ValueError):
        policy(adv=torch.zeros(R, device="meta"))


def test_binding_of_the_optimiser(host):
    torch, _, optim, made = host
    p, g = torch.zeros(300), torch.zeros(300)
    half = torch.zeros(300, dtype=torch.bfloat16)
    s32, s8 = optim.moments(p, 32), optim.moments(p, 8)
    assert [t.numel() for t in s8] == [300, 300, 2, 2] and s8[0].dtype is torch.float8_e4m3fn
    assert optim.moments(torch.zeros(3, dtype=torch.complex64))[0].numel() == 6

    def step(p=p, g=g, s=s32, master=None, **kw):
        optim.adamw_step([p], [g], [s], 1, masters=None if master is None else [master], **kw)

    step(), step(s=s8), step(p=half, g=half, master=p), step(lr=[0.1], weight_decay=[0.0]), optim.adamw_step([], [], [], 1)
    optim.grad_norm([g, half], max_norm=1.0)
    good = len(made)
    assert good == 5
    for kw in (dict(p=p.double()), dict(p=torch.zeros(600)[::2]), dict(g=g[:-1]), dict(g=None), dict(g=g.half()),
               dict(g=g.view(3, 100)), dict(g=torch.zeros(1).expand(300)), dict(s=s32[:1]), dict(s=s8[:3]),
               dict(s=(s32[0], s32[1][:-1])), dict(s=(s32[0], s8[1])), dict(s=(*s8[:2], s8[2][:1], s8[3])),
               dict(s=(*s32, *s8[2:])), dict(master=p), dict(p=half, g=half, master=half), dict(p=half, g=half, master=p[:-1]),
               dict(lr=[0.1, 0.2]), dict(weight_decay=[]), dict(grad_scale=torch.zeros(2)),
               dict(grad_scale=torch.zeros(1, dtype=torch.float64)), dict(g=torch.zeros(300, dtype=torch.complex64))):
        with pytest.raises(ValueError):
            step(**kw)
    with pytest.raises(ValueError):
        optim.adamw_step([p], [g, g], [s32], 1)
    with pytest.raises(ValueError):
        optim.adamw_step([p], [g], [s32], 1, masters=[])
    with pytest.raises(ValueError):
        optim.moments(p, 16)
    for kw in (dict(grads=[]), dict(grads=[p.double()]), dict(grads=[torch.zeros(6)[::2]]), dict(grads=[g], max_norm=0.0),
               dict(grads=[g], max_norm=NAN), dict(grads=[g], out=torch.zeros(3)), dict(grads=[g], out=torch.zeros(2).double())):
        with pytest.raises(ValueError):
            optim.grad_norm(**kw)
    assert len(made) == good
