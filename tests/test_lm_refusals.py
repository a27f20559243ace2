"""What the language-model operators refuse, on the host and before any HIP call (no
GPU needed): the C entry points' checks and the binding's."""

import os
import re
import struct

import pytest

from paper_1511_05946_amd import _lib
from test_train_arguments import freed, freed_part
from test_train_refusals import EINVAL, EWS, INF, NAN, OK, Memory

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def L():
    return _lib.lib()


def test_every_declared_symbol_is_exported(L):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "acdc_train_lm.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(acdc_[a-z_]+)\s*\(", src)))
    assert len(names) == 10
    for n in names:
        assert hasattr(L, n) and n in _lib.SIGNATURES, n


def head(p, **kw):
    v = dict(h=p(0), w=p(1), t=p(2), hs=10, ws=10, rows=4, width=10, classes=12, dtype=0, bits=64)
    v.update(kw)
    return struct.pack("3Q3q4i", *(0 if x is None else x for x in v.values()))


def grads(p, **kw):
    v = dict(h=p(3), w=p(4), hs=10, ws=10, type=0, add=0)
    v.update(kw)
    return struct.pack("2Q2q2i", *(0 if x is None else x for x in v.values()))


BAD_HEADS = (dict(h=None), dict(w=None), dict(t=None), dict(hs=9), dict(ws=9), dict(hs=1 << 41), dict(ws=1 << 41), dict(rows=-1),
             dict(rows=(1 << 24) + 1), dict(width=0), dict(width=(1 << 17) + 1, hs=1 << 18, ws=1 << 18), dict(classes=0),
             dict(classes=(1 << 27) + 1), dict(dtype=2), dict(dtype=-1), dict(bits=16))


def test_vocab_calls(L):
    p = Memory()
    size = L.acdc_vocab_workspace_size(4, 10, 12, 0, 1)
    assert size > L.acdc_vocab_workspace_size(4, 10, 12, 0, 0) > 0
    for bad in ((-1, 10, 12, 0), (4, 0, 12, 0), (4, 10, 0, 0), (4, 10, 12, 3), (1 << 25, 10, 12, 0), (4, 1 << 18, 12, 0)):
        assert L.acdc_vocab_workspace_size(*bad, 1) == 0
    ws, logp, saved, stats, rg, g, scale, w = p(8), p(9), p(10), p(11), p(12), p(13), p(14), p(15)
    big = 1 << 40

    def logprob(hd=None, logp=logp, saved=saved, ws=ws, wsb=big):
        return L.acdc_vocab_logprob(head(p) if hd is None else hd, logp, saved, ws, wsb, None)

    def backward(hd=None, saved=saved, g=g, scale=scale, out=None, ws=ws, wsb=big):
        return L.acdc_vocab_backward(head(p) if hd is None else hd, saved, g, scale, grads(p) if out is None else out, ws, wsb, None)

    def loss(hd=None, w=w, params=struct.pack("fi", 1.0, 1), stats=stats, logp=logp, saved=saved, rg=rg, out=None, ws=ws, wsb=big):
        return L.acdc_vocab_loss(head(p) if hd is None else hd, w, params, stats, logp, saved, rg, grads(p) if out is None else out,
                                 ws, wsb, None)

    assert logprob(hd=head(p, rows=0, h=None, t=None)) == OK
    assert backward(out=grads(p, h=None, w=None)) == OK   # nothing is wanted
    for call in (logprob, backward, loss):
        assert call(hd=b"\0" * 64) == EINVAL
        for bad in BAD_HEADS + (dict(h=p(0) + 2), dict(w=p(1) + 1), dict(t=p(2) + 4)):
            assert call(hd=head(p, **bad)) == EINVAL, (call, bad)
        assert call(ws=None) == EWS and call(wsb=64) == EWS and call(ws=ws + 128) == EINVAL
    assert loss(wsb=size - 1) == EWS and backward(wsb=size - 1) == EWS
    for bad in (dict(logp=None), dict(logp=logp + 2), dict(saved=saved + 4)):
        assert logprob(**bad) == EINVAL, bad
    # gradients in the inputs' memory, in each other's, out of line
    where = (dict(h=p(0)), dict(h=p(0) + 4), dict(h=p(1) + 8), dict(w=p(1)), dict(w=p(0)), dict(h=p(4)), dict(h=p(3) + 2), dict(w=p(4) + 1),
             dict(hs=9), dict(ws=9), dict(type=1), dict(type=-1), dict(hs=1 << 41), dict(ws=1 << 41))
    for bad in where:
        assert backward(out=grads(p, **bad)) == EINVAL, bad
        assert loss(out=grads(p, **bad)) == EINVAL, bad
    for bad in (dict(saved=None), dict(saved=saved + 4), dict(g=None), dict(g=g + 1), dict(scale=scale + 2)):
        assert backward(**bad) == EINVAL, bad
    for bad in (dict(params=None), dict(params=struct.pack("fi", NAN, 1)), dict(params=struct.pack("fi", INF, 0)), dict(stats=None),
                dict(stats=stats + 2), dict(logp=None), dict(w=w + 2), dict(saved=saved + 4), dict(rg=rg + 1)):
        assert loss(**bad) == EINVAL, bad


def test_norm_calls(L):
    p = Memory()
    x, w, b, y, saved, gx, gw, gb, ws = (p(i) for i in range(9))

    def forward(x=x, xt=0, xs=10, w=w, b=b, vt=0, eps=1e-5, y=y, yt=1, ys=10, saved=saved, rows=4, width=10):
        return L.acdc_norm_forward(x, xt, xs, w, b, vt, eps, y, yt, ys, saved, rows, width, None)

    def backward(x=x, xt=0, xs=10, gy=y, yt=0, gs=10, w=w, vt=0, saved=saved, gx=gx, gxs=10, gw=gw, gb=gb, gt=0, add=0, rows=4,
                 width=10, ws=ws, wsb=1 << 20):
        return L.acdc_norm_backward(x, xt, xs, gy, yt, gs, w, vt, saved, gx, gxs, gw, gb, gt, add, rows, width, ws, wsb, None)

    assert forward(rows=0, x=None, y=None) == OK and backward(rows=0, add=1) == OK
    assert backward(gx=None, gw=None, gb=None, ws=None) == OK   # nothing is wanted
    for bad in (dict(x=None), dict(y=None), dict(xt=2), dict(yt=-1), dict(vt=3), dict(xs=9), dict(ys=9), dict(x=x + 2), dict(y=y + 1),
                dict(w=w + 1), dict(b=b + 2), dict(eps=-1e-5), dict(eps=NAN), dict(eps=INF), dict(saved=saved + 4), dict(rows=-1),
                dict(rows=1 << 31), dict(width=0), dict(width=1 << 25, xs=1 << 25, ys=1 << 25), dict(y=x), dict(y=x + 40), dict(y=w),
                dict(xs=1 << 41)):
        assert forward(**bad) == EINVAL, bad
    for bad in (dict(x=None), dict(gy=None), dict(saved=None), dict(xt=2), dict(yt=2), dict(vt=2), dict(gt=2), dict(xs=9), dict(gs=9),
                dict(gxs=9), dict(gx=gx + 2), dict(gw=gw + 1), dict(gb=gb + 2), dict(saved=saved + 4), dict(rows=-1), dict(width=0),
                dict(gx=x), dict(gx=y + 40), dict(gx=y, gxs=11), dict(gx=y, yt=1), dict(gw=gb), dict(gw=w), dict(gb=x), dict(gb=gx),
                dict(ws=ws + 4)):
        assert backward(**bad) == EINVAL, bad
    many = dict(rows=65, xt=1, yt=1)   # more rows than one workgroup takes
    assert backward(**many, ws=None) == EWS and backward(**many, wsb=8) == EWS
    assert L.acdc_norm_workspace_size(4, 10) > 0 and L.acdc_norm_workspace_size(-1, 10) == 0 and L.acdc_norm_workspace_size(4, 0) == 0


def test_embedding_calls(L):
    p = Memory()
    t, w, y, ws = (p(i) for i in range(4))

    def forward(t=t, bits=64, w=w, wt=0, wst=10, scale=1.0, y=y, yt=1, ys=10, rows=4, width=10, classes=12):
        return L.acdc_embedding_forward(t, bits, w, wt, wst, scale, y, yt, ys, rows, width, classes, None)

    def backward(t=t, bits=64, g=y, gt=0, gs=10, scale=1.0, w=w, wt=0, wst=10, add=0, rows=4, width=10, classes=12, ws=ws, wsb=1 << 20):
        return L.acdc_embedding_backward(t, bits, g, gt, gs, scale, w, wt, wst, add, rows, width, classes, ws, wsb, None)

    assert forward(rows=0, t=None, y=None) == OK and backward(rows=0, t=None, g=None, add=1) == OK
    for bad in (dict(t=None), dict(t=t + 4), dict(bits=16), dict(w=None), dict(wt=2), dict(wst=9), dict(w=w + 2), dict(y=None),
                dict(yt=2), dict(ys=9), dict(y=y + 1), dict(scale=NAN), dict(scale=INF), dict(rows=-1), dict(rows=1 << 28), dict(width=0),
                dict(width=(1 << 20) + 1, wst=1 << 21, ys=1 << 21), dict(classes=0), dict(classes=(1 << 30) + 1), dict(y=w), dict(y=w + 400)):
        assert forward(**bad) == EINVAL, bad
    for bad in (dict(t=None), dict(t=t + 4), dict(bits=8), dict(g=None), dict(gt=2), dict(gs=9), dict(g=y + 2), dict(w=None), dict(wt=2),
                dict(wst=9), dict(w=w + 1), dict(scale=NAN), dict(rows=-1), dict(classes=0), dict(width=0), dict(w=y), dict(w=y + 8),
                dict(ws=ws + 64)):
        assert backward(**bad) == EINVAL, bad
    assert backward(ws=None) == EWS and backward(wsb=8) == EWS
    assert L.acdc_embedding_workspace_size(4, 10, 12) > 0
    for bad in ((-1, 10, 12), (4, 0, 12), (4, 10, 0), (1 << 28, 10, 12), ((1 << 28) - 64, 1 << 20, 12)):
        assert L.acdc_embedding_workspace_size(*bad) == 0


# ---------------------------------------------------------------- the binding


@pytest.fixture
def host(monkeypatch):
    """The binding on CPU tensors, with its calls counted instead of made."""
    from paper_1511_05946_amd import layers, losses
    made = []

    def call(fn, device, *args):
        made.append(fn)
        return 0

    monkeypatch.setattr(losses, "_call", call)
    monkeypatch.setattr(layers, "_call", call)
    return losses, layers, made


R, N, V = 6, 10, 12
h, w, t, f = torch.randn(R, N), torch.randn(V, N), torch.zeros(R, dtype=torch.int64), torch.zeros(R)
saved, u = torch.zeros(R, 2), torch.ones(N)
neg = torch._neg_view


def workspace(n=1 << 20):
    full = torch.zeros(n + 256, dtype=torch.uint8)
    skip = -full.data_ptr() % 256
    return full[skip:skip + n]


def vocab_calls(losses):
    def loss(h=h, w=w, t=t, **kw):
        return losses.vocab_loss(h, w, t, **kw)

    def logprobs(h=h, w=w, t=t, **kw):
        return losses.vocab_logprobs(h, w, t, **kw)

    def back(h=h, w=w, t=t, saved=saved, g=f, **kw):
        return losses.vocab_logprobs_backward(h, w, t, saved, g, **kw)

    return loss, logprobs, back


def test_binding_of_the_vocabulary_losses(host):
    losses, _, made = host
    loss, logprobs, back = vocab_calls(losses)
    r = loss(save=True)
    assert r.grad_hidden.shape == (R, N) and r.grad_weight.shape == (V, N) and r.saved.shape == (R, 2) and r.row_grads.shape == (R,)
    assert loss(grad=False).grad_hidden is None and loss(grad="weight").grad_hidden is None and loss(grad="hidden").grad_weight is None
    logprobs(save=True), back(), back(out=torch.zeros(R, N)), back(grad_weight=torch.zeros(V, N), accumulate=True)
    wide = torch.zeros(R, 2 * N)
    loss(h=wide[:, :N], out=torch.zeros(R, 16)[:, 2:2 + N]), loss(h=h.bfloat16(), w=w.bfloat16(), grad_weight=torch.zeros(V, N))
    loss(workspace=workspace(losses.vocab_workspace_bytes(h, w)))
    good = len(made)
    for call in (loss, logprobs, back):
        for kw in (dict(h=h.half()), dict(h=h.double()), dict(h=h[0]), dict(h=torch.zeros(R, 0)), dict(h=wide[:, ::2]),
                   dict(h=h[:1].expand(R, N)), dict(h=torch.zeros(N, R).t()), dict(w=w.bfloat16()), dict(w=w[:, :-1]), dict(w=w[:0]),
                   dict(w=w[0]), dict(w=w[:1].expand(V, N)), dict(t=t[:-1]), dict(t=t.float()), dict(t=t.view(2, 3)),
                   dict(t=torch.zeros(2 * R, dtype=torch.int64)[::2]), dict(w=w.to("meta")), dict(t=t.to("meta")), dict(h=neg(h)),
                   dict(w=neg(w)), dict(workspace=torch.zeros(4, dtype=torch.uint8)), dict(workspace=workspace()[64:]),
                   dict(workspace=torch.zeros(1 << 20)), dict(workspace=workspace(1 << 21)[::2])):
            with pytest.raises(ValueError):
                call(**kw)
    out, gw = torch.zeros(R, N), torch.zeros(V, N)
    for call in (loss, back):
        for kw in (dict(grad="both"), dict(grad=None), dict(out=out[:-1]), dict(out=out.bfloat16()), dict(out=out[:1].expand(R, N)),
                   dict(out=torch.zeros(N, R).t()), dict(out=h), dict(out=w[:R]), dict(grad_weight=gw[:-1]), dict(grad_weight=gw.double()),
                   dict(grad_weight=gw.bfloat16()), dict(grad_weight=w), dict(grad_weight=gw[:1].expand(V, N)), dict(accumulate=True),
                   dict(out=gw[:R], grad_weight=gw), dict(out=neg(out)), dict(grad_weight=neg(gw))):
            with pytest.raises(ValueError):
                call(**kw)
    for kw in (dict(saved=saved[:-1]), dict(saved=torch.zeros(R, 4)), dict(saved=saved.double()), dict(saved=torch.zeros(2, R).t()),
               dict(saved=neg(saved)), dict(g=f[:-1]), dict(g=f[:1].expand(R)), dict(g=f.double()), dict(g=neg(f)), dict(scale=f)):
        with pytest.raises(ValueError):
            back(**kw)
    for kw in (dict(grad_scale=NAN), dict(grad_scale=INF), dict(weights=f[:-1]), dict(weights=f.double()), dict(weights=f[:1].expand(R)), dict(weights=neg(f))):
        with pytest.raises(ValueError):
            loss(**kw)
    big = torch.zeros(1, (1 << 17) + 1)
    with pytest.raises(ValueError, match="supported"):
        loss(h=big, w=big, t=t[:1])
    assert len(made) == good


def test_binding_of_the_layers(host):
    _, layers, made = host

    def norm(x=h, w=u, b=u, **kw):
        return layers.layer_norm(x, w, b, **kw)

    def norm_back(x=h, g=h, w=u, saved=saved, **kw):
        return layers.layer_norm_backward(x, g, w, saved, **kw)

    def embed(t=t, w=w, **kw):
        return layers.embedding(t, w, **kw)

    def embed_back(t=t, g=h, classes=V, **kw):
        return layers.embedding_backward(t, g, classes, **kw)

    r = norm(save=True, dtype=torch.bfloat16)
    assert r.y.dtype is torch.bfloat16 and r.saved.shape == (R, 2)
    norm(w=None, b=None), norm(w=u.bfloat16(), b=None), norm(out=torch.zeros(R, 16)[:, 3:3 + N])
    gx, gw, gb = norm_back(dtype=torch.bfloat16)
    assert gx.dtype is torch.float32 and gw.dtype is gb.dtype is torch.bfloat16
    assert norm_back(grad=(False, True, False))[0] is None
    place = torch.zeros(R, N)
    assert norm_back(g=place, out=place)[0] is place
    norm_back(grads=(torch.zeros(N), None), accumulate=True)
    assert embed(dtype=torch.bfloat16).dtype is torch.bfloat16 and embed(t=t.int(), scale=2.0, out=torch.zeros(R, 12)[:, :N]).shape == (R, N)
    assert embed_back().shape == (V, N) and embed_back(dtype=torch.bfloat16).dtype is torch.bfloat16
    embed_back(grad_weight=torch.zeros(V, 2 * N)[:, :N], accumulate=True)
    norm_back(workspace=workspace()), embed_back(workspace=workspace())
    good = len(made)
    assert good == 15
    wide = torch.zeros(R, 2 * N)
    rows = (lambda a: a.half(), lambda a: a.double(), lambda a: a[0], lambda a: wide[:, ::2], lambda a: a[:1].expand(R, N), neg,
            lambda a: torch.zeros(N, R).t(), lambda a: torch.zeros(R, 0))
    bad = [(norm, dict(x=c(h))) for c in rows] + [(norm_back, dict(x=c(h))) for c in rows] + [(norm_back, dict(g=c(h))) for c in rows]
    bad += [(embed_back, dict(g=c(h))) for c in rows]
    bad += [(call, dict(w=c)) for call in (norm, norm_back) for c in (u[:-1], u.double(), torch.ones(2 * N)[::2], u[:1].expand(N), neg(u),
                                                                   u.view(2, 5), u.to("meta"))]
    bad += [(norm, dict(b=u.bfloat16())), (norm, dict(eps=-1.0)), (norm, dict(eps=NAN)), (norm, dict(eps=INF)),
            (norm, dict(dtype=torch.float16)), (norm, dict(out=wide)), (norm, dict(out=h)), (norm, dict(out=torch.zeros(R, N), dtype=torch.bfloat16)),
            (norm_back, dict(saved=saved[:-1])), (norm_back, dict(saved=torch.zeros(R, 4))), (norm_back, dict(saved=neg(saved))),
            (norm_back, dict(g=h[:-1])), (norm_back, dict(out=h.clone().bfloat16())), (norm_back, dict(out=h)),
            (norm_back, dict(g=place.bfloat16(), out=place[:-1])), (norm_back, dict(grads=(u,))), (norm_back, dict(grads=(u[:-1], None))),
            (norm_back, dict(grads=(torch.zeros(N), torch.zeros(N).bfloat16()))), (norm_back, dict(accumulate=True)),
            (norm_back, dict(grads=(u, None))), (norm_back, dict(dtype=torch.float64)),
            (norm_back, dict(workspace=torch.zeros(4, dtype=torch.uint8))), (embed, dict(scale=NAN)), (embed_back, dict(scale=INF)), (embed, dict(t=t.float())), (embed, dict(t=t.view(2, 3))),
            (embed, dict(t=torch.zeros(2 * R, dtype=torch.int64)[::2])), (embed, dict(t=t.to("meta"))), (embed, dict(w=w[:0])),
            (embed, dict(w=w.half())), (embed, dict(w=w[0])), (embed, dict(w=neg(w))), (embed, dict(out=wide)), (embed, dict(out=w[:R])),
            (embed, dict(dtype=torch.int32)), (embed_back, dict(t=t[:-1])), (embed_back, dict(classes=0)), (embed_back, dict(classes=-3)),
            (embed_back, dict(grad_weight=torch.zeros(V + 1, N))), (embed_back, dict(grad_weight=torch.zeros(V, N).double())),
            (embed_back, dict(accumulate=True)), (embed_back, dict(workspace=workspace()[32:])),
            (embed_back, dict(workspace=torch.zeros(16, dtype=torch.uint8)))]
    shared = torch.zeros(2 * V, N)
    bad += [(embed_back, dict(g=shared[:R], grad_weight=shared[:V]))]
    for fn, kw in bad:
        with pytest.raises(ValueError):
            fn(**kw)
    with pytest.raises(ValueError):   # one tensor for both sums
        one = torch.zeros(N)
        norm_back(grads=(one, one))
    assert len(made) == good


@pytest.mark.parametrize("gone", [freed, freed_part])
def test_tensors_without_memory_are_refused(host, gone):
    losses, layers, made = host
    loss, logprobs, back = vocab_calls(losses)
    for call in (lambda: loss(h=gone(h)), lambda: loss(w=gone(w)), lambda: loss(t=gone(t)), lambda: loss(weights=gone(f)),
                 lambda: loss(out=gone(h)), lambda: loss(grad_weight=gone(w)), lambda: logprobs(h=gone(h)), lambda: back(saved=gone(saved)),
                 lambda: back(g=gone(f)), lambda: back(scale=gone(f[:1])), lambda: layers.layer_norm(gone(h)),
                 lambda: layers.layer_norm(h, gone(u)), lambda: layers.layer_norm(h, u, gone(u)), lambda: layers.layer_norm(h, out=gone(h)),
                 lambda: layers.layer_norm_backward(h, gone(h), u, saved), lambda: layers.layer_norm_backward(h, h, u, gone(saved)),
                 lambda: layers.layer_norm_backward(h, h, u, saved, grads=(gone(u), None)), lambda: layers.embedding(gone(t), w),
                 lambda: layers.embedding(t, gone(w)), lambda: layers.embedding_backward(t, gone(h), V),
                 lambda: layers.embedding_backward(t, h, V, grad_weight=gone(w))):
        with pytest.raises(ValueError, match="without memory"):
            call()
    assert not made


def test_torch_is_told_what_is_written(host):
    losses, layers, _ = host
    loss, _, back = vocab_calls(losses)
    for call in (lambda o, g: loss(out=o, grad_weight=g), lambda o, g: back(out=o, grad_weight=g)):
        out, gw = torch.zeros(R, N), torch.zeros(V, N)
        call(out, gw)
        assert out._version > 0 and gw._version > 0
    out, gw = torch.zeros(R, N), torch.zeros(V, N)
    loss(out=out, grad_weight=gw, grad=False)   # not written
    assert out._version == gw._version == 0
    y, gx, a, b, e = torch.zeros(R, N), torch.zeros(R, N), torch.zeros(N), torch.zeros(N), torch.zeros(V, N)
    layers.layer_norm(h, out=y)
    layers.layer_norm_backward(h, h, u, saved, out=gx, grads=(a, b))
    layers.embedding_backward(t, h, V, grad_weight=e)
    assert all(x._version > 0 for x in (y, gx, a, b, e)) and h._version == u._version == 0
    rows = torch.zeros(R, N)
    layers.embedding(t, w, out=rows)
    assert rows._version > 0
