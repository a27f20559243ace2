"""The AdamW step and the gradient norm on the GPU against their definitions in
64 bits."""

import numpy as np
import pytest

import train_reference as R

pytestmark = pytest.mark.gpu

BETAS, EPS, LR, DECAY = (0.9, 0.999), 1e-8, 1e-2, 0.1


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1511_05946_amd import optim
    return torch, optim


KINDS = {"f32": ("float32", "float32", False), "f32_bf16": ("float32", "bfloat16", False),
         "bf16": ("bfloat16", "bfloat16", False), "bf16_f32": ("bfloat16", "float32", False),
         "master": ("bfloat16", "bfloat16", True), "master_f32": ("bfloat16", "float32", True)}
SIZES = [0, 1, 3, 4, 5, 255, 256, 257, 1000, 4095, 4096, 4097, 70001]


def cut(torch, values, dtype, shift):
    """values on the GPU, `shift` elements into their memory."""
    t = torch.empty(len(values) + shift, dtype=dtype, device="cuda")[shift:]
    t.copy_(torch.from_numpy(np.ascontiguousarray(values)))
    return t


def problem(torch, optim, sizes, kind, bits, seed=0, shift=0):
    """(params, grads, moments, masters) on the GPU and, per tensor, what they stand for in float64."""
    p_type, g_type, master = KINDS[kind]
    rng = np.random.RandomState(seed)
    params, grads, moments, masters, ref = [], [], [], [], []
    for n in sizes:
        w = (1 + 0.3 * rng.randn(n)).astype(np.float32)
        g = (0.1 * rng.randn(n) * np.exp(rng.randn(n))).astype(np.float32)
        m = (0.05 * rng.randn(n)).astype(np.float32)
        root = np.abs(0.1 * rng.randn(n)).astype(np.float32)
        if n > 300:
            g[10:20] = 0
            m[5:290] = 0       # parts of blocks, and a whole one below
            root[256:] = root[256:] * (np.arange(n - 256) % 1024 >= 256)
            m[256:] = m[256:] * (np.arange(n - 256) % 1024 >= 256)
        p = cut(torch, w, getattr(torch, p_type), shift)
        g = cut(torch, g, getattr(torch, g_type), shift)
        if bits == 32:
            state = (cut(torch, m, torch.float32, shift), cut(torch, root ** 2, torch.float32, shift))
            m64, v64 = state[0].double().cpu().numpy(), state[1].double().cpu().numpy()
        else:
            state = optim.moments(p, 8)
            wide = []
            for k, x in enumerate((m, root)):
                scale = R.block_scale(x.astype(float)).astype(np.float32)
                each = np.repeat(scale, R.BLOCK)[:n]
                q = np.where(each > 0, x / np.where(each > 0, each, 1), 0)
                codes = torch.from_numpy(np.ascontiguousarray(q.astype(np.float32))).to(torch.float8_e4m3fn)
                moved = torch.empty(n + shift, dtype=torch.uint8, device="cuda")[shift:]
                moved.copy_(codes.view(torch.uint8))
                state = list(state)
                state[k] = moved.view(torch.float8_e4m3fn)
                state[2 + k].copy_(torch.from_numpy(scale))
                wide.append(codes.double().numpy() * each.astype(float))
            state = tuple(state)
            m64, v64 = wide[0], wide[1] ** 2
        params.append(p)
        grads.append(g)
        moments.append(state)
        masters.append(cut(torch, w, torch.float32, shift) if master else None)
        ref.append((w.astype(float) if master else p.double().cpu().numpy(), g.double().cpu().numpy(), m64, v64))
    return params, grads, moments, masters if master else None, ref


def check(torch, params, moments, masters, ref, bits, step, lr, decay, scale=1.0):
    for i, (w, g, m, v) in enumerate(ref):
        n = len(w)
        lr_i = lr[i] if isinstance(lr, list) else lr
        d_i = decay[i] if isinstance(decay, list) else decay
        w2, m2, v2, move = R.adamw(w, g * scale, m, v, step, lr_i, BETAS, EPS, d_i)
        # m, v: three roundings of their terms; the step: those, a root, a quotient
        m_tol = 4 * R.EPS * (np.abs(m) + np.abs(g * scale))
        v_tol = 4 * R.EPS * v2
        with np.errstate(all="ignore"):
            part = np.where(np.abs(m2) > 0, m_tol / np.abs(m2), 0.0)
        w_tol = 4 * R.EPS * np.abs(w) + move * (16 * R.EPS + part) + 1e-30
        got = masters[i] if masters else params[i]
        if got.dtype is torch.bfloat16:
            w_tol = w_tol + R.BF16 * np.abs(w2)
        err = np.abs(got.double().cpu().numpy() - w2)
        assert np.all(err <= w_tol), (i, n, np.argmax(err - w_tol), err.max())
        if masters:
            assert torch.equal(params[i], masters[i].to(torch.bfloat16))
        if bits == 32:
            assert np.all(np.abs(moments[i][0].double().cpu().numpy() - m2) <= m_tol)
            assert np.all(np.abs(moments[i][1].double().cpu().numpy() - v2) <= v_tol)
            continue
        for k, (x, tol) in enumerate(((m2, m_tol), (np.sqrt(v2), 8 * R.EPS * np.sqrt(v2)))):
            codes = moments[i][k].double().cpu().numpy()
            scales = moments[i][2 + k].double().cpu().numpy()
            want = R.block_scale(x)
            assert np.all(np.abs(scales - want) <= 8 * R.EPS * want)
            each = np.repeat(scales, R.BLOCK)[:n]
            # a code is the nearest one: half a step of 1/8 of its power of two away, or of the smallest step
            half = np.maximum(np.abs(x) / 16, each * R.TINY / 2) * (1 + 1e-5) + tol
            off = np.abs(codes * each - x)
            if k == 1:
                small = (x > 0) & (x < each * R.TINY)
                assert np.all(codes[x > 0] > 0)
                off, half = np.where(small, 0.0, off), half
            assert np.all(off <= half), (i, k, np.argmax(off - half))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("shift", [0, 1])
def test_step(env, kind, bits, shift):
    torch, optim = env
    print(f"[case] adamw {kind} {bits} bits shift={shift}", flush=True)
    params, grads, moments, masters, ref = problem(torch, optim, SIZES, kind, bits, 1, shift)
    optim.adamw_step(params, grads, moments, 3, lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY, masters=masters)
    check(torch, params, moments, masters, ref, bits, 3, LR, DECAY)


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors_of_every_kind_in_one_call(env, bits):
    """More tensors than one launch takes, types and moments mixed, a rate and a decay for each."""
    torch, optim = env
    print(f"[case] adamw mixed {bits}", flush=True)
    rng = np.random.RandomState(2)
    every = []
    for k in range(230):
        kind = sorted(KINDS)[k % len(KINDS)]
        b = bits if k % 3 else (8 if bits == 32 else 32)
        one = problem(torch, optim, [int(rng.randint(1, 9000))], kind, b, 100 + k, k % 2)
        every.append((one, b))
    params, grads, moments, masters = ([e[0][j][0] if e[0][j] is not None else None for e, *_ in
                                        [((o,), b) for o, b in every]] for j in range(4))
    lr, decay = [LR * (1 + k % 4) for k in range(230)], [0.0 if k % 2 else DECAY for k in range(230)]
    scale = torch.tensor([0.3], device="cuda")
    optim.adamw_step(params, grads, moments, 11, lr=lr, betas=BETAS, eps=EPS, weight_decay=decay, masters=masters,
                     grad_scale=scale)
    s = float(scale.double()[0])
    for k, (one, b) in enumerate(every):
        check(torch, [params[k]], [moments[k]], [masters[k]] if masters[k] is not None else None, one[4], b, 11, lr[k],
              decay[k], s)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind", ["f32", "master_f32"])
@pytest.mark.parametrize("rates", [1, 11])
def test_lists_of_every_length(env, kind, bits, rates):
    """One kind of tensor: lists about as long as short and long arguments hold, and longer than any
    launch's, with as many rates as a launch has and with more, to the bit as the tensors one by one."""
    torch, optim = env
    for count in (1, 6, 7, 8, 9, 10, 11, 12, 61, 62, 63, 64, 65, 70, 74, 75, 104, 105, 210):
        print(f"[case] adamw list of {count} {kind} {bits} {rates}", flush=True)
        lr = [LR * (1 + k % rates) for k in range(count)]
        state = []
        for together in (True, False):
            params, grads, moments, masters, _ = problem(torch, optim, [1 + 37 * k % 1500 for k in range(count)], kind, bits,
                                                         count)
            for at in [slice(None)] if together else [slice(k, k + 1) for k in range(count)]:
                optim.adamw_step(params[at], grads[at], moments[at], 5, lr=lr[at], betas=BETAS, eps=EPS, weight_decay=DECAY,
                                 masters=masters[at] if masters else None)
            state.append((params, moments, masters or []))
        (p, m, w), (p1, m1, w1) = state
        for a, b in zip([*p, *w, *(x for t in m for x in t)], [*p1, *w1, *(x for t in m1 for x in t)]):
            bytes_a, bytes_b = a.view(torch.uint8), b.view(torch.uint8)
            assert torch.equal(bytes_a, bytes_b)


def same_as_one_by_one(torch, optim, make):
    """The step of a list, to the bit that of its tensors one by one; `make` builds the same list twice."""
    state = []
    for together in (True, False):
        params, grads, moments, masters = make()
        count = len(params)
        lr = [LR * (1 + k % 3) for k in range(count)]
        for at in [slice(None)] if together else [slice(k, k + 1) for k in range(count)]:
            optim.adamw_step(params[at], grads[at], moments[at], 5, lr=lr[at], betas=BETAS, eps=EPS, weight_decay=DECAY,
                             masters=masters[at] if masters else None)
        state.append([x.clone().view(torch.uint8) for x in [*params, *(masters or []), *(x for t in moments for x in t)]])
    assert all(torch.equal(a, b) for a, b in zip(*state))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind", ["f32", "master"])
@pytest.mark.parametrize("shift", [0, 1])
def test_long_lists(env, kind, bits, shift):
    """Lists about as long as a launch takes as offsets, and with one tensor off their alignment."""
    torch, optim = env
    for count in (102, 103, 116, 117, 133, 134, 156, 157, 320):
        print(f"[case] adamw long list of {count} {kind} {bits} shift={shift}", flush=True)

        def make():
            lists = problem(torch, optim, [1 + 53 * k % 2900 for k in range(count)], kind, bits, count)[:4]
            if bits == 8:  # all scales in one buffer, a float apart
                scales = [torch.cat([m[j] for m in lists[2]]) for j in (2, 3)]
                at = np.cumsum([0, *(len(m[2]) for m in lists[2])])
                for k, m in enumerate(lists[2]):
                    lists[2][k] = (*m[:2], *(x[at[k]:at[k + 1]] for x in scales))
            if shift:
                odd = problem(torch, optim, [777], kind, bits, 1, shift)[:4]
                for x, y in zip(lists, odd):
                    if x is not None:
                        x[count // 2] = y[0]
            return lists

        same_as_one_by_one(torch, optim, make)


def test_long_list_with_a_large_tensor(env):
    """A list of offsets holds tensors of up to 2^29 - 1 elements: one at that length, one longer."""
    torch, optim = env
    for large in ((1 << 29) - 1, (1 << 29) + 5):
        print(f"[case] adamw long list with {large} elements", flush=True)

        def make():
            lists = problem(torch, optim, [1 + 53 * k % 2900 for k in range(110)], "bf16", 8, 4)[:4]
            lists[0][70] = torch.full((large,), 1.0, dtype=torch.bfloat16, device="cuda")
            lists[1][70] = torch.full((large,), 0.5, dtype=torch.bfloat16, device="cuda")
            lists[1][70][-3:] = 2.0
            lists[2][70] = optim.moments(lists[0][70], 8)
            return lists

        same_as_one_by_one(torch, optim, make)
        torch.cuda.empty_cache()


@pytest.mark.parametrize("span", [60, 66])
def test_lists_far_apart(env, span):
    """Tensors up to `span` GiB from each other, inside and outside what 32 bits of 16 bytes reach."""
    torch, optim = env
    if torch.cuda.mem_get_info()[0] < 90e9:
        pytest.skip("not enough free memory")
    size = (span << 30) + (5 << 30)
    room = torch.empty(size, dtype=torch.uint8, device="cuda")
    count, n = 130, 1000
    rng = np.random.RandomState(9)
    values = [torch.from_numpy((0.1 * rng.randn(4, n)).astype(np.float32)) for _ in range(count)]

    def make():
        lists = [[], [], [], []]
        for k in range(count):
            for j in range(4):
                at = ((span << 30) * (k % 7) // 6 + 16384 * (k + 200 * j)) // 16 * 16
                t = room[at:at + 4 * n].view(torch.float32)
                t.copy_(values[k][j].abs() if j == 3 else values[k][j])
                lists[j].append(t)
        return lists[0], lists[1], list(zip(lists[2], lists[3])), None

    print(f"[case] adamw list over {span} GB", flush=True)
    same_as_one_by_one(torch, optim, make)


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_follow_each_other(env, bits):
    """Fifty steps towards a minimum, first from zero moments: within the 8-bit
    moments' own error (one step in 16 of each update) of the steps in 64 bits."""
    torch, optim = env
    rng = np.random.RandomState(4)
    n = 5000
    goal = torch.from_numpy(rng.randn(n)).cuda()
    p = torch.zeros(n, device="cuda")
    state = optim.moments(p, bits)
    w = np.zeros(n)
    m, v = np.zeros(n), np.zeros(n)
    goal64 = goal.cpu().numpy()
    for step in range(1, 51):
        optim.adamw_step([p], [(p - goal).float()], [state], step, lr=LR, betas=BETAS, eps=EPS, weight_decay=0.0)
        w, m, v, _ = R.adamw(w, w - goal64, m, v, step, LR, BETAS, EPS, 0.0)
    err = np.abs(p.double().cpu().numpy() - w).max()
    assert err <= (2e-5 if bits == 32 else 50 * LR * 2 / 16), err
    assert np.abs(w - goal64).mean() < np.abs(goal64).mean()


def test_complex_parameters(env):
    torch, optim = env
    rng = np.random.RandomState(6)
    p = torch.from_numpy((rng.randn(3, 70) + 1j * rng.randn(3, 70)).astype(np.complex64)).cuda()
    g = torch.from_numpy((rng.randn(3, 70) + 1j * rng.randn(3, 70)).astype(np.complex64)).cuda()
    state = optim.moments(p, 32)
    real = torch.view_as_real(p).reshape(-1).clone()
    state2 = optim.moments(real, 32)
    optim.adamw_step([p], [g], [state], 1)
    optim.adamw_step([real], [torch.view_as_real(g).reshape(-1)], [state2], 1)
    assert torch.equal(torch.view_as_real(p).reshape(-1), real) and torch.equal(state[1], state2[1])


@pytest.mark.parametrize("bits", [32, 8])
def test_scale_that_is_not_finite_leaves_everything(env, bits):
    torch, optim = env
    for bad in (float("nan"), float("inf")):
        params, grads, moments, masters, _ = problem(torch, optim, [700, 5], "master", bits, 3)
        before = [t.clone() for t in (*params, *masters, *(x.view(torch.uint8) for s in moments for x in s))]
        optim.adamw_step(params, grads, moments, 1, masters=masters, grad_scale=torch.tensor([bad], device="cuda"))
        after = [*params, *masters, *(x.view(torch.uint8) for s in moments for x in s)]
        assert all(torch.equal(a, b) for a, b in zip(before, after))


def test_not_a_number_stays_in_its_element(env):
    """8-bit moments: one NaN gradient spoils its element, not its block."""
    torch, optim = env
    params, grads, moments, _, ref = problem(torch, optim, [600], "f32", 8, 5)
    grads[0][300] = float("nan")
    optim.adamw_step(params, grads, moments, 2, lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY)
    bad = torch.isnan(params[0]).cpu().numpy()
    assert bad[300] and bad.sum() == 1
    for k in range(2):
        code = torch.isnan(moments[0][k].float()).cpu().numpy()
        assert code[300] and code.sum() == 1 and torch.isfinite(moments[0][2 + k]).all()


def test_moments_keep_their_decay(env):
    """With zero gradients the blocks' scales follow the decay, whatever the codes' spacing."""
    torch, optim = env
    params, grads, moments, _, _ = problem(torch, optim, [1024], "f32", 8, 8)
    grads[0].zero_()
    first = [moments[0][2 + k].double().cpu().numpy() for k in range(2)]
    for step in range(1, 21):
        optim.adamw_step(params, grads, moments, step, lr=0.0)
    for k, factor in ((0, 0.9 ** 20), (1, 0.999 ** 10)):
        now = moments[0][2 + k].double().cpu().numpy()
        assert np.all(np.abs(now - first[k] * factor) <= 20 * 8 * R.EPS * first[k])


@pytest.mark.parametrize("kinds", ["float32", "bfloat16", "mixed"])
def test_grad_norm(env, kinds):
    torch, optim = env
    rng = np.random.RandomState(7)
    grads = []
    for k, n in enumerate([*SIZES, 100003, *rng.randint(1, 3000, 90)]):
        dt = torch.bfloat16 if kinds == "bfloat16" or (kinds == "mixed" and k % 2) else torch.float32
        grads.append(cut(torch, (0.1 * rng.randn(n)).astype(np.float32), dt, k % 2))
    print(f"[case] grad_norm {kinds}", flush=True)
    want = np.sqrt(sum(float(g.double().square().sum()) for g in grads))
    # squares and the sums of up to 64 of them in 32 bits, the rest in 64
    tol = 40 * R.EPS
    norm, scale = optim.grad_norm(grads).tolist()
    assert norm == pytest.approx(want, rel=tol) and scale == 1.0
    for most in (0.5 * want, 2 * want):
        r = optim.grad_norm(grads, max_norm=most)
        assert r[0].item() == pytest.approx(want, rel=tol) and r[1].item() == pytest.approx(min(1, most / want), rel=2 * tol)
    assert torch.equal(optim.grad_norm(grads, max_norm=1.0), optim.grad_norm(grads, max_norm=1.0))
    grads[3][0] = float("inf")
    r = optim.grad_norm(grads, max_norm=1.0)
    assert r[0].item() == float("inf") and r[1].item() == 0.0
    grads[3][0] = float("nan")
    r = optim.grad_norm(grads, max_norm=1.0)
    assert torch.isnan(r).all()
    assert optim.grad_norm([torch.zeros(0, device="cuda")], max_norm=1.0).tolist() == [0.0, 1.0]


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_past_32_bit_offsets(env, bits):
    torch, optim = env
    n = (1 << 31) + 300
    print(f"[case] adamw {n} elements {bits} bits", flush=True)
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    state = optim.moments(p, bits)
    tail = slice(n - 300, n)
    p[tail] = 1.0
    g[tail] = 0.5
    optim.adamw_step([p], [g], [state], 1, lr=0.25, weight_decay=0.0)
    assert (p[tail] == 0.75).all() and not p[:1000].any() and not p[n - 1300:n - 300].any()
    assert optim.grad_norm([g])[0].item() == pytest.approx(np.sqrt(300 * 0.25), rel=1e-6)


def test_another_stream(env):
    torch, optim = env
    side = torch.cuda.Stream()
    a = problem(torch, optim, [70001, 257], "f32", 8, 9)
    b = problem(torch, optim, [70001, 257], "f32", 8, 9)
    torch.cuda.synchronize()
    for one, stream in ((a, side), (b, torch.cuda.current_stream())):
        with torch.cuda.stream(stream):
            for step in (1, 2, 3):
                clip = optim.grad_norm(one[1], max_norm=0.1)
                optim.adamw_step(one[0], one[1], one[2], step, grad_scale=clip[1:])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a[0], b[0]))


def test_wrong_arguments_on_the_gpu(env):
    """What the native part of the binding does not take is refused as on the CPU,
    and leaves every tensor as it is."""
    torch, optim = env
    p, g = torch.ones(300, device="cuda"), torch.ones(300, device="cuda")
    s32, s8 = optim.moments(p, 32), optim.moments(p, 8)
    half = p.bfloat16()
    for args, kw in ((([p], [g.cpu()], [s32]), {}), (([p], [g[:-1]], [s32]), {}), (([p], [None], [s32]), {}),
                     (([p], [g[:1].expand(300)], [s32]), {}), (([p], [g], [s32[:1]]), {}), (([p], [g], [(s32[0], s8[1])]), {}),
                     (([p], [g], [(*s8[:3], s8[3][:1])]), {}), (([p, p], [g], [s32]), {}), (([p], [g], [s32]), dict(lr=[1.0, 2.0])),
                     (([p], [g], [s32]), dict(masters=[p])), (([half], [g], [s32]), dict(masters=[half])),
                     (([p], [g], [s32]), dict(grad_scale=torch.ones(2, device="cuda"))),
                     (([p], [g], [s32]), dict(grad_scale=torch.ones(1))), (([p.double()], [g], [s32]), {})):
        with pytest.raises(ValueError):
            optim.adamw_step(*args, 1, **kw)
    from paper_1511_05946_amd.acdc import ACDCError
    for kw in (dict(betas=(1.0, 0.999)), dict(eps=-1.0), dict(lr=float("nan"))):
        with pytest.raises(ACDCError, match="invalid argument"):
            optim.adamw_step([p], [g], [s32], 1, **kw)
    with pytest.raises(ACDCError, match="invalid argument"):
        optim.adamw_step([p], [g], [s32], 0)
    assert (p == 1).all() and not s32[0].any()
    for bad in ([g.cpu(), g], [g, g.cpu()], [g[::2]], [g.half()]):
        with pytest.raises(ValueError):
            optim.grad_norm(bad, max_norm=1.0)
    with pytest.raises(ValueError):
        optim.grad_norm([g], max_norm=-1.0)


def test_numbers_of_other_types(env):
    """Steps and rates as numpy numbers, moments and tensors as tuples."""
    torch, optim = env
    a, b = (problem(torch, optim, [700, 33], "f32", 8, 12) for _ in range(2))
    optim.adamw_step(a[0], a[1], a[2], 4, lr=0.01, weight_decay=0.1)
    optim.adamw_step(tuple(b[0]), tuple(b[1]), [list(m) for m in b[2]], np.int64(4), lr=[np.float64(0.01), 0.01],
                     betas=[0.9, 0.999], weight_decay=(0.1, np.float32(0.1)))
    assert all(torch.allclose(x, y, rtol=1e-6) for x, y in zip(a[0], b[0]))


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_of_every_size(env, bits):
    """Second moments from denormal numbers to 1e36 in one block and in blocks of
    their own: nothing becomes NaN, and every moment keeps its size."""
    torch, optim = env
    sizes = [1e-22, 3e-21, 1e-15, 1e-8, 1.0, 1e9, 1e18]
    g = np.concatenate([np.full(256, x) for x in sizes] + [np.tile(sizes, 40)]).astype(np.float32)
    n = len(g)
    p, gt = torch.ones(n, device="cuda"), torch.from_numpy(g).cuda()
    state = optim.moments(p, bits)
    optim.adamw_step([p], [gt], [state], 1, lr=LR, betas=BETAS, eps=EPS, weight_decay=0.0)
    w, m, v, move = R.adamw(np.ones(n), g.astype(float), np.zeros(n), np.zeros(n), 1, LR, BETAS, EPS, 0.0)
    # v is rounded to a multiple of 2^-149 where it is that small: sqrt(v) by up to 2^-74.5, eps being 1e-8
    assert np.all(np.abs(p.double().cpu().numpy() - w) <= 4 * R.EPS + 20 * R.EPS * move)
    for k, x in enumerate((m, np.sqrt(v))):
        got = state[k].double().cpu().numpy()
        if bits == 32:
            want = x if k == 0 else v
            assert np.all(np.abs(got - want) <= 4 * R.EPS * want + 2.0 ** -149)
            continue
        each = np.repeat(state[2 + k].double().cpu().numpy(), R.BLOCK)[:n]
        top = np.repeat(R.block_scale(x), R.BLOCK)[:n] * R.TOP
        off = np.abs(got * each - x)
        # half a step of the code, or of the smallest one, and the rounding of denormal v
        bound = np.maximum(x / 16, each * R.TINY / 2) * (1 + 1e-5) + (0.0 if k == 0 else 2.0 ** -74)
        bound = np.where(top < 2.0 ** -99, top, bound)   # blocks below 2^-100 are 0
        if k == 1:
            off = np.where(x < each * R.TINY, 0.0, off)   # positive ones never are, unless all are
        assert np.all(off <= bound), (k, np.argmax(off - bound))
