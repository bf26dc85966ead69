"""The gated delta rule on the GPU against its recurrence in float64."""
import math
import sys

import pytest

import delta_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def sata():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    import paper_2602_00294_amd as m
    m.load_library()
    return m


def _cuda(*xs):
    return [x.cuda() if x is not None else None for x in xs]


def state_tol(n, dk):
    """Relative, of a state's norm.  A token multiplies a state by matrices of norm at most 1 (keys of length one, beta
    below 1), so errors do not grow; each adds roundings of 2^-24 of a state's entries, two or
    three of them, and products over d_k entries.  They are of both signs: they add up as a root, and four times
    that covers the extremes and the products of a chunk's triangular inverse."""
    return 4 * 2.0 ** -24 * (math.sqrt(3 * n) + math.sqrt(dk))


def check_rows(y, want, q, states, dk, dtype, extra):
    """Every row of every head: its rounding, and c |q| |S_t|, the size of the sum that it is, at 16 bits (bfloat16) or
    at the state's own error.  extra: the state's relative error."""
    B, H, n, dv = want.shape
    G = H // q.shape[1]
    qa = q.double().cpu().abs().repeat_interleave(G, dim=1)
    eps, bits = (2.0 ** -8, 2.0 ** -16) if dtype == "bf16" else (2.0 ** -24, 2.0 ** -22)
    for t in range(n):
        size = (qa[:, :, t, :, None] * states[t].abs()).sum(-2) / math.sqrt(dk)
        norm = qa[:, :, t].norm(dim=-1) * states[t].flatten(2).norm(dim=-1) / math.sqrt(dk)
        off = (y[:, :, t].double().cpu() - want[:, :, t]).norm(dim=-1)
        tol = eps * want[:, :, t].norm(dim=-1) + bits * size.norm(dim=-1) + extra * norm
        assert (off <= tol + 1e-300).all(), (t, (off / tol).max())


PROMPTS = [  # B, Hk, G, n, dk, dv, dtype, lengths, state
    (1, 1, 1, 1, 16, 16, "f32", None, False),
    (2, 2, 1, 70, 64, 64, "bf16", None, True),
    (2, 1, 3, 97, 40, 24, "f32", [97, 30], True),
    (1, 2, 2, 64, 128, 128, "bf16", None, True),
    (1, 1, 2, 33, 128, 128, "f32", None, False),
    (3, 1, 1, 50, 1, 3, "f32", [0, 1, 50], True),
    (2, 1, 1, 65, 33, 65, "bf16", [64, 65], False),
    (1, 3, 1, 31, 96, 100, "bf16", None, True),
    (2, 1, 2, 200, 17, 128, "f32", [200, 160], False),
    (1, 1, 1, 300, 128, 7, "bf16", None, True),
]


@pytest.mark.parametrize("case", PROMPTS, ids=str)
def test_prompt(sata, case):
    B, Hk, G, n, dk, dv, dtype, lengths, state = case
    print("prompt", case, file=sys.stderr, flush=True)
    q, k, v, g, beta, S0 = ref.draw(n + dk, B, Hk, G, n, dk, dv, dtype, state=state)
    L = torch.tensor(lengths, dtype=torch.int32) if lengths else None
    want, S, states = ref.delta(*ref.to64(q, k, v, g, beta), L, *ref.to64(S0))
    if lengths:  # (padding is not used, whatever it holds)
        for b, e in enumerate(lengths):
            for x in (q, k, v, g, beta):
                x[b, :, e:] = math.nan
    y, got = sata.delta_prefill(*_cuda(q, k, v, g, beta), lengths=L.cuda() if lengths else None, S_in=_cuda(S0)[0])
    tol = state_tol(n, dk)
    off = (got.double().cpu() - S).flatten(2).norm(dim=-1)
    assert (off <= tol * S.flatten(2).norm(dim=-1) + 1e-300).all(), (off / S.flatten(2).norm(dim=-1)).max() / tol
    q = torch.nan_to_num(q.float())
    check_rows(y, want, q, states, dk, dtype, tol)


def test_prompt_in_pieces_and_tokens(sata):
    """A prompt, one that goes on from its state, then tokens: the whole sequence."""
    B, Hk, G, n, dk, dv = 2, 2, 2, 140, 64, 48
    q, k, v, g, beta, _ = ref.draw(11, B, Hk, G, n, dk, dv, "f32")
    want, S, states = ref.delta(*ref.to64(q, k, v, g, beta))
    cut = lambda a, b: _cuda(*(x[:, :, a:b].contiguous() for x in (q, k, v, g, beta)))  # noqa: E731
    y1, S1 = sata.delta_prefill(*cut(0, 75))
    y2, S2 = sata.delta_prefill(*cut(75, 130), S_in=S1)
    ys = [y1, y2]
    for t in range(130, n):
        ys.append(sata.delta_step(S2, *(x[:, :, 0].contiguous() for x in cut(t, t + 1)))[:, :, None])
    tol = state_tol(n, dk)
    assert ((S2.double().cpu() - S).flatten(2).norm(dim=-1) <= tol * S.flatten(2).norm(dim=-1)).all()
    check_rows(torch.cat(ys, 2), want, q, states, dk, "f32", tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hk,G,dk,dv", [(2, 3, 1, 64, 64), (1, 1, 4, 128, 128), (3, 2, 2, 5, 3), (1, 1, 1, 128, 1),
                                          (2, 1, 2, 1, 128), (1, 2, 1, 100, 36), (1, 2, 1, 33, 130 - 2)])
def test_token(sata, B, Hk, G, dk, dv, dtype):
    print("token", B, Hk, G, dk, dv, dtype, file=sys.stderr, flush=True)
    q, k, v, g, beta, S0 = ref.draw(dk + dv, B, Hk, G, 1, dk, dv, dtype, state=True)
    want, S, states = ref.delta(*ref.to64(q, k, v, g, beta), None, S0.double())
    got = S0.cuda()
    y = sata.delta_step(got, *_cuda(*(x[:, :, 0].contiguous() for x in (q, k, v, g, beta))))
    # (two products over d_k entries, in float32)
    tol = 2.0 ** -24 * (4 + 2 * math.sqrt(dk))
    assert ((got.double().cpu() - S).flatten(2).norm(dim=-1) <= tol * S.flatten(2).norm(dim=-1)).all()
    check_rows(y[:, :, None], want, q, states, dk, dtype, tol)


def test_unaligned_state_token(sata):
    q, k, v, g, beta, S0 = ref.draw(5, 1, 2, 1, 1, 16, 8, "f32", state=True)
    args = _cuda(*(x[:, :, 0].contiguous() for x in (q, k, v, g, beta)))
    buf = torch.zeros(S0.numel() + 1, device="cuda")
    S = buf[1:].view(S0.shape)
    S.copy_(S0)
    T = S0.cuda()
    assert (sata.delta_step(S, *args) - sata.delta_step(T, *args)).abs().max() <= 16 * 2.0 ** -24 * 4
    assert (S - T).abs().max() <= 16 * 2.0 ** -24 * 8 and buf[0] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rates_and_decays_at_their_ends(sata, dtype):
    """beta 0 leaves the state alone but for its decay, beta 1 with a key of length one replaces what it held; a decay of
    minus infinity forgets all before its token, one below float32's range too; none at all keeps everything."""
    n, d = 80, 32
    q, k, v, g, beta, S0 = ref.draw(21, 1, 1, 1, n, d, d, dtype, state=True)
    beta[..., ::3], beta[..., 1::7] = 0.0, 1.0
    g[...] = 0.0
    g[..., 10], g[..., 40], g[..., 41], g[..., 70] = -math.inf, -150.0, -1e-3, -1e30
    g[..., 45:50] = -30.0
    g64 = g.double().clamp(min=-1000.0)
    want, S, states = ref.delta(*ref.to64(q, k, v), g64, beta.double(), None, S0.double())
    y, got = sata.delta_prefill(*_cuda(q, k, v, g, beta), S_in=S0.cuda())
    tol = state_tol(n, d)
    assert ((got.double().cpu() - S).norm() <= tol * S.norm())
    check_rows(y, want, q, states, d, dtype, tol)
    T = S0.cuda()
    for t in range(n):
        yt = sata.delta_step(T, *_cuda(*(x[:, :, t].contiguous() for x in (q, k, v, g, beta))))
        check_rows(yt[:, :, None], want[:, :, t:t + 1], q[:, :, t:t + 1], states[t:t + 1], d, dtype, tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["q", "k", "v", "g", "beta"])
def test_not_finite(sata, what, dtype):
    """Earlier tokens, other columns (v), other heads and sequences do not feel it; what does is not finite."""
    B, Hk, G, n, d, at = 2, 2, 2, 75, 40, 37
    x = dict(zip(("q", "k", "v", "g", "beta"), ref.draw(31, B, Hk, G, n, d, d, dtype)))
    clean, Sc = sata.delta_prefill(*_cuda(*x.values()))
    hit = torch.zeros(B, Hk * G, n, d, dtype=torch.bool)
    hitS = torch.zeros(B, Hk * G, d, d, dtype=torch.bool)
    bad = math.nan
    if what == "q":
        x["q"][1, 0, at, 5] = bad
        hit[1, :G, at] = True
    elif what == "k":
        x["k"][1, 0, at, 5] = bad
        hit[1, :G, at:] = True
        hitS[1, :G] = True
    elif what == "v":
        x["v"][1, 2, at, 7] = math.inf if dtype == "f32" else bad
        hit[1, 2, at:, 7] = True
        hitS[1, 2, :, 7] = True
    else:
        x[what][0, 3, at] = bad
        hit[0, 3, at:] = True
        hitS[0, 3] = True
    y, S = sata.delta_prefill(*_cuda(*x.values()))
    tol = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -18  # (chunks may be cut elsewhere)
    for got, was, h in ((y, clean, hit), (S, Sc, hitS)):
        got, was = got.float().cpu(), was.float().cpu()
        assert torch.equal(~torch.isfinite(got), h)
        t = tol if got is not S else 2.0 ** -18
        assert (got - was)[~h].norm() <= t * was[~h].norm()


def test_large_values(sata):
    """Values near float32's ends, of small weight: nothing overflows that the recurrence does not."""
    n, d = 50, 16
    q, k, v, g, beta, _ = ref.draw(41, 1, 1, 1, n, d, d, "f32")
    v[0, 0, 20] *= 1e36
    v[0, 0, 30] = 0.0
    want, S, states = ref.delta(*ref.to64(q, k, v, g, beta))
    y, got = sata.delta_prefill(*_cuda(q, k, v, g, beta))
    assert torch.isfinite(y).all() and torch.isfinite(got).all()
    assert (got.double().cpu() - S).norm() <= state_tol(n, d) * S.norm()
    # (tokens before the large one are as exact as without it)
    check_rows(y[:, :, :20], want[:, :, :20], q, states[:20], d, "f32", state_tol(n, d))


def test_lengths_out_of_range_and_empty_prompts(sata):
    q, k, v, g, beta, S0 = ref.draw(51, 2, 1, 1, 8, 16, 16, "f32", state=True)
    L = torch.tensor([-3, 100], dtype=torch.int32)
    y, S = sata.delta_prefill(*_cuda(q, k, v, g, beta), lengths=L.cuda(), S_in=S0.cuda())
    want, Sw, _ = ref.delta(*ref.to64(q, k, v, g, beta), torch.tensor([0, 8]), S0.double())
    assert (y[0] == 0).all() and torch.equal(S[0].cpu(), S0[0])
    assert (S.double().cpu() - Sw).norm() <= state_tol(8, 16) * Sw.norm()
    e = [x[:, :, :0].contiguous().cuda() for x in (q, k, v, g, beta)]
    y, S = sata.delta_prefill(*e, S_in=S0.cuda())
    assert y.shape == (2, 1, 0, 16) and torch.equal(S.cpu(), S0)
    assert (sata.delta_prefill(*e)[1] == 0).all()
    assert sata.delta_prefill(*e, want_state=False)[1] is None


def test_rows_behind_are_zero_and_results_the_same_twice(sata):
    q, k, v, g, beta, _ = ref.draw(61, 2, 2, 2, 150, 64, 64, "bf16")
    L = torch.tensor([7, 150], dtype=torch.int32).cuda()
    y = torch.full((2, 4, 150, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    args = _cuda(q, k, v, g, beta)
    a, S = sata.delta_prefill(*args, lengths=L, y=y)
    assert a is y and (y[0, :, 7:] == 0).all()
    b, T = sata.delta_prefill(*args, lengths=L)
    assert torch.equal(a, b) and torch.equal(S, T)


def test_captured(sata):
    """A graph of a prompt and of a token, replayed on new inputs between eager calls."""
    q, k, v, g, beta, S0 = _cuda(*ref.draw(71, 1, 2, 2, 100, 64, 64, "bf16", state=True))
    tok = [x[:, :, 0].contiguous() for x in (q, k, v, g, beta)]
    S, y = torch.empty_like(S0), torch.empty_like(v)
    yt = torch.empty_like(tok[2])
    run = lambda: (sata.delta_prefill(q, k, v, g, beta, S_in=S0, y=y, S=S), sata.delta_step(S, *tok, y=yt))  # noqa: E731
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        v.mul_(0.5)
        tok[2].add_(0.25)
        graph.replay()
        y2, S2 = sata.delta_prefill(q, k, v, g, beta, S_in=S0)
        yt2 = sata.delta_step(S2, *tok)
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(S, S2) and torch.equal(yt, yt2)


def test_refusals(sata):
    q, k, v, g, beta, S0 = _cuda(*ref.draw(81, 1, 2, 2, 5, 16, 16, "f32", state=True))
    with pytest.raises(sata.SataError):
        sata.delta_prefill(q, k, v, g, beta, S_in=S0, S=S0)
    with pytest.raises(ValueError):
        sata.delta_prefill(q, k, v[:, :3].contiguous(), g, beta)
    with pytest.raises(ValueError):
        sata.delta_prefill(q, k, v, g[:, :2].contiguous(), beta)
    with pytest.raises(TypeError):
        sata.delta_prefill(q, k, v, g.double(), beta)
    with pytest.raises(TypeError):
        sata.delta_prefill(q.half(), k.half(), v.half(), g, beta)
    with pytest.raises(ValueError):
        sata.delta_prefill(q, k[:, :1].contiguous(), v, g, beta)
    with pytest.raises(ValueError):
        sata.delta_step(S0.transpose(-1, -2), q[:, :, 0].contiguous(), k[:, :, 0].contiguous(), v[:, :, 0].contiguous(),
                        g[:, :, 0].contiguous(), beta[:, :, 0].contiguous())
    wide = torch.zeros(1, 1, 2, 129, device="cuda")
    with pytest.raises(sata.SataError):
        sata.delta_prefill(wide, wide, wide, torch.zeros(1, 1, 2, device="cuda"), torch.zeros(1, 1, 2, device="cuda"))


# ------------------------------------------------------------------ gradients

GRADIENTS = [  # B, Hk, G, n, dk, dv, dtype, lengths, state
    (1, 1, 1, 1, 16, 16, "f32", None, False),
    (1, 1, 1, 33, 32, 32, "f32", None, True),
    (2, 2, 1, 64, 64, 64, "bf16", None, True),
    (2, 1, 3, 97, 40, 24, "f32", [97, 30], True),
    (1, 2, 2, 65, 128, 128, "bf16", None, True),
    (1, 1, 2, 130, 128, 128, "f32", None, False),
    (3, 1, 1, 50, 1, 3, "f32", [0, 1, 50], True),
    (2, 1, 1, 129, 33, 65, "bf16", [128, 64], False),
    (1, 3, 1, 31, 96, 100, "bf16", None, True),
    (2, 1, 2, 200, 17, 128, "f32", [200, 160], False),
    (1, 1, 1, 150, 128, 7, "bf16", None, True),
    (1, 1, 4, 70, 64, 96, "f32", [69], True),
]


def gradient_reference(q, k, v, g, beta, dy, L, S0, dS):
    """The gradients in float64, and for every token the sizes of the sums that they are."""
    x = ref.to64(q, k, v, g, beta) + ([S0.double()] if S0 is not None else [])
    leaves = [a.clone().requires_grad_() for a in x]
    y, S, states = ref.delta(*leaves[:5], L, leaves[5] if S0 is not None else None)
    loss = (y * dy.double()).sum() + ((S * dS.double()).sum() if dS is not None else 0.0)
    out = torch.autograd.grad(loss, leaves + states, allow_unused=True)
    grads = [torch.zeros_like(l) if o is None else o for l, o in zip(leaves, out)]
    n, dk = q.shape[2], q.shape[3]
    zero = torch.zeros_like(states[0])
    norm = lambda a: a.detach().flatten(2).norm(dim=-1)  # noqa: E731
    U = torch.stack([norm(zero if o is None else o) for o in out[len(leaves):]], -1)   # [B, H, n]
    before = torch.stack([norm(s) for s in states], -1)
    first = norm(leaves[5]) if S0 is not None else torch.zeros_like(before[..., 0])
    before = torch.maximum(before, torch.cat((first[..., None], before[..., :-1]), -1))
    values, rate = x[2].norm(dim=-1), x[4]
    size = {"dq": before * dy.double().norm(dim=-1) / math.sqrt(dk), "dv": U * rate, "dbeta": U * (values + before),
            "dk": 2 * U * rate * (values + before), "dg": U * before}
    return grads, size


def check_gradients(got, want, size, n, dk, dv, dtype, G):
    """Each row's error against its rounding and, as states and gradients of states carry their own error
    (state_tol) into every sum, twice that of the sum's size; a chunk's inverse and the sums over a block's tokens
    double it again."""
    eps = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    off = 4 * state_tol(n, max(dk, dv))
    for i, name in enumerate(("dq", "dk", "dv", "dg", "dbeta")):
        w, s = want[i], size[name]
        a = got[i].double().cpu()
        assert a.shape == w.shape
        if name in ("dq", "dk"):
            s = s.reshape(s.shape[0], -1, G, s.shape[-1]).sum(2)
        err, mag = ((a - w).norm(dim=-1), w.norm(dim=-1)) if w.dim() == 4 else ((a - w).abs(), w.abs())
        tol = (eps if w.dim() == 4 else 2.0 ** -24) * mag + off * s.amax(-1, keepdim=True) * (1 if name == "dg" else 0) + off * s
        assert (err <= tol + 1e-300).all(), (name, (err / (tol + 1e-300)).max())
    if len(want) > 5:
        S = want[5]
        err = (got[5].double().cpu() - S).flatten(2).norm(dim=-1)
        assert (err <= off * S.flatten(2).norm(dim=-1) + off * size["dv"].amax(-1) + 1e-300).all()


@pytest.mark.parametrize("case", GRADIENTS, ids=str)
def test_gradients(sata, case):
    B, Hk, G, n, dk, dv, dtype, lengths, state = case
    print("gradients", case, file=sys.stderr, flush=True)
    q, k, v, g, beta, S0 = ref.draw(n + dk + 1, B, Hk, G, n, dk, dv, dtype, state=state)
    gen = torch.Generator().manual_seed(n)
    dy = torch.randn(B, Hk * G, n, dv, generator=gen).to(q.dtype)
    dS = torch.randn(B, Hk * G, dk, dv, generator=gen) if state else None
    L = torch.tensor(lengths, dtype=torch.int32) if lengths else None
    if lengths:
        for b, e in enumerate(lengths):
            dy[b, :, e:] = 0.0
    want, size = gradient_reference(q, k, v, g, beta, dy, L, S0, dS)
    if lengths:  # (padding is not used, whatever it holds)
        for b, e in enumerate(lengths):
            for x in (q, k, v, g, beta, dy):
                x[b, :, e:] = math.nan
    got = sata.delta_backward(*_cuda(q, k, v, g, beta, dy), lengths=_cuda(L)[0], S_in=_cuda(S0)[0], dS=_cuda(dS)[0])
    assert (got[5] is None) == (not state)
    check_gradients(got, want, size, n, dk, dv, dtype, G)
    if lengths:
        for b, e in enumerate(lengths):
            assert all((x[b, :, e:] == 0).all() for x in got[:5])


def test_gradients_of_a_state_alone(sata):
    """dS without an earlier state, and an earlier state without dS."""
    q, k, v, g, beta, S0 = ref.draw(91, 1, 2, 1, 40, 24, 16, "f32", state=True)
    gen = torch.Generator().manual_seed(92)
    dy, dS = torch.randn(1, 2, 40, 16, generator=gen), torch.randn(1, 2, 24, 16, generator=gen)
    for s, d in ((S0, None), (None, dS)):
        want, size = gradient_reference(q, k, v, g, beta, dy, None, s, d)
        got = sata.delta_backward(*_cuda(q, k, v, g, beta, dy), S_in=_cuda(s)[0], dS=_cuda(d)[0])
        check_gradients(got, want, size, 40, 24, 16, "f32", 1)


def test_gradients_at_rates_of_zero_and_strong_decays(sata):
    """beta 0 has a gradient of its own; a decay of minus infinity cuts the sequence in two."""
    n, d = 100, 32
    q, k, v, g, beta, S0 = ref.draw(93, 1, 1, 1, n, d, d, "f32", state=True)
    beta[..., ::3], beta[..., 1::7] = 0.0, 1.0
    g[..., 10], g[..., 40], g[..., 70] = -300.0, -150.0, -1e30
    g[..., 45:50] = -30.0
    gen = torch.Generator().manual_seed(94)
    dy, dS = torch.randn(1, 1, n, d, generator=gen), torch.randn(1, 1, d, d, generator=gen)
    want, size = gradient_reference(q, k, v, g.clamp(min=-1000.0), beta, dy, None, S0, dS)
    g[..., 70] = -math.inf
    got = sata.delta_backward(*_cuda(q, k, v, g, beta, dy), S_in=S0.cuda(), dS=dS.cuda())
    check_gradients(got, want, size, n, d, d, "f32", 1)


def test_gradients_by_differences(sata):
    """The forward call's own slope along random directions, in float32: differences over a step of 2^-6 lose
    14 bits to it and as many to the third derivative's share; 2^-9 of the gradients' sizes are left."""
    x = list(ref.draw(95, 1, 1, 2, 45, 16, 12, "f32", state=True))
    gen = torch.Generator().manual_seed(96)
    w, wS = torch.randn(1, 2, 45, 12, generator=gen), torch.randn(1, 2, 16, 12, generator=gen)
    grads = sata.delta_backward(*_cuda(*x[:5], w), S_in=x[5].cuda(), dS=wS.cuda())

    def loss(*a):
        y, S = sata.delta_prefill(*_cuda(*a[:5]), S_in=a[5].cuda())
        return (y.cpu().double() * w).sum() + (S.cpu().double() * wS).sum()

    h = 2.0 ** -6
    for i, grad in enumerate(grads):
        e = torch.randn(x[i].shape, generator=gen)
        e = e / e.norm()
        at = lambda s: loss(*(a + s * e if j == i else a for j, a in enumerate(x)))  # noqa: E731
        slope = (at(h) - at(-h)) / (2 * h)
        # (the losses are sums of some 700 terms, of float32's error each)
        assert abs(slope - (grad.cpu().double() * e).sum()) <= 2.0 ** -9 * grad.double().norm().item() + 2.0 ** -24 * 700 / h, i


def test_gradients_of_bad_values_stay_in_their_sequence_and_head(sata):
    q, k, v, g, beta, _ = ref.draw(97, 2, 2, 2, 70, 32, 32, "bf16")
    dy = torch.randn(2, 4, 70, 32, generator=torch.Generator().manual_seed(98)).bfloat16()
    clean = sata.delta_backward(*_cuda(q, k, v, g, beta, dy))
    k[1, 0, 30, 3], v[0, 3, 11, 2], dy[0, 2, 69, 0] = math.nan, math.inf, math.nan
    got = sata.delta_backward(*_cuda(q, k, v, g, beta, dy))
    for i, (a, b) in enumerate(zip(got[:5], clean[:5])):
        # heads that hold none: of queries and keys (0, 0) and (1, 1), of values their two each
        for bb, h in (((0, 0), (1, 1)) if i < 2 else ((0, 0), (0, 1), (1, 2), (1, 3))):
            assert torch.equal(a[bb, h], b[bb, h])


def test_gradients_twice_and_captured(sata):
    q, k, v, g, beta, S0 = _cuda(*ref.draw(99, 2, 2, 2, 100, 64, 64, "bf16", state=True))
    dy, dS = torch.randn_like(v), torch.randn_like(S0)
    first = sata.delta_backward(q, k, v, g, beta, dy, S_in=S0, dS=dS)
    second = sata.delta_backward(q, k, v, g, beta, dy, S_in=S0, dS=dS)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = sata.delta_backward(q, k, v, g, beta, dy, S_in=S0, dS=dS)
    for _ in range(4):
        dy.mul_(0.5)
        graph.replay()
        want = sata.delta_backward(q, k, v, g, beta, dy, S_in=S0, dS=dS)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_gradients_of_empty_prompts(sata):
    q, k, v, g, beta, S0 = _cuda(*ref.draw(100, 2, 1, 2, 4, 16, 8, "f32", state=True))
    e = [x[:, :, :0].contiguous() for x in (q, k, v, g, beta)]
    dS = torch.randn_like(S0)
    out = sata.delta_backward(*e, torch.zeros_like(e[2]), S_in=S0, dS=dS)
    assert torch.equal(out[5], dS) and out[0].shape == (2, 1, 0, 16)
    L = torch.zeros(2, dtype=torch.int32, device="cuda")
    out = sata.delta_backward(q, k, v, g, beta, torch.ones_like(v), lengths=L, S_in=S0, dS=dS)
    assert torch.equal(out[5], dS) and all((x == 0).all() for x in out[:5])
    assert (sata.delta_backward(q, k, v, g, beta, torch.ones_like(v), lengths=L, S_in=S0)[5] == 0).all()
