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
