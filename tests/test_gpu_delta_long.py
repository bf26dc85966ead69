"""The gated delta rule over long sequences, and with keys that are much alike, on the GPU against float64."""
import math
import sys

import pytest

import delta_ref as ref
from test_gpu_delta import check_gradients, check_rows, gradient_reference, state_tol

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def sata():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    import paper_2602_00294_amd as m
    m.load_library()
    return m


def _inexact(low, high, tokens):
    """A log decay whose power over so many tokens float32 rounds by nearly half a step, always the same way."""
    g = torch.linspace(low, high, 20001, dtype=torch.float64).float()
    lam = torch.exp(g.double() * tokens)
    off = (lam.float().double() - lam) / lam
    return float(g[off.argmax()]), float(off.max())


def test_a_constant_decay_over_many_tokens(sata):
    """What no key reaches of a state only decays: exp(n g) of it is left, and of its gradient.  A block's factor is the
    same 2048 times over: rounded to float32 it would leave 2048 times its error."""
    n, dk, dv = 2048 * 64, 32, 16
    g0, off = _inexact(-2e-6, -1e-6, 64)
    assert off > 0.9 * 2.0 ** -25
    print("constant decay", n, g0, file=sys.stderr, flush=True)
    q, k, v, _, beta, S0 = ref.draw(1, 1, 1, 1, n, dk, dv, "f32", state=True)
    q[..., dk // 2:], k[..., dk // 2:] = 0.0, 0.0
    g = torch.full((1, 1, n), g0)
    args = [x.cuda() for x in (q, k, v, g, beta)]
    _, S = sata.delta_prefill(*args, S_in=S0.cuda())
    dy, dS = torch.zeros_like(v), torch.randn(S0.shape, generator=torch.Generator().manual_seed(2))
    back = sata.delta_backward(*args, dy.cuda(), S_in=S0.cuda(), dS=dS.cuda())[5]
    whole = math.exp(n * float(torch.tensor(g0)))
    for got, start in ((S, S0), (back, dS)):
        want = start[:, :, dk // 2:].double() * whole
        # (2048 products, each rounded to the nearest: their errors, of either sign, add up as a root; four times that)
        err = ((got[:, :, dk // 2:].double().cpu() - want) / want).abs().max()
        assert err <= 4 * 2.0 ** -24 * math.sqrt(2048), err / (2.0 ** -24 * math.sqrt(2048))


def test_a_constant_decay_beside_a_column_of_nan(sata):
    """The same where a column of values is NaN, whose neighbours go on token by token: factors of one token each."""
    n, dk, dv = 3000, 24, 20
    g0, off = _inexact(-2e-6, -1e-6, 1)
    assert off > 0.9 * 2.0 ** -25
    print("constant decay beside NaN", n, g0, file=sys.stderr, flush=True)
    q, k, v, _, beta, S0 = ref.draw(3, 1, 1, 1, n, dk, dv, "f32", state=True)
    q[..., dk // 2:], k[..., dk // 2:] = 0.0, 0.0
    v[0, 0, 0, 3] = math.nan
    g = torch.full((1, 1, n), g0)
    y, S = sata.delta_prefill(*(x.cuda() for x in (q, k, v, g, beta)), S_in=S0.cuda())
    others = [c for c in range(dv) if c != 3]
    assert torch.isnan(y[..., 3]).all() and torch.isnan(S[..., 3]).all() and torch.isfinite(y[..., others]).all()
    want = (S0[:, :, dk // 2:].double() * math.exp(n * float(torch.tensor(g0))))[..., others]
    got = S[:, :, dk // 2:].double().cpu()[..., others]
    err = ((got - want) / want).abs().max()
    # (A token's product is rounded by at most 2^-24.  These roundings are not of either sign: a token takes off some 12 to 25
    # units in the last place, a number whose fraction changes by 4e-5 a token, so for thousands of tokens all are rounded the
    # same way, and their errors add up to n of them at most.  A factor that is itself 2^-25 off would add half as much.)
    assert err <= n * 2.0 ** -24, err / (n * 2.0 ** -24)


def _alike(seed, B, H, G, n, dk, dv, dtype):
    """Keys that are nearly one another, with rates near 1: the pairs of a block are nearly all ones, what is right of
    their triangular inverse is small."""
    q, k, v, g, beta, S0 = ref.draw(seed, B, H, G, n, dk, dv, dtype, decay=1e-3, state=True)
    k = k.float() * 0.05 + torch.randn(B, H, 1, dk, generator=torch.Generator().manual_seed(seed + 1)) / math.sqrt(dk)
    k = (k / k.norm(dim=-1, keepdim=True) * (1 - 2.0 ** -8)).to(q.dtype)  # (rounded, none is longer than one)
    return q, k, v, g, 1.0 - 0.02 * beta, S0


SIZES = [(1, 1, 1, 2500, 64, 48, "f32"), (1, 1, 2, 2500, 128, 16, "bf16"), (2, 1, 1, 1100, 33, 20, "f32")]


@pytest.mark.parametrize("case", SIZES, ids=str)
@pytest.mark.parametrize("alike", [False, True])
def test_long_prompts(sata, alike, case):
    B, H, G, n, dk, dv, dtype = case
    print("long prompt", alike, case, file=sys.stderr, flush=True)
    draw = _alike if alike else lambda *a: ref.draw(*a, decay=1e-3, state=True)
    q, k, v, g, beta, S0 = draw(n, *case)
    want, S, states = ref.delta(*ref.to64(q, k, v, g, beta), None, S0.double())
    y, got = sata.delta_prefill(*(x.cuda() for x in (q, k, v, g, beta)), S_in=S0.cuda())
    tol = state_tol(n, dk)
    off = (got.double().cpu() - S).flatten(2).norm(dim=-1) / S.flatten(2).norm(dim=-1)
    assert (off <= tol).all(), off / tol
    check_rows(y, want, q.float(), states, dk, dtype, tol)


@pytest.mark.parametrize("case", [(1, 1, 1, 700, 64, 48, "f32"), (1, 1, 2, 700, 64, 64, "bf16"), (2, 1, 1, 333, 33, 20, "f32")], ids=str)
@pytest.mark.parametrize("alike", [False, True])
def test_long_gradients(sata, alike, case):
    B, H, G, n, dk, dv, dtype = case
    print("long gradients", alike, case, file=sys.stderr, flush=True)
    draw = _alike if alike else lambda *a: ref.draw(*a, decay=1e-3, state=True)
    q, k, v, g, beta, S0 = draw(n + 1, *case)
    gen = torch.Generator().manual_seed(n)
    dy, dS = torch.randn(v.shape, generator=gen).to(q.dtype), torch.randn(S0.shape, generator=gen)
    want, size = gradient_reference(q, k, v, g, beta, dy, None, S0, dS)
    got = sata.delta_backward(*(x.cuda() for x in (q, k, v, g, beta, dy)), S_in=S0.cuda(), dS=dS.cuda())
    check_gradients(got, want, size, n, dk, dv, dtype, G)
