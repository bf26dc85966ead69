"""The gated delta rule over long sequences, and with keys that are much alike, on the GPU against float64."""
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
