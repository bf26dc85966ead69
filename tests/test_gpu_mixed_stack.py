"""A stack of three layers, decayed linear, exact softmax and Taylor attention, as
one would train and serve it: prompt, gradients through all three, then tokens
one by one, against the same stack in float64."""
import math
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

P = 5


@pytest.fixture(scope="module")
def sata():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    import paper_2602_00294_amd as m
    m.load_library()
    return m


def _taylor(q, k, v):
    """Causal attention with the first P terms of the exponential series (odd P: positive weights)."""
    s = q @ k.transpose(-1, -2) / math.sqrt(q.shape[-1])
    w = sum(s ** p / math.factorial(p) for p in range(P)).tril()
    return w @ v / w.sum(-1, keepdim=True)


def _reference(q, k, v, g):
    """The stack in float64 on the CPU: each layer's output is the next one's query and is added to its values."""
    n, d = q.shape[-2:]
    t = torch.arange(n, dtype=torch.float64)
    D = torch.where(t[:, None] >= t[None, :], torch.exp((t[:, None] - t[None, :]).clamp(min=0) * g[:, None, None]), 0.0)
    y1 = ((q @ k.transpose(-1, -2)) * D[None] / math.sqrt(d)) @ v
    s = (y1 @ k.transpose(-1, -2) / math.sqrt(d)).masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
    y2 = torch.softmax(s, -1) @ (v + y1)
    return y1, y2, _taylor(y2, k, v + y2)


def test_stack(sata):
    B, H, n, steps, d = 2, 3, 150, 5, 16
    print("mixed stack", file=sys.stderr, flush=True)
    gen = torch.Generator().manual_seed(1)
    q, k, v, dy = (torch.randn(B, H, n + steps, d, generator=gen) * 0.5 for _ in range(4))
    g = torch.tensor([-0.05, -0.5, -0.2])
    ref = _reference(*(x.double() for x in (q, k, v)), g.double())

    dev = lambda x: x[:, :, :n].contiguous().cuda()  # noqa: E731
    Q, K, V, DY, gd = dev(q), dev(k), dev(v), dev(dy), g.cuda()
    y1, S1 = sata.decay_prefill(Q, K, V, gd)
    v2 = V + y1
    y2, lse = sata.softmax_prefill(y1, K, v2)
    v3 = V + y2
    y3, S3 = sata.prefill(y2, K, v3, P)
    torch.cuda.synchronize()
    # the layers' roundings are relative 1e-6 and pass through scores and weights of order one;
    # Taylor prefills are held to 1e-4 in this library's parity tests
    for got, want in zip((y1, y2, y3), ref):
        assert (got.double().cpu() - want[:, :, :n]).norm() <= 1e-4 * want[:, :, :n].norm()

    # gradients: each layer's, chained by hand as a training program does
    dq3, dk3, dv3 = sata.backward(y2, K, v3, DY, P)
    dy2 = dq3 + dv3
    dq2, dk2, dv2 = sata.softmax_backward(y1, K, v2, y2, lse, dy2)
    dy1 = dq2 + dv2
    dq1, dk1, dv1, _ = sata.decay_backward(Q, K, V, gd, dy1)
    got = (dq1, dk1 + dk2 + dk3, dv1 + dv2 + dv3)
    leaves = [x[:, :, :n].double().requires_grad_() for x in (q, k, v)]
    want = torch.autograd.grad((_reference(*leaves, g.double())[2] * dy[:, :, :n].double()).sum(), leaves)
    torch.cuda.synchronize()
    for a, w in zip(got, want):
        assert (a.double().cpu() - w).norm() <= 3e-4 * w.norm()  # (three layers at 1e-4)

    # tokens: the decay layer from its state, softmax over a cache of n + steps rows, Taylor from its state
    cK, cV = torch.full((2, B, H, n + steps, d), math.nan, device="cuda")
    cK[:, :, :n], cV[:, :, :n] = K, v2
    at = torch.full((B,), n, dtype=torch.int32, device="cuda")
    for t in range(n, n + steps):
        x = [a[:, :, t].contiguous().cuda() for a in (q, k, v)]
        a1 = sata.decay_step(S1, *x, gd)
        a2 = sata.softmax_step(cK, cV, at, a1, x[1], x[2] + a1)
        a3 = sata.decode_step(S3, a2, x[1], x[2] + a2, P)
        at += 1
        for got, want in zip((a1, a2, a3), ref):
            w = want[:, :, t]
            assert (got.double().cpu() - w).norm() <= 1e-4 * w.norm()
    torch.cuda.synchronize()
