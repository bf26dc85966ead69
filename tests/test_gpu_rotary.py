"""Rotary positions on the GPU against their definition in float64."""
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


def _bound(x, want, positions, freq, interleaved, scale):
    """Sine and cosine are off by at most 8.2 2^-24: what is left of an angle, below pi, by half a step (pi 2^-24) and the
    function by two units (2 2^-24), the scale and the product with it by half a step each; the sums by another
    each.  The angle itself, in turns, by 2^-51 of its size.  Then the output's rounding."""
    R = freq.numel()
    off = 10 * 2.0 ** -24 + 2 * math.pi * 2.0 ** -51 * positions.double().abs().max().item()
    size = torch.zeros_like(want)
    for i in range(R):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, R + i)
        size[..., a] = size[..., b] = abs(scale) * (x.double()[..., a].abs() + x.double()[..., b].abs())
    return off * size + torch.finfo(x.dtype).eps / 2 * want.abs()


CASES = [  # B, Hq, Hk, n, d, pairs, interleaved, dtype
    (2, 4, 2, 33, 64, 32, False, "bf16"),
    (1, 3, 1, 7, 64, 32, True, "f32"),
    (2, 5, 5, 19, 80, 30, False, "bf16"),
    (2, 2, 1, 130, 80, 30, True, "bf16"),
    (1, 1, 0, 5, 7, 3, False, "f32"),
    (1, 2, 1, 5, 7, 3, True, "bf16"),
    (3, 1, 2, 1, 128, 8, True, "bf16"),
    (1, 9, 4, 11, 128, 64, False, "f32"),
    (1, 2, 2, 3, 2, 1, False, "bf16"),
    (1, 17, 9, 300, 20, 10, False, "f32"),
    (1, 2, 2, 3, 22, 5, True, "f32"),
    (2, 40, 8, 700, 128, 64, False, "bf16"),
]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_against_definition(sata, case, back):
    B, Hq, Hk, n, d, pairs, inter, dtype = case
    print("rotary", case, back, file=sys.stderr, flush=True)
    gen = torch.Generator().manual_seed(n * d + Hq)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k = (torch.randn(B, h, n, d, generator=gen).to(dt) for h in (Hq, Hk))
    pos = torch.randint(-3000, 2 ** 21, (B, n), generator=gen, dtype=torch.int32)
    freq, _ = sata.rotary_frequencies(pairs, 10000.0, device="cpu")
    scale = 1.25
    f = sata.rotary_backward if back else sata.rotary
    got = f(q.cuda(), k.cuda() if Hk else None, pos.cuda(), freq.cuda(), interleaved=inter, scale=scale)
    for x, y in ((q, got[0]),) + (((k, got[1]),) if Hk else ()):
        want = ref.rotary(x.double(), pos, freq, inter, scale, back)
        err = (y.double().cpu() - want).abs()
        assert (err <= _bound(x, want, pos, freq, inter, scale)).all(), err.max()
        assert torch.equal(y.cpu()[..., 2 * pairs:], x[..., 2 * pairs:])
    if not Hk:
        assert got[1] is None


def test_far_positions(sata):
    """Positions up to the largest int32 keep their angles."""
    pos = torch.tensor([[2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 12345678]], dtype=torch.int32)
    q = torch.randn(1, 2, 4, 32, generator=torch.Generator().manual_seed(3))
    freq, _ = sata.rotary_frequencies(16, 500000.0, device="cpu")
    y, _ = sata.rotary(q.cuda(), None, pos.cuda(), freq.cuda())
    want = ref.rotary(q.double(), pos, freq, False, 1.0)
    assert ((y.double().cpu() - want).abs() <= _bound(q, want, pos, freq, False, 1.0)).all()


@pytest.mark.parametrize("inter", [False, True])
def test_in_place_tokens_and_back(sata, inter):
    """One token of every sequence, in place; turned forth and back is the square of the scale."""
    gen = torch.Generator().manual_seed(5)
    q, k = torch.randn(3, 4, 48, generator=gen), torch.randn(3, 2, 48, generator=gen)
    pos = torch.tensor([0, 7, 100000], dtype=torch.int32)
    freq, scale = sata.rotary_frequencies(20, 10000.0, "by_turns", 8.0, 4096.0, device="cuda")
    Q, K = q.cuda(), k.cuda()
    a, b = sata.rotary(Q, K, pos.cuda(), freq, interleaved=inter, scale=scale, q_out=Q, k_out=K)
    assert a is Q and b is K
    for x, y in ((q, Q), (k, K)):
        want = ref.rotary(x[:, :, None].double(), pos[:, None], freq.cpu(), inter, scale)[:, :, 0]
        assert ((y.double().cpu() - want).abs() <= _bound(x[:, :, None], want[:, :, None], pos, freq, inter, scale)[:, :, 0]).all()
    assert torch.equal(Q.cpu()[0, :, 40:], q[0, :, 40:])
    back, _ = sata.rotary_backward(Q, K, pos.cuda(), freq, interleaved=inter, scale=scale)
    want = torch.cat((q[..., :40] * scale * scale, q[..., 40:]), -1)
    assert (back.cpu() - want).abs().max() <= 64 * 2.0 ** -24 * q.abs().max() * scale * scale


def test_gradient(sata):
    """<dy, turn(x)> has the gradient turn_back(dy): against differences along random directions (the map is linear)."""
    gen = torch.Generator().manual_seed(6)
    x, dy, e = (torch.randn(2, 3, 9, 24, generator=gen).cuda() for _ in range(3))
    pos = torch.arange(18, dtype=torch.int32).reshape(2, 9).cuda() * 37
    freq, _ = sata.rotary_frequencies(9, device="cuda")
    grad, _ = sata.rotary_backward(dy, None, pos, freq, scale=1.5)
    turn = lambda z: sata.rotary(z, None, pos, freq, scale=1.5)[0].double()  # noqa: E731
    slope = ((turn(x + e) - turn(x - e)) * dy.double()).sum() / 2
    # (each of the 1296 terms is off by a few 2^-24 of sizes around 4)
    assert abs(slope - (grad.double() * e.double()).sum()) <= 1296 * 16 * 4 * 2.0 ** -24


def test_not_finite_stays_in_its_pair(sata):
    q = torch.randn(1, 1, 3, 16, generator=torch.Generator().manual_seed(7))
    q[0, 0, 1, 2] = math.inf
    q[0, 0, 1, 13] = math.nan
    for inter in (False, True):
        freq, _ = sata.rotary_frequencies(6, device="cuda")
        y = sata.rotary(q.cuda(), None, torch.tensor([[1, 2, 3]], dtype=torch.int32).cuda(), freq, interleaved=inter)[0].cpu()
        bad = ~torch.isfinite(y)
        want = torch.zeros_like(bad)
        for i in ((2, 8) if not inter else (2, 3)):
            want[0, 0, 1, i] = True
        want[0, 0, 1, 13] = True  # (behind the pairs: as it is)
        assert torch.equal(bad, want)


def test_unaligned(sata):
    """Tensors that start in the middle of a vector."""
    gen = torch.Generator().manual_seed(8)
    pos = torch.arange(6, dtype=torch.int32)[None]
    freq, _ = sata.rotary_frequencies(16, device="cuda")
    for dt in (torch.bfloat16, torch.float32):
        x = torch.randn(1, 2, 6, 32, generator=gen).to(dt)
        want = sata.rotary(x.cuda(), None, pos.cuda(), freq)[0]
        for inter in (False, True):
            want = sata.rotary(x.cuda(), None, pos.cuda(), freq, interleaved=inter)[0]
            for off in (1, 2, 3, 4):
                buf = torch.zeros(x.numel() + 8, dtype=dt, device="cuda")
                at = buf[off:off + x.numel()].view(x.shape)
                at.copy_(x)
                assert torch.equal(sata.rotary(at, None, pos.cuda(), freq, interleaved=inter, q_out=at)[0], want)
                assert (buf[:off] == 0).all() and (buf[off + x.numel():] == 0).all()


def test_empty_and_refusals(sata):
    z = torch.zeros(2, 3, 0, 16, device="cuda")
    freq, _ = sata.rotary_frequencies(8, device="cuda")
    pos = torch.zeros(2, 0, dtype=torch.int32, device="cuda")
    assert sata.rotary(z, z, pos, freq)[0].shape == z.shape
    q = torch.zeros(2, 3, 4, 16, device="cuda")
    pos = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    with pytest.raises(sata.SataError):
        sata.rotary(q, None, pos, sata.rotary_frequencies(9, device="cuda")[0])
    with pytest.raises(sata.SataError):
        sata.rotary(q, q.clone(), pos, freq, q_out=q, k_out=q)
    with pytest.raises(TypeError):
        sata.rotary(q, None, pos.long(), freq)
    with pytest.raises(TypeError):
        sata.rotary(q, None, pos, freq.double())
    with pytest.raises(ValueError):
        sata.rotary(q, None, pos[:, :3], freq)
    with pytest.raises(ValueError):
        sata.rotary(q.transpose(1, 2), None, pos, freq)
    with pytest.raises(ValueError):
        sata.rotary(q, None, pos.cpu(), freq)
    with pytest.raises(TypeError):
        sata.rotary(q, q.bfloat16(), pos, freq)


def test_captured(sata):
    q = torch.randn(2, 4, 1, 64, generator=torch.Generator().manual_seed(9)).cuda()
    pos = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    freq, _ = sata.rotary_frequencies(32, device="cuda")
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sata.rotary(q, None, pos, freq, q_out=out)
    for i in range(4):
        pos.fill_(1000 * i)
        q.add_(1.0)
        graph.replay()
        want = sata.rotary(q, None, pos, freq)[0]
        torch.cuda.synchronize()
        assert torch.equal(out, want)
