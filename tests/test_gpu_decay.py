"""Decayed linear attention on the GPU against its definition in float64, element
by element within derived bounds (pair_ref.py): prompts, single tokens and
gradients over types, head sizes, lengths and decays; values that are not
finite; streams and captured graphs."""
import math
import sys

import pytest

import pair_ref
import routes

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def sata():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    import paper_2602_00294_amd as m
    m.load_library()
    return m


def _say(*msg):
    print(*msg, file=sys.stderr, flush=True)


def _make(seed, B, H, G, n, dk, dv, dtype, offset=0):
    """q, k, v, dy, S_in, dS, log_decay; `offset` elements off the allocations' alignment."""
    g = torch.Generator().manual_seed(seed)

    def r(*s, dtype=DT[dtype]):
        x = torch.randn(*s, generator=g).to(dtype)
        if not offset:
            return x.cuda()
        held = torch.empty(x.numel() + offset, dtype=dtype, device="cuda")
        held[offset:] = x.reshape(-1).cuda()
        return held[offset:].view(*s)

    rate = torch.tensor([[0.0, -0.02, -0.7, -1e-4, -25.0, -math.inf][(h + seed) % 6] for h in range(H)])
    return (r(B, H * G, n, dk), r(B, H, n, dk), r(B, H, n, dv), r(B, H * G, n, dv),
            r(B, H, dk, dv, dtype=torch.float32), r(B, H, dk, dv, dtype=torch.float32), rate.cuda())


def _lengths(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


CASES = [  # B, H, G, n, dk, dv, dtype, lengths, states
    (1, 1, 1, 1, 1, 1, "f32", None, False),
    (1, 2, 1, 1, 64, 64, "bf16", None, True),
    (2, 6, 1, 63, 16, 16, "bf16", None, True),
    (1, 3, 2, 64, 32, 32, "bf16", None, False),
    (1, 6, 1, 65, 32, 32, "f32", None, True),
    (2, 2, 3, 130, 24, 40, "f32", [0, 130], True),
    (3, 2, 1, 129, 8, 5, "bf16", [1, 64, 128], True),
    (2, 3, 2, 200, 33, 31, "bf16", [199, 7], True),
    (1, 2, 1, 257, 128, 128, "bf16", None, True),
    (1, 1, 2, 190, 128, 128, "f32", None, True),
    (2, 1, 1, 150, 128, 16, "bf16", [150, 90], False),
    (2, 1, 1, 150, 16, 128, "f32", [-3, 1000], True),
    (1, 2, 4, 100, 100, 72, "f32", None, True),
    (1, 1, 1, 2500, 64, 64, "bf16", None, True),
    (2, 1, 2, 1700, 96, 64, "f32", [1650, 3], True),
    (1, 1, 8, 300, 17, 127, "bf16", None, True),
]


@pytest.mark.parametrize("B,H,G,n,dk,dv,dtype,lengths,states", CASES)
def test_prompt(sata, B, H, G, n, dk, dv, dtype, lengths, states):
    _say("decay prompt", B, H, G, n, dk, dv, dtype, lengths, states)
    q, k, v, _, S_in, _, g = _make(n + dk, B, H, G, n, dk, dv, dtype)
    S_in = S_in if states else None
    y, S = sata.decay_prefill(q, k, v, g, _lengths(lengths), S_in)
    torch.cuda.synchronize()
    ry, rS = pair_ref.decay_prefill(q, k, v, g, lengths, S_in)
    _say("  of the bound: y %.3f, S %.3f" % (pair_ref.check(y, ry, "y"), pair_ref.check(S, rS, "S")))
    none, gone = sata.decay_prefill(q, k, v, g, _lengths(lengths), S_in, want_state=False)
    assert gone is None and torch.equal(none, y)


@pytest.mark.parametrize("B,H,G,n,dk,dv,dtype,lengths,states", CASES)
def test_gradients(sata, B, H, G, n, dk, dv, dtype, lengths, states):
    _say("decay gradients", B, H, G, n, dk, dv, dtype, lengths, states)
    q, k, v, dy, S_in, dS, g = _make(n + dv, B, H, G, n, dk, dv, dtype)
    S_in, dS = (S_in, dS) if states else (None, None)
    got = sata.decay_backward(q, k, v, g, dy, _lengths(lengths), S_in, dS)
    torch.cuda.synchronize()
    want = pair_ref.decay_backward(q, k, v, g, dy, lengths, S_in, dS)
    assert (got[3] is None) == (S_in is None)
    _say("  of the bounds:", ["%.3f" % pair_ref.check(a, w, name) for name, a, w in
                              zip(("dq", "dk", "dv", "dS_in"), got, want) if a is not None])


@pytest.mark.parametrize("B,H,G,dk,dv,dtype", [(1, 1, 1, 1, 1, "f32"), (3, 2, 1, 64, 64, "bf16"), (2, 3, 4, 128, 128, "bf16"),
                                               (1, 5, 3, 33, 7, "f32"), (70, 16, 1, 16, 16, "bf16"), (2, 2, 9, 100, 60, "f32"),
                                               (1, 2, 2, 128, 3, "bf16"), (1, 2, 16, 5, 128, "bf16")])
@pytest.mark.parametrize("offset", [0, 1])
def test_token(sata, B, H, G, dk, dv, dtype, offset):
    _say("decay token", B, H, G, dk, dv, dtype, offset)
    q, k, v, _, S, _, g = _make(dk, B, H, G, 1, dk, dv, dtype, offset)
    q, k, v = q[:, :, 0], k[:, :, 0], v[:, :, 0]
    ry, rS = pair_ref.decay_step(S, q, k, v, g)
    y = sata.decay_step(S, q, k, v, g)
    torch.cuda.synchronize()
    pair_ref.check(y, ry, "y")
    pair_ref.check(S, rS, "S")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unaligned_tensors(sata, dtype):
    q, k, v, dy, S_in, dS, g = _make(5, 2, 2, 2, 77, 32, 64, dtype, offset=1)
    _say("decay, tensors one element off", dtype)
    y, S = sata.decay_prefill(q, k, v, g, None, S_in)
    got = sata.decay_backward(q, k, v, g, dy, None, S_in, dS)
    torch.cuda.synchronize()
    ry, rS = pair_ref.decay_prefill(q, k, v, g, None, S_in)
    pair_ref.check(y, ry, "y")
    pair_ref.check(S, rS, "S")
    for a, w in zip(got, pair_ref.decay_backward(q, k, v, g, dy, None, S_in, dS)):
        pair_ref.check(a, w)


def test_prompt_in_pieces_and_tokens(sata):
    """A prompt in two pieces of odd sizes, then token by token, is the whole prompt."""
    n, cut, steps = 260, 101, 30
    q, k, v, _, _, _, g = _make(6, 2, 3, 2, n + steps, 32, 48, "f32")
    g = torch.tensor([0.0, -0.03, -1e-3], device="cuda")
    _say("decay prompt in pieces, then tokens")
    part = lambda x, a, b: x[:, :, a:b].contiguous()  # noqa: E731
    y1, S1 = sata.decay_prefill(*(part(x, 0, cut) for x in (q, k, v)), g)
    y2, S = sata.decay_prefill(*(part(x, cut, n) for x in (q, k, v)), g, S_in=S1)
    ys = [sata.decay_step(S, *(x[:, :, t].contiguous() for x in (q, k, v)), g)[:, :, None] for t in range(n, n + steps)]
    torch.cuda.synchronize()
    ry, rS = pair_ref.decay_prefill(q, k, v, g)
    pair_ref.check(torch.cat([y1, y2] + ys, 2), ry, "y")
    pair_ref.check(S, rS, "S")


def test_many_tokens_keep_the_decay(sata):
    """exp(log_decay) is not a float32 number: 4096 steps with a slow decay stay within
    the roundings of one step each, which are independent, not 4096 times the decay's."""
    g = torch.tensor([-1.1e-4], device="cuda")
    S = torch.ones(1, 1, 8, 8, device="cuda")
    z = torch.zeros(1, 1, 8, device="cuda")
    steps = 4096
    for _ in range(steps):
        sata.decay_step(S, z, z, z, g)
    want = math.exp(steps * float(g.double()))
    # each step rounds by at most 2^-24, either way; by chance the sum is sqrt(steps) of them, 6 times that is never seen
    assert abs(S[0, 0, 0, 0].item() / want - 1) < 6 * math.sqrt(steps) * 2.0 ** -24
    q, k, v, _, S_in, _, _ = _make(7, 1, 1, 1, 6000, 8, 8, "f32")
    y, S = sata.decay_prefill(q, torch.zeros_like(k), v, g, S_in=S_in)
    torch.cuda.synchronize()
    assert torch.allclose(S.double(), S_in.double() * math.exp(6000 * float(g.double())), rtol=3e-6, atol=0)


def test_no_tokens(sata):
    q, k, v, dy, S_in, dS, g = _make(8, 2, 2, 1, 0, 8, 4, "bf16")
    y, S = sata.decay_prefill(q, k, v, g, None, S_in)
    got = sata.decay_backward(q, k, v, g, dy, None, S_in, dS)
    zero = sata.decay_prefill(q, k, v, g)[1]
    torch.cuda.synchronize()
    assert y.shape == (2, 2, 0, 4) and torch.equal(S, S_in) and torch.equal(got[3], dS)
    assert not zero.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_values_that_are_not_finite(sata, dtype, bad):
    """Padding rows may hold anything; a token's values reach later outputs only, its gradient earlier ones only."""
    n, ends, at = 200, [150, 200], 100
    _say("decay, not finite", dtype, bad)
    q, k, v, dy, S_in, dS, g = _make(9, 2, 2, 2, n, 40, 24, dtype)
    g = torch.tensor([-0.01, -0.3], device="cuda")
    lens = _lengths(ends)
    y, S = sata.decay_prefill(q, k, v, g, lens, S_in)
    grads = sata.decay_backward(q, k, v, g, dy, lens, S_in, dS)
    holes = [x.clone() for x in (q, k, v, dy)]
    for x in holes:
        x[0, :, ends[0]:] = bad
    y2, S2 = sata.decay_prefill(*holes[:3], g, lens, S_in)
    assert torch.equal(y2, y) and torch.equal(S2, S)
    for a, b in zip(sata.decay_backward(*holes[:3], g, holes[3], lens, S_in, dS), grads):
        assert torch.equal(a, b)
    for name, x in (("k", 1), ("v", 2)):
        args = [t.clone() for t in (q, k, v)]
        args[x][1, 1, at, 3] = bad
        y2, S2 = sata.decay_prefill(*args, g, lens, S_in)
        assert torch.equal(y2[0], y[0]) and torch.equal(y2[1, :2], y[1, :2]) and torch.equal(S2[1, 0], S[1, 0])
        assert torch.equal(y2[1, 2:, :at], y[1, 2:, :at])
        assert not torch.isfinite(y2[1, 2:, at]).all() and not torch.isfinite(S2[1, 1]).all()
        dq = sata.decay_backward(*args, g, dy, lens, S_in, dS)[0]
        assert torch.equal(dq[1, 2:, :at], grads[0][1, 2:, :at]) and torch.equal(dq[1, :2], grads[0][1, :2])
        assert not torch.isfinite(dq[1, 2:, at]).all()
    args = [t.clone() for t in (q, dy)]
    args[0][1, 3, at, 0] = bad
    args[1][1, 3, at, 0] = bad
    y2, S2 = sata.decay_prefill(args[0], k, v, g, lens, S_in)
    keep = torch.arange(n, device="cuda") != at
    assert torch.equal(y2[:, :, keep], y[:, :, keep]) and torch.equal(S2, S)
    got = sata.decay_backward(args[0], k, v, g, args[1], lens, S_in, dS)
    assert torch.equal(got[0][:, :, keep], grads[0][:, :, keep])
    for a, b in zip(got[1:3], grads[1:3]):
        assert torch.equal(a[1, 1, at + 1:], b[1, 1, at + 1:]) and torch.equal(a[1, 0], b[1, 0]) and torch.equal(a[0], b[0])
        assert not torch.isfinite(a[1, 1, at]).all()


def test_streams_and_repeats(sata):
    """The same bits on every run, on the default stream and on two others at once."""
    q, k, v, dy, S_in, dS, g = _make(10, 2, 4, 2, 900, 64, 64, "bf16")
    want = [*sata.decay_prefill(q, k, v, g, None, S_in), *sata.decay_backward(q, k, v, g, dy, None, S_in, dS)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    runs = []
    for _ in range(2):
        for s in streams:
            with torch.cuda.stream(s):
                runs.append([*sata.decay_prefill(q, k, v, g, None, S_in),
                             *sata.decay_backward(q, k, v, g, dy, None, S_in, dS)])
    torch.cuda.synchronize()
    for r in runs:
        assert all(torch.equal(a, b) for a, b in zip(r, want))


def test_captured(sata):
    """Prompt, gradients and token in one graph, replayed with other inputs and eager work in between."""
    make = lambda seed: list(_make(seed, 1, 2, 2, 700, 32, 64, "bf16"))  # noqa: E731
    held = make(11)
    tok = [t[:, :, 0].contiguous() for t in held[:3]]
    stream = torch.cuda.Stream()

    def work(h, S):
        y, last = sata.decay_prefill(h[0], h[1], h[2], h[6], None, h[4])
        grads = sata.decay_backward(h[0], h[1], h[2], h[6], h[3], None, h[4], h[5])
        S.copy_(last)
        return [y, last, *grads, sata.decay_step(S, *tok, h[6]), S]

    S = torch.zeros(1, 2, 32, 64, device="cuda")
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        work(held, S)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = work(held, S)
    for seed in (12, 13, 14):
        with torch.cuda.stream(stream):
            for a, b in zip(held, make(seed)):
                a.copy_(b)
            graph.replay()
        stream.synchronize()
        want = work(held, torch.zeros_like(S))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_offsets_past_32_bits(sata):
    """Tensors of more than 2^31 entries: the last head's rows lie behind them."""
    H, n, d, end = 17, 1 << 20, 128, 70
    _say("decay, offsets past 32 bits")
    gen = torch.Generator().manual_seed(13)
    small = [torch.randn(1, 1, end, d, generator=gen).bfloat16().cuda() for _ in range(4)]
    big = [torch.zeros(1, H, n, d, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    assert big[0].numel() > 2 ** 31
    for x, part in zip(big, small):
        x[:, -1:, :end] = part
    g, lens = torch.full((H,), -0.02, device="cuda"), torch.tensor([end], dtype=torch.int32, device="cuda")
    q, k, v, dy = big
    y, S = sata.decay_prefill(q, k, v, g, lens)
    torch.cuda.synchronize()
    ry, rS = pair_ref.decay_prefill(*small[:3], g[:1])
    pair_ref.check(y[:, -1:, :end], ry, "y")
    pair_ref.check(S[:, -1:], rS, "S")
    assert not y[:, -1, end:].any()
    del y
    grads = sata.decay_backward(q, k, v, g, dy, lens)[:3]
    torch.cuda.synchronize()
    for name, a, w in zip(("dq", "dk", "dv"), grads, pair_ref.decay_backward(*small[:3], g[:1], small[3])):
        pair_ref.check(a[:, -1:, :end], w, name)
        assert not a[:, -1, end:].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,lengths", [(100, [100, 37]), (700, [700, 1])])
def test_a_decay_that_is_no_number(sata, dtype, n, lengths):
    """NaN as a head's decay: what its powers enter is NaN, what they do not (the last token's share of its own
    gradients, states that no token follows, other heads) is what it was."""
    _say("decay of NaN", dtype, n, lengths)
    q, k, v, dy, S_in, dS, _ = _make(21, 2, 2, 2, n, 24, 40, dtype)
    g = torch.tensor([math.nan, -0.1], device="cuda")
    lens = _lengths(lengths)

    def same(name, got, ref):
        got, (want, bound) = got.double().cpu(), ref
        gone = torch.isnan(want)
        assert torch.equal(torch.isnan(got), gone), f"{name}: NaN in {int(torch.isnan(got).sum())}, not {int(gone.sum())} places"
        assert ((got - want).abs()[~gone] <= bound[~gone]).all(), name

    for S0 in (None, S_in):
        y, S = sata.decay_prefill(q, k, v, g, lens, S0)
        torch.cuda.synchronize()
        ry, rS = pair_ref.decay_prefill(q, k, v, g, lengths, S0)
        assert torch.isnan(ry[0][:, :2, 0]).all() and torch.isnan(rS[0][:, 0]).all() and not torch.isnan(ry[0][:, 2:]).any()
        same("y", y, ry)
        same("S", S, rS)
    grads = sata.decay_backward(q, k, v, g, dy, lens, S_in, dS)
    torch.cuda.synchronize()
    for name, a, w in zip(("dq", "dk", "dv", "dS_in"), grads, pair_ref.decay_backward(q, k, v, g, dy, lengths, S_in, dS)):
        assert torch.isnan(w[0]).any()
        same(name, a, w)
    row = [x[:, :, 0].contiguous() for x in (q, k, v)]
    ry, rS = pair_ref.decay_step(S_in, *row, g)
    y = sata.decay_step(S_in, *row, g)
    torch.cuda.synchronize()
    same("token's y", y, ry)
    same("token's S", S_in, rS)


PARTS = [  # dtype, B, H, G, n, dk, dv: sequences in several parts of several chunks, of more than 8 heads
    ("bf16", 3, 3, 2, 1600, 128, 128), ("bf16", 2, 9, 1, 1000, 96, 96), ("bf16", 2, 20, 2, 900, 96, 72),
    ("f32", 4, 16, 1, 600, 128, 100), ("bf16", 2, 25, 1, 500, 96, 96), ("f32", 2, 9, 1, 700, 64, 64),
    ("bf16", 3, 40, 1, 600, 32, 32), ("bf16", 4, 16, 1, 1200, 96, 96),
]


@pytest.mark.parametrize("dtype,B,H,G,n,dk,dv", PARTS)
@pytest.mark.parametrize("offset", [0, 1])
def test_parts_of_several_chunks(sata, dtype, B, H, G, n, dk, dv, offset):
    """Lengths that end inside a chunk, at a part's border and in a part in the middle; decays that take the state's
    unit below 2^-8 never, in each chunk and after some chunks of a part."""
    plans = [routes.decay_parts(gradients, dtype, B, H, G, n, dk, dv) for gradients in (False, True)]
    _say("decay in parts", dtype, B, H, G, n, dk, dv, plans, offset)
    length = max(length for parts, length in plans if parts > 1)
    assert length >= 64 and B * H > 8
    q, k, v, dy, S_in, dS, _ = _make(n + dv, B, H, G, n, dk, dv, dtype, offset)
    rates = [0.0, -0.02, -0.1, -0.7, -1e-4, -0.06, -25.0, -math.inf]
    g = torch.tensor([rates[h % 8] for h in range(H)], device="cuda")
    for lengths in (None, [n - 7, length * 2 + 37, length, 0][:B]):
        y, S = sata.decay_prefill(q, k, v, g, _lengths(lengths), S_in)
        got = sata.decay_backward(q, k, v, g, dy, _lengths(lengths), S_in, dS)
        torch.cuda.synchronize()
        ry, rS = pair_ref.decay_prefill(q, k, v, g, lengths, S_in)
        worst = [pair_ref.check(y, ry, "y"), pair_ref.check(S, rS, "S")]
        worst += [pair_ref.check(a, w, name) for name, a, w in
                  zip(("dq", "dk", "dv", "dS_in"), got, pair_ref.decay_backward(q, k, v, g, dy, lengths, S_in, dS))]
        _say("  of the bounds: y, S, dq, dk, dv, dS_in", ["%.3f" % x for x in worst])
        if offset:
            break


@pytest.mark.parametrize("dk,dv", [(96, 96), (72, 96), (96, 65)])
@pytest.mark.parametrize("offset", [0, 1])
def test_three_tiles_of_columns(sata, dk, dv, offset):
    """d of 65 to 96 in bfloat16: a staging pass covers 12 rows, the third one more than the tile has."""
    _say("decay, three tiles of columns", dk, dv, offset)
    n, lengths = 203, [203, 97]
    q, k, v, dy, S_in, dS, g = _make(dk + dv, 2, 6, 2, n, dk, dv, "bf16", offset)
    y, S = sata.decay_prefill(q, k, v, g, _lengths(lengths), S_in)
    got = sata.decay_backward(q, k, v, g, dy, _lengths(lengths), S_in, dS)
    torch.cuda.synchronize()
    ry, rS = pair_ref.decay_prefill(q, k, v, g, lengths, S_in)
    pair_ref.check(y, ry, "y")
    pair_ref.check(S, rS, "S")
    for name, a, w in zip(("dq", "dk", "dv", "dS_in"), got, pair_ref.decay_backward(q, k, v, g, dy, lengths, S_in, dS)):
        pair_ref.check(a, w, name)


@pytest.mark.parametrize("B,H,G,n,dk,dv,lengths", [(1, 6, 2, 300, 64, 64, None), (2, 9, 1, 700, 128, 100, [700, 333]),
                                                   (2, 3, 2, 190, 24, 40, [190, 1])])
def test_bfloat16_sums_carry_sixteen_bits(sata, monkeypatch, B, H, G, n, dk, dv, lengths):
    """Sums of signed terms cancel, so the weights and the state's entries of bfloat16 calls are two bfloat16
    numbers each, 2^-17 of them off, not one; what is rounded to bfloat16 is the result."""
    _say("decay, sixteen bits", B, H, G, n, dk, dv, lengths)
    monkeypatch.setitem(pair_ref.WEIGHT, torch.bfloat16, 2.0 ** -17)
    q, k, v, dy, S_in, dS, g = _make(n + dk, B, H, G, n, dk, dv, "bf16")
    S_in[:, :, ::2] += 1000.0  # (large entries that cancel in the readout)
    S_in[:, :, 1::2] -= 1000.0
    y, S = sata.decay_prefill(q, k, v, g, _lengths(lengths), S_in)
    got = sata.decay_backward(q, k, v, g, dy, _lengths(lengths), S_in, dS)
    torch.cuda.synchronize()
    ry, rS = pair_ref.decay_prefill(q, k, v, g, lengths, S_in)
    pair_ref.check(y, ry, "y")
    pair_ref.check(S, rS, "S")
    for name, a, w in zip(("dq", "dk", "dv", "dS_in"), got, pair_ref.decay_backward(q, k, v, g, dy, lengths, S_in, dS)):
        pair_ref.check(a, w, name)
