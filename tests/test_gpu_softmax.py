"""Exact softmax attention on the GPU against its definition in float64, element by
element within derived bounds (pair_ref.py): prompts, gradients and single
tokens over a cache; values that are not finite; streams and captured graphs."""
import math
import sys

import pytest

import pair_ref

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


def _rand(seed, dtype, *shapes, offset=0, size=1.0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for s in shapes:
        x = (torch.randn(*s, generator=g) * size).to(DT[dtype])
        held = torch.empty(x.numel() + offset, dtype=x.dtype, device="cuda")
        held[offset:] = x.reshape(-1).cuda()
        out.append(held[offset:].view(*s))
    return out


def _prompt(seed, B, H, G, n, dk, dv, dtype, **more):
    return _rand(seed, dtype, (B, H * G, n, dk), (B, H, n, dk), (B, H, n, dv), (B, H * G, n, dv), **more)


def _lengths(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


CASES = [  # B, H, G, n, dk, dv, dtype, lengths
    (1, 1, 1, 1, 1, 1, "f32", None),
    (1, 2, 1, 1, 64, 64, "bf16", None),
    (2, 2, 1, 63, 16, 16, "bf16", None),
    (1, 3, 2, 64, 32, 32, "bf16", None),
    (1, 2, 1, 65, 32, 32, "f32", None),
    (2, 2, 3, 130, 24, 40, "f32", [0, 130]),
    (3, 2, 1, 129, 8, 5, "bf16", [1, 64, 128]),
    (2, 3, 2, 200, 33, 31, "bf16", [199, 7]),
    (1, 2, 1, 257, 128, 128, "bf16", None),
    (1, 1, 2, 190, 128, 128, "f32", None),
    (2, 1, 1, 150, 128, 16, "bf16", [150, 90]),
    (2, 1, 1, 150, 16, 128, "f32", [-3, 1000]),
    (1, 2, 4, 100, 100, 72, "f32", None),
    (1, 1, 1, 1500, 64, 64, "bf16", None),
    (2, 1, 2, 700, 96, 64, "f32", [650, 3]),
    (1, 1, 8, 300, 17, 127, "bf16", None),
    (1, 9, 2, 385, 64, 96, "bf16", None),
]


def _check_prompt(sata, q, k, v, dy, lengths):
    lens = _lengths(lengths)
    y, lse = sata.softmax_prefill(q, k, v, lens)
    torch.cuda.synchronize()
    ry, rl = pair_ref.softmax_prefill(q, k, v, lengths)
    worst = [pair_ref.check(y, ry, "y"), pair_ref.check(lse, rl, "lse")]
    again, none = sata.softmax_prefill(q, k, v, lens, want_lse=False)
    assert none is None and torch.equal(again, y)
    got = sata.softmax_backward(q, k, v, y, lse, dy, lens)
    torch.cuda.synchronize()
    want = pair_ref.softmax_backward(q, k, v, y, lse, dy, lengths)
    worst += [pair_ref.check(a, w, name) for name, a, w in zip(("dq", "dk", "dv"), got, want)]
    _say("  of the bounds: y, lse, dq, dk, dv", ["%.3f" % x for x in worst])


@pytest.mark.parametrize("B,H,G,n,dk,dv,dtype,lengths", CASES)
def test_prompt_and_gradients(sata, B, H, G, n, dk, dv, dtype, lengths):
    _say("softmax prompt", B, H, G, n, dk, dv, dtype, lengths)
    _check_prompt(sata, *_prompt(n + dk, B, H, G, n, dk, dv, dtype), lengths)


MANY_HEADS = [  # B, H, G, n, dk, dv, dtype, lengths
    (8, 16, 1, 300, 32, 32, "bf16", None),
    (2, 16, 4, 513, 16, 128, "bf16", [513, 400]),
    (3, 30, 3, 33, 64, 64, "bf16", [33, 0, 32]),
    (4, 16, 4, 65, 96, 80, "f32", [65, 64, 1, 33]),
    (5, 30, 1, 200, 24, 32, "f32", None),
    (5, 30, 1, 200, 64, 40, "f32", [200, 130, 1, 0, 150]),
    (5, 30, 1, 161, 96, 96, "f32", [161, 96, 97, 64, 31]),
    (5, 30, 1, 160, 128, 100, "f32", None),
    (5, 30, 1, 130, 33, 31, "bf16", [130, 129, 128, 127, -4]),
    (5, 30, 1, 200, 64, 40, "bf16", [64, 200, 193, 32, 192]),
    (5, 30, 1, 290, 96, 72, "bf16", [289, 290, 1, 256, 225]),
    (2, 80, 2, 257, 128, 128, "bf16", None),
    (8, 32, 1, 300, 32, 32, "bf16", None),
    (4, 64, 1, 270, 64, 40, "bf16", [270, 257, 256, 0]),
    (2, 66, 2, 300, 96, 72, "bf16", [289, 300]),
    (2, 33, 4, 513, 16, 128, "bf16", [513, 400]),
]


@pytest.mark.parametrize("B,H,G,n,dk,dv,dtype,lengths", MANY_HEADS)
def test_many_heads(sata, B, H, G, n, dk, dv, dtype, lengths):
    _say("softmax prompt, many heads", B, H, G, n, dk, dv, dtype, lengths)
    _check_prompt(sata, *_prompt(n + dk, B, H, G, n, dk, dv, dtype), lengths)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unaligned_tensors(sata, dtype):
    _say("softmax, tensors one element off", dtype)
    _check_prompt(sata, *_prompt(3, 2, 2, 2, 77, 32, 64, dtype, offset=1), None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_scores(sata, dtype):
    """Scores of some hundreds: most weights vanish, the maximum moves late, and nothing overflows."""
    _say("softmax, far scores", dtype)
    q, k, v, dy = _prompt(4, 1, 2, 1, 300, 32, 32, dtype)
    k = k * torch.linspace(0.1, 40.0, 300, device="cuda")[None, None, :, None].to(k.dtype)
    _check_prompt(sata, q, k.contiguous(), v, dy, None)


TOKENS = [  # B, H, G, capacity, dk, dv, dtype, lengths
    (1, 1, 1, 1, 1, 1, "f32", [0]),
    (2, 2, 1, 70, 64, 64, "bf16", [0, 69]),
    (4, 2, 4, 300, 128, 128, "bf16", [299, 255, 1, 64]),
    (3, 3, 2, 130, 33, 40, "f32", [129, 63, 5]),
    (4, 1, 8, 200, 16, 16, "bf16", [-1, 200, 199, 100]),
    (1, 2, 3, 5000, 64, 32, "f32", [4321]),
    (2, 1, 1, 4099, 128, 128, "f32", [4098, 17]),
    (1, 1, 20, 2600, 96, 100, "bf16", [2599]),
    (2, 2, 1, 3001, 40, 24, "bf16", [3000, 2047]),
    # groups of more than 32
    (2, 2, 33, 70, 32, 32, "bf16", [69, 31]),
    (1, 2, 70, 700, 64, 40, "f32", [650]),
    # one long sequence among short ones, ones without a token among them
    (5, 2, 2, 9000, 32, 32, "bf16", [3, 8999, -1, 100, 9000]),
    (70, 4, 1, 1100, 16, 16, "bf16", [(397 * b) % 1103 - 1 for b in range(70)]),
    # more heads than the card holds workgroups, and about as many
    (150, 4, 2, 600, 16, 24, "bf16", [(211 * b) % 600 for b in range(150)]),
    (65, 4, 1, 900, 16, 16, "f32", [899] + [(97 * b) % 300 for b in range(64)]),
    (48, 8, 1, 800, 16, 16, "bf16", [(173 * b) % 800 for b in range(48)]),
    # very many sequences
    (400, 1, 2, 3000, 16, 8, "bf16", [(457 * b) % 3003 - 1 for b in range(400)]),
    (390, 2, 1, 270, 32, 32, "f32", [(97 * b) % 270 for b in range(390)]),
]


@pytest.mark.parametrize("B,H,G,cap,dk,dv,dtype,lengths", TOKENS)
@pytest.mark.parametrize("offset", [0, 1])
def test_token(sata, B, H, G, cap, dk, dv, dtype, lengths, offset):
    _say("softmax token", B, H, G, cap, dk, dv, dtype, lengths, offset)
    K, V, q, k, v = _rand(cap, dtype, (B, H, cap, dk), (B, H, cap, dv), (B, H * G, dk), (B, H, dk), (B, H, dv),
                          offset=offset)
    for b, e in enumerate(lengths):  # rows behind a sequence may hold anything
        K[b, :, max(e, 0):], V[b, :, max(e, 0):] = math.nan, math.inf
    at = _lengths(lengths)
    ry, rK, rV = pair_ref.softmax_step(K, V, lengths, q, k, v)
    y = sata.softmax_step(K, V, at, q, k, v)
    torch.cuda.synchronize()
    pair_ref.check(y, ry, "y")
    assert torch.equal(K.cpu().nan_to_num(7.0), rK.nan_to_num(7.0)) and torch.equal(V.cpu(), rV)
    assert at.tolist() == lengths


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_then_tokens(sata, dtype):
    """Tokens over the cache of a prompt are the rows of the longer prompt."""
    _say("softmax prompt, then tokens", dtype)
    ends, n, steps = [60, 33], 60, 12
    q, k, v, _ = _prompt(5, 2, 2, 2, n + steps, 32, 48, dtype)
    K, V = torch.full_like(k, math.nan), torch.full_like(v, math.nan)
    K[:, :, :n], V[:, :, :n] = k[:, :, :n], v[:, :, :n]
    at = _lengths(ends)
    ys = []
    for t in range(steps):
        row = lambda x: torch.stack([x[b, :, e + t] for b, e in enumerate(ends)])  # noqa: E731
        ys.append(sata.softmax_step(K, V, at, row(q), row(k), row(v)))
        at += 1
    torch.cuda.synchronize()
    ref = pair_ref.softmax_prefill(q, k, v)[0]
    for t, y in enumerate(ys):
        for b, e in enumerate(ends):
            pair_ref.check(y[b], (ref[0][b, :, e + t], ref[1][b, :, e + t]), f"token {t} of {b}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("H,G", [(2, 2), (70, 1)])
def test_values_that_are_not_finite(sata, dtype, bad, H, G):
    """Padding rows may hold anything; a token's values reach later rows only, its query and gradient earlier keys
    only.  What does not depend on the value is the same in bits in other heads, sequences and rows further off;
    in the value's own 32 rows the pairs are summed in another way, so that both ways are held to the bound of the
    exact result."""
    n, ends, at = 200, [150, 200], 100
    _say("softmax, not finite", dtype, bad, H, G)
    q, k, v, dy = _prompt(6, 2, H, G, n, 40, 24, dtype)
    lens = _lengths(ends)
    y, lse = sata.softmax_prefill(q, k, v, lens)
    grads = sata.softmax_backward(q, k, v, y, lse, dy, lens)
    exact = pair_ref.softmax_prefill(q, k, v, ends)
    exact_grads = pair_ref.softmax_backward(q, k, v, y, lse, dy, ends)
    tile = 32 * (at // 32)  # the first row of the value's 32

    def same(got, was, ref, head, rows, close):
        """Rows `rows` of sequence 1's head: within the bound, and the same bits but for those in `close`."""
        pair_ref.check(got[1, head, rows], (ref[0][1, head, rows], ref[1][1, head, rows]))
        far = [r for r in range(n)[rows] if r not in close]
        assert torch.equal(got[1, head, far], was[1, head, far])

    holes = [x.clone() for x in (q, k, v, dy, y, lse)]
    for x in holes:
        x[0, :, ends[0]:] = bad
    y2, lse2 = sata.softmax_prefill(*holes[:3], lens)
    assert torch.equal(y2, y) and torch.equal(lse2, lse)
    for a, b in zip(sata.softmax_backward(*holes[:3], holes[4], holes[5], holes[3], lens), grads):
        assert torch.equal(a, b)
    for x in (1, 2):
        args = [t.clone() for t in (q, k, v)]
        args[x][1, 1, at, 3] = bad
        y2, lse2 = sata.softmax_prefill(*args, lens)
        assert torch.equal(y2[0], y[0]) and torch.equal(y2[1, :G], y[1, :G])
        dq = sata.softmax_backward(*args, y2, lse2, dy, lens)[0]
        assert torch.equal(dq[0], grads[0][0]) and torch.equal(dq[1, :G], grads[0][1, :G])
        for head in range(G, 2 * G):
            same(y2, y, exact[0], head, slice(0, at), range(tile, at))
            same(lse2, lse, exact[1], head, slice(0, at), range(tile, at))
            same(dq, grads[0], exact_grads[0], head, slice(0, at), range(tile, at))
        for head in range(G, 2 * G):  # (a key with +inf where the query is below 0: score -inf, exp(-inf) = 0, no weight)
            if x == 2 or math.isnan(bad) or q[1, head, at, 3] > 0:
                assert not torch.isfinite(y2[1, head, at]).all()
    args = [t.clone() for t in (q, dy)]
    args[0][1, 2 * G - 1, at, 0] = bad
    args[1][1, 2 * G - 1, at, 0] = bad
    y2, lse2 = sata.softmax_prefill(args[0], k, v, lens)
    keep = torch.arange(n, device="cuda") != at
    assert torch.equal(y2[:, :, keep], y[:, :, keep]) and torch.equal(lse2[:, :, keep], lse[:, :, keep])
    got = sata.softmax_backward(args[0], k, v, y2, lse2, args[1], lens)
    assert torch.equal(got[0][:, :, keep], grads[0][:, :, keep])
    for a, b, ref in zip(got[1:], grads[1:], exact_grads[1:]):
        same(a, b, ref, 1, slice(at + 1, n), range(at + 1, tile + 32))
        assert torch.equal(a[1, 0], b[1, 0]) and torch.equal(a[0], b[0])
        assert not torch.isfinite(a[1, 1, at]).all()


def test_streams_and_repeats(sata):
    q, k, v, dy = _prompt(7, 2, 3, 2, 400, 64, 64, "bf16")
    y, lse = sata.softmax_prefill(q, k, v)
    want = [y, lse, *sata.softmax_backward(q, k, v, y, lse, dy)]
    torch.cuda.synchronize()
    streams, runs = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for _ in range(2):
        for s in streams:
            with torch.cuda.stream(s):
                a, b = sata.softmax_prefill(q, k, v)
                runs.append([a, b, *sata.softmax_backward(q, k, v, a, b, dy)])
    torch.cuda.synchronize()
    for r in runs:
        assert all(torch.equal(a, b) for a, b in zip(r, want))


def test_captured(sata):
    """Prompt, gradients and tokens in one graph, replayed with other inputs and eager work in between; the
    lengths move on inside the graph."""
    make = lambda seed: _prompt(seed, 1, 2, 2, 300, 32, 64, "bf16")  # noqa: E731
    held = make(8)
    at = torch.tensor([100], dtype=torch.int32, device="cuda")
    tok = [held[0][:, :, 5].contiguous(), held[1][:, :, 5].contiguous(), held[2][:, :, 5].contiguous()]
    stream = torch.cuda.Stream()

    def work(h, K, V, at):
        y, lse = sata.softmax_prefill(*h[:3])
        out = [y, lse, *sata.softmax_backward(*h[:3], y, lse, h[3])]
        K.copy_(h[1])
        V.copy_(h[2])
        for _ in range(2):
            out.append(sata.softmax_step(K, V, at, *tok))
            at += 1
        return out + [K, V]

    K, V = torch.zeros_like(held[1]), torch.zeros_like(held[2])
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        work(held, K, V, at)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = work(held, K, V, at)
    for seed in (9, 10, 11):
        before = at.clone()
        with torch.cuda.stream(stream):
            for a, b in zip(held, make(seed)):
                a.copy_(b)
            graph.replay()
        stream.synchronize()
        assert at.item() == before.item() + 2
        want = work(held, torch.zeros_like(K), torch.zeros_like(V), before)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_offsets_past_32_bits(sata):
    """Tensors of more than 2^31 entries: the last head's rows lie behind them."""
    H, n, d, end = 17, 1 << 20, 128, 70
    _say("softmax, offsets past 32 bits")
    last = _prompt(12, 1, 1, 1, end + 1, d, d, "bf16")
    q, k, v, dy = (torch.zeros(1, H, n, d, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    assert q.numel() > 2 ** 31
    for x, part in zip((q, k, v, dy), last):
        x[:, -1:, :end] = part[:, :, :end]
    lens = _lengths([end])
    tokens = [x[:, :, end].contiguous().expand(1, H, d).contiguous() for x in last[:3]]
    ry, rK, rV = pair_ref.softmax_step(k[:, -1:, :end + 2].clone(), v[:, -1:, :end + 2].clone(), [end], *(x[:, -1:] for x in tokens))
    small = [x[:, -1:, :end].contiguous() for x in (q, k, v, dy)]
    y, lse = sata.softmax_prefill(q, k, v, lens)
    torch.cuda.synchronize()
    ref_y, ref_lse = pair_ref.softmax_prefill(*small[:3])
    pair_ref.check(y[:, -1:, :end], ref_y, "y")
    pair_ref.check(lse[:, -1:, :end], ref_lse, "lse")
    assert not y[:, -1, end:].any()
    grads = sata.softmax_backward(q, k, v, y, lse, dy, lens)
    torch.cuda.synchronize()
    want = pair_ref.softmax_backward(*small[:3], y[:, -1:, :end].contiguous(), lse[:, -1:, :end].contiguous(), small[3])
    for name, a, w in zip(("dq", "dk", "dv"), grads, want):
        pair_ref.check(a[:, -1:, :end], w, name)
        assert not a[:, -1, end:].any()
    del grads, y
    got = sata.softmax_step(k, v, lens, *tokens)
    torch.cuda.synchronize()
    pair_ref.check(got[:, -1:], ry, "token")
    assert torch.equal(k[:, -1:, :end + 2].cpu(), rK) and torch.equal(v[:, -1:, :end + 2].cpu(), rV)
    assert not k[:, -1, end + 2:].any()


def test_two_graphs_at_once(sata):
    """Two captured graphs, replayed side by side on two streams, share no scratch."""
    _say("softmax, two graphs at once")
    graphs, outs, wants, streams = [], [], [], [torch.cuda.Stream() for _ in range(2)]
    for i, stream in enumerate(streams):
        h = _prompt(20 + i, 2, 2, 2, 1200, 64, 64, "bf16")
        K, V, at = h[1].clone(), h[2].clone(), _lengths([1100, 700])
        tok = [h[0][:, :, 5].contiguous(), h[1][:, :, 5].contiguous(), h[2][:, :, 5].contiguous()]

        def work(h=h, K=K, V=V, at=at, tok=tok):
            y, lse = sata.softmax_prefill(*h[:3])
            return [y, lse, *sata.softmax_backward(*h[:3], y, lse, h[3]), sata.softmax_step(K, V, at, *tok)]

        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            wants.append([x.clone() for x in work()])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            outs.append(work())
        graphs.append((graph, work))
    for _ in range(3):
        for (graph, _), stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(outs, wants):
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            for x in got:
                x.zero_()
        torch.cuda.synchronize()


def _by_rows(q, k, v, lengths):
    """y and lse row by row in float64, so that a row meets the keys it sees and no others: (value, bound) pairs
    with pair_ref's bounds, counted over what is finite."""
    dt = q.dtype
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    B, Hq, n, dk = q.shape
    G, dv = Hq // k.shape[1], v.shape[-1]
    y, yb = (torch.zeros(B, Hq, n, dv, dtype=torch.float64) for _ in range(2))
    lse, lb = torch.full((B, Hq, n), -math.inf, dtype=torch.float64), torch.zeros(B, Hq, n, dtype=torch.float64)
    for b, e in enumerate(lengths):
        for i in range(Hq):
            for t in range(e):
                K, V, x = k[b, i // G, :t + 1], v[b, i // G, :t + 1], q[b, i, t]
                s = K @ x / math.sqrt(dk)
                z = torch.logsumexp(s, 0)
                p = torch.exp(s - z)
                off = ((dk + 8) * 2.0 ** -23 / math.sqrt(dk) * (K.abs() @ x.abs())).masked_fill(p == 0, 0.0)
                y[b, i, t], lse[b, i, t] = p @ V, z
                rel = 2 * off + 2 * (p * off).sum() + (n + 32) * 2.0 ** -23
                yb[b, i, t] = pair_ref.HALF[dt] * y[b, i, t].abs() + (p * (1.01 * pair_ref.WEIGHT[dt] + rel)) @ V.abs() + 1e-30
                lb[b, i, t] = 2.0 ** -22 * z.abs() + (p * off).sum() + (n + 16) * 2.0 ** -23
    return (y, yb), (lse, lb)


# few workgroups, four waves a workgroup, and (bfloat16) eight
INFINITE = [("f32", 1, 2, 2, 150, 0), ("f32", 1, 2, 2, 150, 1), ("f32", 70, 1, 2, 70, 0), ("f32", 70, 1, 2, 70, 1),
            ("bf16", 1, 2, 2, 150, 0), ("bf16", 70, 1, 2, 70, 0), ("bf16", 256, 2, 1, 33, 0), ("bf16", 256, 2, 1, 33, 1)]


@pytest.mark.parametrize("dtype,H,G,B,end,offset", INFINITE)
def test_infinite_values(sata, dtype, H, G, B, end, offset):
    """An infinite entry of v is an infinity in its column of every row that sees it, and nowhere else; dv,
    which v does not enter, keeps its bits (from the same lse)."""
    n, at = end + 7, min(end - 20, 100)
    _say("softmax, infinite values", dtype, H, G, B, end, offset)
    q, k, v, dy = _prompt(31, B, H, G, n, 40, 24, dtype, offset=offset)
    lengths = [end] + [n] * (B - 1)
    y, lse = sata.softmax_prefill(q, k, v, _lengths(lengths))
    dv = sata.softmax_backward(q, k, v, y, lse, dy, _lengths(lengths))[2]
    v2 = v.clone() if not offset else _prompt(31, B, H, G, n, 40, 24, dtype, offset=offset)[2]
    v2[0, 0, at, 3], v2[0, 0, at - 3, 5] = math.inf, -math.inf
    y2, lse2 = sata.softmax_prefill(q, k, v2, _lengths(lengths))
    dv2 = sata.softmax_backward(q, k, v2, y2, lse, dy, _lengths(lengths))[2]
    torch.cuda.synchronize()
    want = y.clone()
    want[0, :G, at:end, 3], want[0, :G, at - 3:end, 5] = math.inf, -math.inf
    hit = torch.isinf(want)
    assert torch.equal(y2[hit], want[hit]) and torch.isfinite(y2[~hit]).all()
    off = (lse2 - lse)[0, :, :end].abs().max()
    assert off <= 1e-5 and torch.equal(dv2, dv)
    ry, rl = _by_rows(q[:1, :G], k[:1, :1], v2[:1, :1], lengths[:1])
    pair_ref.check(y2[:1, :G], ry, "y")
    pair_ref.check(lse2[:1, :G], rl, "lse")


@pytest.mark.parametrize("dtype,H,G,B,end,offset", INFINITE)
def test_keys_without_weight(sata, dtype, H, G, B, end, offset):
    """A key whose score is minus infinity has no weight: the rows that see it are those without it, and so
    are all gradients of k and v, its own being zero (0 times its infinity makes dq NaN)."""
    n, at = end + 7, min(end - 20, 100)
    _say("softmax, keys without weight", dtype, H, G, B, end, offset)
    q, k, v, dy = _prompt(32, B, H, G, n, 40, 24, dtype, offset=offset)
    q[..., 3] = -q[..., 3].abs() - 0.125
    lengths = [end] + [n] * (B - 1)
    k[0, 0, at, 3] = math.inf
    y, lse = sata.softmax_prefill(q, k, v, _lengths(lengths))
    grads = sata.softmax_backward(q, k, v, y, lse, dy, _lengths(lengths))
    torch.cuda.synchronize()
    ry, rl = _by_rows(q[:1, :G], k[:1, :1], v[:1, :1], lengths[:1])
    assert torch.isfinite(ry[0]).all()
    pair_ref.check(y[:1, :G], ry, "y")
    pair_ref.check(lse[:1, :G], rl, "lse")
    # a key of -2^60 in its place is the same, in finite numbers
    far = k.clone()
    far[0, 0, at, 3] = 2.0 ** 60
    want = pair_ref.softmax_backward(q[:1, :G], far[:1, :1], v[:1, :1], y[:1, :G], lse[:1, :G], dy[:1, :G], lengths[:1])
    for name, a, (w, bound) in zip(("dk", "dv"), grads[1:], want[1:]):
        assert not w[0, 0, at].any() and torch.isfinite(a).all(), name
        keep = torch.arange(n) != at
        pair_ref.check(a[:1, :1, keep], (w[:, :, keep], bound[:, :, keep]), name)
        assert not a[0, 0, at].any(), name
    assert torch.isfinite(grads[0][:1, :G, :at]).all()
    pair_ref.check(grads[0][:1, :G, :at], (want[0][0][:, :, :at], want[0][1][:, :, :at]), "dq")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_in_the_cache(sata, dtype):
    _say("softmax token, infinities in the cache", dtype)
    K, V, q, k, v = _rand(33, dtype, (2, 2, 900, 40), (2, 2, 900, 24), (2, 4, 40), (2, 2, 40), (2, 2, 24))
    q[..., 3] = -q[..., 3].abs() - 0.125
    K[0, 0, 77, 3] = math.inf          # no weight
    V[1, 1, 500, 7] = -math.inf        # an infinity in its column
    at = [860, 700]
    rows = lambda x, new: [torch.cat([x[b, :, :e], new[b, :, None]], 1)[None] for b, e in enumerate(at)]  # noqa: E731
    rK, rV = rows(K, k), rows(V, v)
    y = sata.softmax_step(K, V, _lengths(at), q, k, v)
    torch.cuda.synchronize()
    for b, e in enumerate(at):
        for h in range(4):
            s = rK[b][0, h // 2].double().cpu() @ q[b, h].double().cpu() / math.sqrt(40)
            p, vv = torch.softmax(s, 0), rV[b][0, h // 2].double().cpu()
            assert torch.isfinite(s).all() or (b, h // 2) == (0, 0)
            rel = 1.01 * pair_ref.WEIGHT[DT[dtype]] + (2 * 48 * 40 + e + 32) * 2.0 ** -23  # (|q||k| below 40)
            ref = p @ vv
            pair_ref.check(y[b, h], (ref, pair_ref.HALF[DT[dtype]] * ref.abs() + rel * (p @ vv.abs()) + 1e-30), f"y {b} {h}")
    assert torch.isneginf(y[1, 2:, 7]).all() and torch.isfinite(y[0]).all()


def test_largest_float32_values(sata):
    """Float32 numbers beyond bfloat16's largest (3.39e38) are numbers like others."""
    _say("softmax, largest values")
    n, at = 150, 70
    q, k, v, dy = _prompt(34, 1, 2, 1, n, 40, 24, "f32")
    v[0, 0, at, 3], v[0, 0, at, 4] = 3.4e38, -3.4e38
    q[..., 5] = 2.0 ** -125
    k[0, 1, at, 5] = 3.4e38            # (a score of 8 / sqrt(40))
    y, lse = sata.softmax_prefill(q, k, v)
    K, V = k.clone(), v.clone()
    last = sata.softmax_step(K, V, _lengths([n - 1]), q[:, :, -1].contiguous(), k[:, :, -1].contiguous(), v[:, :, -1].contiguous())
    torch.cuda.synchronize()
    ry, rl = _by_rows(q, k, v, [n])
    pair_ref.check(y, ry, "y")
    pair_ref.check(lse, rl, "lse")
    pair_ref.check(last, (ry[0][:, :, -1], ry[1][:, :, -1]), "token")


@pytest.mark.parametrize("G", [32, 33])
@pytest.mark.parametrize("dv", [127, 128])
@pytest.mark.parametrize("cap,end", [(100, 99), (3000, 2500)])
def test_token_of_wide_groups(sata, G, dv, cap, end):
    """The waves' sums of 32 query heads of 128 columns are 64 KB of LDS."""
    _say("softmax token, wide groups", G, dv, cap, end)
    K, V, q, k, v = _rand(35, "bf16", (1, 2, cap, 128), (1, 2, cap, dv), (1, 2 * G, 128), (1, 2, 128), (1, 2, dv))
    ry, rK, rV = pair_ref.softmax_step(K, V, [end], q, k, v)
    y = sata.softmax_step(K, V, _lengths([end]), q, k, v)
    torch.cuda.synchronize()
    pair_ref.check(y, ry, "y")
    assert torch.equal(K.cpu(), rK) and torch.equal(V.cpu(), rV)


def test_as_many_tokens_as_a_launch_holds(sata):
    """The largest prompts and gradients by their number of heads and tokens: a sequence of 70 tokens in the
    last head, none elsewhere."""
    _say("softmax, the largest launches")
    end, n = 70, 1 << 21
    for H, grads in ((953, False), (476, True)):
        last = _prompt(36, 1, 1, 1, end, 1, 1, "bf16")
        q, k, v, dy = (torch.zeros(H, 1, n, 1, dtype=torch.bfloat16, device="cuda") for _ in range(4))
        for x, part in zip((q, k, v, dy), last):
            x[-1:, :, :end] = part
        lens = torch.zeros(H, dtype=torch.int32, device="cuda")
        lens[-1] = end
        y, lse = sata.softmax_prefill(q, k, v, lens)
        torch.cuda.synchronize()
        ref_y, ref_lse = pair_ref.softmax_prefill(*last[:3])
        pair_ref.check(y[-1:, :, :end], ref_y, "y")
        pair_ref.check(lse[-1:, :, :end], ref_lse, "lse")
        assert not y[-1, :, end:].any() and not y[0].any() and torch.isneginf(lse[-1, :, end:]).all()
        if not grads:
            continue
        got = sata.softmax_backward(q, k, v, y, lse, dy, lens)
        torch.cuda.synchronize()
        want = pair_ref.softmax_backward(*last[:3], y[-1:, :, :end], lse[-1:, :, :end], last[3])
        for name, a, w in zip(("dq", "dk", "dv"), got, want):
            pair_ref.check(a[-1:, :, :end], w, name)
            assert not a[-1, :, end:].any() and not a[0].any()


@pytest.mark.parametrize("heads,n,d", [(1, 600, 128), (60, 600, 128), (180, 600, 128), (1, 600, 64), (60, 600, 64),
                                       (180, 600, 64), (1, 300, 32), (100, 300, 32), (260, 300, 32)])
def test_one_entry_a_row(sata, heads, n, d):
    """Inputs whose bounds feel every single key and query in bfloat16: few workgroups, four and eight waves."""
    _say("softmax, one entry a row", heads, n, d)
    one = pair_ref.one_entry_a_row(1, n, d, d)
    q, k, v, dy = (x.cuda().expand(1, heads, n, d).contiguous() for x in one)
    y, lse = sata.softmax_prefill(q, k, v)
    grads = sata.softmax_backward(q, k, v, y, lse, dy)
    torch.cuda.synchronize()
    ref_y, ref_lse = pair_ref.softmax_prefill(*one[:3])
    pair_ref.check(y[:, :1], ref_y, "y")
    pair_ref.check(lse[:, :1], ref_lse, "lse")
    want = pair_ref.softmax_backward(*one[:3], y[:, :1], lse[:, :1], one[3])
    for name, a, w in zip(("dq", "dk", "dv"), grads, want):
        pair_ref.check(a[:, :1], w, name)
    for x in (y, lse, *grads):  # all heads hold the same
        assert torch.equal(x, x[:, :1].expand_as(x))


@pytest.mark.parametrize("end", [31, 127, 128, 2047, 2900])
def test_token_of_one_entry_a_row(sata, end):
    """Nearly equal weights over values of one entry a row: a row of the cache lost or read twice is felt."""
    _say("softmax token, one entry a row", end)
    K, q, k = _rand(37, "bf16", (1, 2, 3000, 128), (1, 2, 128), (1, 2, 128))
    q *= 2.0 ** -6
    rows = pair_ref.one_entry_a_row(2, end + 1, 128, 128)[2].cuda()
    V = torch.full((1, 2, 3000, 128), math.nan, dtype=torch.bfloat16, device="cuda")
    V[:, :, :end] = rows[:, :, :end]
    v = rows[:, :, end].expand(1, 2, 128).contiguous()
    ref, _, _ = pair_ref.softmax_step(K, V, [end], q, k, v)
    # a weight is near 1 / (end + 1), the least entry 1/2, and the bound below that: a row more or less is beyond it
    assert ref[1].max() < 0.4 / (end + 1)
    y = sata.softmax_step(K, V, _lengths([end]), q, k, v)
    torch.cuda.synchronize()
    pair_ref.check(y, ref, "y")


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_values_that_are_not_finite_by_eight_waves(sata, bad):
    test_values_that_are_not_finite(sata, "bf16", bad, 256, 1)


@pytest.mark.parametrize("at", [100, 255, 256, 300])
def test_not_finite_in_later_blocks_of_eight_waves(sata, at):
    """NaN in the first or a later block of 256 rows, whose keys other blocks see whole."""
    _say("softmax by eight waves, NaN at", at)
    H, n = 256, 330
    q, k, v, dy = _prompt(38, 1, H, 1, n, 40, 24, "bf16")
    y, lse = sata.softmax_prefill(q, k, v)
    grads = sata.softmax_backward(q, k, v, y, lse, dy)
    ry, rl = pair_ref.softmax_prefill(q[:, :1], k[:, :1], v[:, :1])
    rg = pair_ref.softmax_backward(q[:, :1], k[:, :1], v[:, :1], y[:, :1], lse[:, :1], dy[:, :1])
    cut = lambda ref, rows: tuple(x[:, :, rows] for x in ref)  # noqa: E731
    before, behind = slice(0, at), slice(at + 1, n)
    for x in (1, 2):
        args = [q, k.clone(), v.clone()]
        args[x][0, 0, at, 3] = math.nan
        y2, lse2 = sata.softmax_prefill(*args)
        dq = sata.softmax_backward(*args, y2, lse2, dy)[0]
        torch.cuda.synchronize()
        for a, was in ((y2, y), (lse2, lse), (dq, grads[0])):
            assert torch.equal(a[:, 1:], was[:, 1:])
        pair_ref.check(y2[:, :1, before], cut(ry, before), "y")
        pair_ref.check(lse2[:, :1, before], cut(rl, before), "lse")
        pair_ref.check(dq[:, :1, before], cut(rg[0], before), "dq")
        assert torch.isnan(y2[0, 0, at:]).any(1).all() and torch.isnan(dq[0, 0, at:]).any(1).all()
    for x in (0, 1):
        args = [q.clone(), dy.clone()]
        args[x][0, 0, at, 3] = math.nan
        got = sata.softmax_backward(args[0], k, v, y, lse, args[1])
        torch.cuda.synchronize()
        for name, a, was, ref in zip(("dk", "dv"), got[1:], grads[1:], rg[1:]):
            assert torch.equal(a[:, 1:], was[:, 1:])
            pair_ref.check(a[:, :1, behind], cut(ref, behind), name)
        assert torch.isnan(got[1][0, 0, :at + 1]).any(1).all() and torch.isnan(got[2][0, 0, :at + 1]).any(1).all()


@pytest.mark.parametrize("B,H,G,cap,dk,dv,lengths", [(2, 2, 4, 300, 128, 128, [299, 100]), (1, 2, 3, 5000, 64, 40, [4321]),
                                                     (3, 2, 33, 700, 33, 100, [650, 3, 0])])
def test_token_weights_carry_fifteen_bits(sata, monkeypatch, B, H, G, cap, dk, dv, lengths):
    """A token's weights are two bfloat16 numbers in bfloat16 calls: cut off below 2^-7 + 2^-9 of the weight and then
    rounded by 2^-9 of that rest, 2^-15.6 in all."""
    _say("softmax token, fifteen bits", B, H, G, cap, dk, dv, lengths)
    monkeypatch.setitem(pair_ref.WEIGHT, torch.bfloat16, 2.0 ** -15)
    K, V, q, k, v = _rand(cap + 1, "bf16", (B, H, cap, dk), (B, H, cap, dv), (B, H * G, dk), (B, H, dk), (B, H, dv))
    ry, _, _ = pair_ref.softmax_step(K, V, lengths, q, k, v)
    y = sata.softmax_step(K, V, _lengths(lengths), q, k, v)
    torch.cuda.synchronize()
    pair_ref.check(y, ry, "y")
