"""A layer of the gated delta rule and one of softmax attention with rotary positions over caches of 4 bits an entry, as one would
train and serve them; and the calls that such a program makes that the operators' own tests do not: two graphs and two
streams at once, tensors beyond 2^31 entries, tensors that do not lie on whole vectors."""
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


def _attend(q, k, v):
    """Causal softmax attention of q [B, G*H, n, d], the last n of the tokens that k and v hold."""
    G, n, m = q.shape[1] // k.shape[1], q.shape[2], k.shape[2]
    k, v = (x.repeat_interleave(G, dim=1) for x in (k, v))
    s = (q[..., :, None, :] * k[..., None, :, :]).sum(-1) / math.sqrt(q.shape[-1])
    s = s.masked_fill(torch.ones(n, m, dtype=torch.bool).triu(m - n + 1), -math.inf)
    return (torch.softmax(s, -1)[..., None] * v[..., None, :, :]).sum(-2)


def _stack(q, k, v, g, beta, v2, at, freq):
    """float64: the delta rule's outputs are the queries of the attention, and the keys of both are the same."""
    y1, S, _ = ref.delta(q, k, v, g, beta)
    turned = [ref.rotary(x, at, freq, False, 1.0) for x in (y1, k)]
    return y1, turned, _attend(turned[0], turned[1], v2)


def test_stack(sata):
    B, H, G, n, steps, d = 2, 2, 2, 90, 4, 32
    print("stack of a delta layer and a softmax layer", file=sys.stderr, flush=True)
    q, k, v, g, beta, _ = ref.draw(5, B, H, G, n + steps, d, d, "f32")
    gen = torch.Generator().manual_seed(6)
    v2 = torch.randn(B, H, n + steps, d, generator=gen)
    dy = torch.randn(B, G * H, n, d, generator=gen)
    at = torch.arange(n + steps, dtype=torch.int32)[None] + torch.tensor([[0], [1000]], dtype=torch.int32)
    freq, scale = sata.rotary_frequencies(d // 2)
    assert scale == 1.0
    f64 = freq.double().cpu()
    y1, turned, y2 = _stack(*ref.to64(q, k, v, g, beta, v2), at, f64)

    # the prompt.  Each operator's float32 outputs are within 2e-5 of their norms (24-bit operands, sums of under 100 terms), and
    # scores of order one pass a query's error on at most as it is: 1e-4 for three of them in a row.
    dev = lambda x: x[:, :, :n].contiguous().cuda()  # noqa: E731
    Q, K, V, Gd, Be, V2 = (dev(x) for x in (q, k, v, g, beta, v2))
    pos = at[:, :n].contiguous().cuda()
    o1, S = sata.delta_prefill(Q, K, V, Gd, Be)
    tq, tk = sata.rotary(o1, K, pos, freq)
    o2, lse = sata.softmax_prefill(tq, tk, V2)
    torch.cuda.synchronize()
    for got, want in ((o1, y1), (tq, turned[0]), (tk, turned[1]), (o2, y2)):
        assert (got.double().cpu() - want[:, :, :n]).norm() <= 1e-4 * want[:, :, :n].norm()

    # gradients through all three (three times that: errors of the outputs and of each backward pass)
    DY = dy.cuda()
    dtq, dtk, dv2 = sata.softmax_backward(tq, tk, V2, o2, lse, DY)
    do1, dk2 = sata.rotary_backward(dtq, dtk, pos, freq)
    dq, dk1, dv, dg, db, _ = sata.delta_backward(Q, K, V, Gd, Be, do1)
    leaves = [x[:, :, :n].double().requires_grad_() for x in (q, k, v, g, beta, v2)]
    out = _stack(*leaves, at[:, :n], f64)[2]
    want = torch.autograd.grad((out * dy.double()).sum(), leaves)
    torch.cuda.synchronize()
    for name, a, w in zip("q k v g beta v2".split(), (dq, dk1 + dk2, dv, dg, db, dv2), want):
        assert (a.double().cpu() - w).norm() <= 3e-4 * w.norm(), name

    # tokens: the state, and caches of 4 bits an entry
    cap = n + steps + 3
    cK, cV = (torch.zeros(B, H, cap, sata.packed_row_bytes(d), dtype=torch.uint8, device="cuda") for _ in range(2))
    sata.packed_write(cK, cV, None, tk, V2)
    lengths = torch.full((B,), n, dtype=torch.int32, device="cuda")
    for t in range(n, n + steps):
        one = [x[:, :, t].contiguous().cuda() for x in (q, k, v, g, beta, v2)]
        p = at[:, t].contiguous().cuda()
        a1 = sata.delta_step(S, *one[:5])
        a1, kt = sata.rotary(a1, one[1], p, freq)
        a2 = sata.softmax_step_packed(cK, cV, lengths, a1, kt, one[5])
        lengths += 1
        assert (a1.double().cpu() - turned[0][:, :, t]).norm() <= 1e-4 * turned[0][:, :, t].norm()
        # what the caches' rows stand for: half a step of 15 to a group's span, its two numbers' roundings of 2^-8 and
        # the keys' own errors beside
        rows = [sata.packed_read(c, None, t + 1, d, torch.float32).double().cpu() for c in (cK, cV)]
        for r, x in zip(rows, (turned[1], v2.double())):
            x = x[:, :, :t + 1]
            span = x.amax(-1, keepdim=True) - x.amin(-1, keepdim=True)
            slack = span / 30 + 2.0 ** -8 * (span + x.abs().amax(-1, keepdim=True)) + 1e-4
            assert ((r - x).abs() <= slack).all()
        want = _attend(turned[0][:, :, t:t + 1], *rows)[:, :, 0]
        assert (a2.double().cpu() - want).norm() <= 1e-4 * want.norm()
    torch.cuda.synchronize()


def _serving(sata, seed, n, stream):
    """Everything of a program of its own: (run, its outputs, the inputs that change)."""
    with torch.cuda.stream(stream):
        q, k, v, g, beta, S0 = (x.cuda() for x in ref.draw(seed, 2, 2, 2, n, 64, 64, "bf16", state=True))
        dy = torch.ones_like(v)
        freq, _ = sata.rotary_frequencies(32)
        pos = torch.arange(n, dtype=torch.int32, device="cuda").repeat(2, 1)
        cK, cV = (torch.zeros(2, 2, 2000, sata.packed_row_bytes(64), dtype=torch.uint8, device="cuda") for _ in range(2))
        old = torch.randn(2, 2, 1500, 64, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()
        sata.packed_write(cK, cV, None, old, old.flip(1).contiguous())
        lengths = torch.tensor([1500, 700], dtype=torch.int32, device="cuda")
        stream.synchronize()

    def run():
        y, S = sata.delta_prefill(q, k, v, g, beta, S_in=S0)
        grads = sata.delta_backward(q, k, v, g, beta, dy, S_in=S0, dS=S)
        tq, tk = sata.rotary(y, k, pos, freq)
        token = [x[:, :, n - 1].contiguous() for x in (tq, tk, v[:, ::2])]
        return [y, S, tq, tk, sata.softmax_step_packed(cK, cV, lengths, *token), *grads]

    return run, (v, k)


def test_two_graphs_and_two_streams_at_once(sata):
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    programs = [_serving(sata, 11, 400, streams[0]), _serving(sata, 12, 333, streams[1])]
    graphs, outs = [], []
    for (run, _), s in zip(programs, streams):
        with torch.cuda.stream(s):
            run()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs.append(run())
        graphs.append(graph)
    for i in range(3):
        for (_, inputs), s in zip(programs, streams):
            with torch.cuda.stream(s):
                for x in inputs:
                    x.mul_(0.75)
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        got = [[x.clone() for x in o] for o in outs]
        torch.cuda.synchronize()
        eager = []
        for (run, _), s in zip(programs, streams):  # (both at once)
            with torch.cuda.stream(s):
                eager.append(run())
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            assert all(torch.equal(x, y) for x, y in zip(a, b)), i


def test_more_than_2_31_entries(sata):
    """A head behind 2^31 entries of the others gives what it gives alone."""
    H, n, d = 16, 2 ** 20 + 5, 128
    print("delta prompt of 2^31 entries", file=sys.stderr, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(1, H, n, d, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    for x in (q, k):
        x.mul_(d ** -0.5)
    g = torch.full((1, H, n), -0.1, device="cuda")
    beta = torch.full((1, H, n), 0.5, device="cuda")
    y, S = sata.delta_prefill(q, k, v, g, beta)
    last = [x[:, H - 1:].contiguous() for x in (q, k, v, g, beta)]
    y1, S1 = sata.delta_prefill(*last)
    assert torch.isfinite(y1).all() and torch.equal(y[:, H - 1:], y1) and torch.equal(S[:, H - 1:], S1)
    del y
    print("rotary of 2^31 entries", file=sys.stderr, flush=True)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    freq, _ = sata.rotary_frequencies(d // 2)
    tq, tk = sata.rotary(q, k, pos, freq)
    for a, x in ((tq, q), (tk, k)):
        assert torch.equal(a[:, H - 1:], sata.rotary(x[:, H - 1:].contiguous(), None, pos, freq)[0])


def test_gradients_of_more_than_2_31_entries_of_states(sata):
    H, n, d = 16, 2 ** 19 + 5, 128
    print("delta gradients with 2^31 entries of states", file=sys.stderr, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(4)
    q, k, v, dy = (torch.randn(1, H, n, d, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    for x in (q, k):
        x.mul_(d ** -0.5)
    g = torch.full((1, H, n), -0.1, device="cuda")
    beta = torch.full((1, H, n), 0.5, device="cuda")
    all_heads = sata.delta_backward(q, k, v, g, beta, dy)
    alone = sata.delta_backward(*(x[:, H - 1:].contiguous() for x in (q, k, v, g, beta, dy)))
    for a, b in zip(all_heads[:5], alone[:5]):
        assert torch.isfinite(b).all() and torch.equal(a[:, H - 1:], b)


def test_cache_of_more_than_2_31_bytes(sata):
    """The last head of the last sequence: 40 rows at the end of a cache whose others are zero, which count as keys and values of
    zero."""
    B, H, cap, d = 8, 8, 2 ** 19, 128
    print("cache of more than 2^31 bytes", file=sys.stderr, flush=True)
    K, V = (torch.zeros(B, H, cap, sata.packed_row_bytes(d), dtype=torch.uint8, device="cuda") for _ in range(2))
    assert K.numel() > 2 ** 31
    gen = torch.Generator().manual_seed(8)
    rows = torch.randn(2, B, H, 40, d, generator=gen)
    first = torch.full((B,), -40, dtype=torch.int32)
    first[-1] = cap - 41
    sata.packed_write(K, V, first.cuda(), rows[0].cuda(), rows[1].cuda())
    q, k, v = torch.randn(3, B, H, d, generator=gen)
    lengths = torch.full((B,), -1, dtype=torch.int32)
    lengths[-1] = cap - 1
    y = sata.softmax_step_packed(K, V, lengths.cuda(), q.cuda(), k.cuda(), v.cuda()).double().cpu()
    assert (y[:-1] == 0).all()
    stand = lambda x: torch.from_numpy(ref.pack(x.numpy())[1]).double()  # noqa: E731
    ks, vs = (torch.cat((stand(x), stand(one)[:, :, None]), 2)[-1] for x, one in ((rows[0], k), (rows[1], v)))
    last = sata.packed_read(K, torch.full((B,), cap - 41, dtype=torch.int32, device="cuda"), 41, d, torch.float32)
    assert torch.equal(last[-1].double().cpu(), ks) and (last[:-1] == 0).all()
    s = (ks * q[-1, :, None].double()).sum(-1) / math.sqrt(d)
    w = torch.exp(s)
    want = (w[..., None] * vs).sum(1) / (w.sum(-1, keepdim=True) + (cap - 41))
    # (a sum of 2^19 weights of about one, 2^-24 of it off for each of 2^11 sums behind one another at the most)
    size = (w[..., None] * vs.abs()).sum(1) / (cap - 41)
    assert ((y[-1] - want).abs() <= 2.0 ** -13 * size + 1e-12).all()


def _off(x, by=1):
    """x at an address `by` entries off a whole vector."""
    buf = torch.empty(x.numel() + by, dtype=x.dtype, device="cuda")
    buf[by:].copy_(x.reshape(-1))
    return buf[by:].view(x.shape)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,G,n,dk,dv", [(2, 2, 1, 100, 128, 128), (1, 1, 3, 70, 64, 32), (1, 2, 2, 65, 40, 72)])
def test_off_whole_vectors(sata, B, H, G, n, dk, dv, dtype):
    """Results do not depend on where the tensors lie."""
    q, k, v, g, beta, S = (x.cuda() for x in ref.draw(31, B, H, G, n, dk, dv, dtype, state=True))
    dy = v.flip(-1).contiguous()
    y, S1 = sata.delta_prefill(q, k, v, g, beta, S_in=S)
    grads = sata.delta_backward(q, k, v, g, beta, dy, S_in=S, dS=S1)
    o = [_off(x) for x in (q, k, v, g, beta)]
    y2, S2 = sata.delta_prefill(*o, S_in=_off(S), y=_off(torch.zeros_like(v)), S=_off(torch.zeros_like(S)))
    assert torch.equal(y, y2) and torch.equal(S1, S2)
    for a, b in zip(grads, sata.delta_backward(*o, _off(dy), S_in=_off(S), dS=_off(S1))):
        assert torch.equal(a, b)


def test_most_heads(sata):
    """65535 heads, the most that a call takes: some of them as alone, bit by bit; one more is refused."""
    most = 65535
    print("most heads", file=sys.stderr, flush=True)
    for B, Hk, G in ((most, 1, 1), (1, most // 3, 3)):
        q, k, v, g, beta, S = (x.cuda() for x in ref.draw(41, B, Hk, G, 2, 4, 3, "f32", state=True))
        y, S1 = sata.delta_prefill(q, k, v, g, beta, S_in=S)
        grads = sata.delta_backward(q, k, v, g, beta, v, S_in=S, dS=S1)
        S2 = S1.clone()
        tokens = [x[:, :, 1].contiguous() for x in (q, k, v, g, beta)]
        yt = sata.delta_step(S2, *tokens)
        for h in (0, 255, 256, most // G - 1):
            part = (slice(h, h + 1), slice(None)) if B > 1 else (slice(None), slice(h, h + 1))
            many = part if B > 1 else (slice(None), slice(G * h, G * h + G))
            a = [x[part].contiguous() for x in (q, k)] + [x[many].contiguous() for x in (v, g, beta)]
            o, T = sata.delta_prefill(*a, S_in=S[many].contiguous())
            assert torch.equal(o, y[many]) and torch.equal(T, S1[many])
            alone = sata.delta_backward(*a, a[2], S_in=S[many].contiguous(), dS=T)
            for i, (x, z) in enumerate(zip(alone, grads)):
                assert torch.equal(x, z[part if i < 2 else many]), (h, i)
            assert torch.equal(sata.delta_step(T, *(x[:, :, 1].contiguous() for x in a)), yt[many])
    x = torch.randn(1, most, 1, 8, device="cuda")
    pos = torch.full((1, 1), 7, dtype=torch.int32, device="cuda")
    freq, _ = sata.rotary_frequencies(4)
    tq, tk = sata.rotary(x, x, pos, freq)
    assert torch.equal(tq, tk) and torch.equal(tq[:, -1:], sata.rotary(x[:, -1:].contiguous(), None, pos, freq)[0])
    cK, cV = (torch.zeros(1, most, 3, sata.packed_row_bytes(8), dtype=torch.uint8, device="cuda") for _ in range(2))
    sata.packed_write(cK, cV, None, x, x)
    at = torch.ones(1, dtype=torch.int32, device="cuda")
    one = x[:, :, 0].contiguous()
    y = sata.softmax_step_packed(cK, cV, at, one, one, one)
    last = [c[:, -1:].contiguous() for c in (cK, cV)]
    assert torch.equal(y[:, -1:], sata.softmax_step_packed(*last, at, *(one[:, -1:].contiguous() for _ in range(3))))
    assert torch.equal(sata.packed_read(cK, None, 2, 8, torch.float32)[:, :, 0], sata.packed_read(cK, None, 2, 8, torch.float32)[:, :, 1])
    with pytest.raises(sata.SataError):
        z = torch.zeros(1, most + 1, 1, 8, device="cuda")
        sata.delta_prefill(z, z, z, z[..., 0].contiguous(), z[..., 0].contiguous())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_with_lengths_out_of_range(sata, dtype):
    q, k, v, g, beta, S = (x.cuda() for x in ref.draw(51, 3, 1, 2, 70, 16, 16, dtype, state=True))
    out = [sata.delta_backward(q, k, v, g, beta, v, lengths=torch.tensor(L, dtype=torch.int32, device="cuda"), S_in=S, dS=S)
           for L in ([-3, 1000, 66], [0, 70, 66])]
    for a, b in zip(*out):
        assert torch.equal(a, b)
    assert torch.equal(out[0][5][0], S[0])
