"""Caches of 4 bits an entry on the GPU: rows against a plain form bit by bit, tokens against softmax attention in
float64 over what the rows stand for."""
import math
import sys

import numpy as np
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


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _cache(sata, B, H, cap, d):
    return torch.full((B, H, cap, sata.packed_row_bytes(d)), 0xA5, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk,dv", [(128, 128), (64, 64), (32, 32), (1, 5), (33, 31), (40, 128), (96, 65), (127, 16)])
def test_rows(sata, dk, dv, dtype):
    """Written rows bit by bit, the others untouched; what they stand for."""
    print("rows", dk, dv, dtype, file=sys.stderr, flush=True)
    B, H, n, cap = 3, 2, 9, 14
    gen = torch.Generator().manual_seed(dk * 131 + dv)
    k, v = (torch.randn(B, H, n, d, generator=gen).to(_dtype(dtype)) for d in (dk, dv))
    k[0, 0, 0] = 1.5                       # no range at all
    k[0, 0, 1] = torch.arange(dk) % 16     # codes as they are
    k[0, 1, 2] *= 1e30
    v[0, 0, 3] = 0.0
    v[1, 0, 4] *= 1e-38
    first = torch.tensor([0, 5, -2], dtype=torch.int32)
    counts = torch.tensor([9, 20, 7], dtype=torch.int32)  # (20: as many as there are; rows behind the cache are left out)
    K, V = _cache(sata, B, H, cap, dk), _cache(sata, B, H, cap, dv)
    sata.packed_write(K, V, first.cuda(), k.cuda(), v.cuda(), counts=counts.cuda())
    for C, x, d in ((K, k, dk), (V, v, dv)):
        rows, values = ref.pack(x.float().numpy())
        want = np.full(tuple(C.shape), 0xA5, dtype=np.uint8)
        for b in range(B):
            for t in range(min(n, int(counts[b]))):
                if 0 <= first[b] + t < cap:
                    want[b, :, first[b] + t] = rows[b, :, t]
        assert np.array_equal(C.cpu().numpy(), want)
        got = sata.packed_read(C, first.cuda(), n, d, torch.float32).cpu()
        low = sata.packed_read(C, first.cuda(), n, d, torch.bfloat16).cpu()
        for b in range(B):
            for t in range(min(n, int(counts[b]))):
                w = torch.from_numpy(values[b, :, t]) if 0 <= first[b] + t < cap else torch.zeros(H, d)
                assert torch.equal(got[b, :, t], w), (b, t)
                assert torch.equal(low[b, :, t], w.bfloat16())


def test_one_tensor_without_first(sata):
    x = torch.randn(2, 1, 5, 48, generator=torch.Generator().manual_seed(1))
    K = _cache(sata, 2, 1, 5, 48)
    sata.packed_write(K, None, None, x.cuda(), None)
    assert np.array_equal(K.cpu().numpy(), ref.pack(x.numpy())[0])
    assert torch.equal(sata.packed_read(K, None, 5, 48, torch.float32).cpu(), torch.from_numpy(ref.pack(x.numpy())[1]))


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 1e37])
def test_not_finite(sata, value):
    """A group with an entry out of range stands for NaN, the others for what they are."""
    x = torch.randn(1, 1, 2, 100, generator=torch.Generator().manual_seed(2))
    x[0, 0, 0, 40] = value
    K = _cache(sata, 1, 1, 2, 100)
    sata.packed_write(K, None, None, x.cuda(), None)
    y = sata.packed_read(K, None, 2, 100, torch.float32).cpu()
    bad = torch.zeros(1, 1, 2, 100, dtype=torch.bool)
    bad[0, 0, 0, 32:64] = True
    assert torch.equal(torch.isnan(y), bad)
    assert np.array_equal(K.cpu().numpy(), ref.pack(x.numpy())[0])


def _attend(K, V, q, ends, dtype):
    """y and its bound: K, V [B, H, cap, d] float64 values with their groups' scales, rows 0..ends[b]."""
    (K, ks, km), (V, vs, vm) = K, V
    B, H, _, dk = K.shape
    G, dv = q.shape[1] // H, V.shape[-1]
    y, tol = torch.zeros(B, H * G, dv, dtype=torch.float64), torch.zeros(B, H * G, dv, dtype=torch.float64)
    eps, weight = (2.0 ** -8, 2.0 ** -16) if dtype == "bf16" else (2.0 ** -24, 2.0 ** -23)
    for b in range(B):
        e = ends[b]
        for h in range(H):
            for m in range(G):
                x = q[b, h * G + m].double()
                s = K[b, h, :e] @ x / math.sqrt(dk)
                p = torch.softmax(s, -1)
                y[b, h * G + m] = p @ V[b, h, :e]
                # sums over (16 + code) q and least values, in float32: some 80 roundings of their sizes a score, which
                # count twice in a weight; products with v of that weight's bits, and their sums
                size = ((31 + 16) * ks[b, h, :e] + km[b, h, :e]) @ x.abs() / math.sqrt(dk)
                off = weight + 2 * 80 * 2.0 ** -24 * size.max() + (40 + 2 * math.sqrt(e)) * 2.0 ** -24
                tol[b, h * G + m] = eps * y[b, h * G + m].abs() + off * (p @ ((31 + 16) * vs[b, h, :e] + vm[b, h, :e]))
    return y, tol


def _stands(x):
    """(values, scales, sizes of the least values) [.., d] float64 of rows made from x."""
    rows, values = ref.pack(x.float().numpy())
    d, groups = x.shape[-1], rows.shape[-1] // 20
    p = torch.from_numpy(rows[..., 16 * groups:].copy()).view(torch.bfloat16).double()
    each = lambda j: p[..., j::2].repeat_interleave(32, dim=-1)[..., :d]  # noqa: E731
    return torch.from_numpy(values).double(), each(0).abs(), each(1).abs()


STEPS = [  # B, H, G, cap, dk, dv, dtype
    (2, 3, 1, 100, 64, 64, "bf16"),
    (3, 2, 4, 333, 128, 128, "bf16"),
    (2, 2, 3, 257, 40, 24, "f32"),
    (1, 1, 1, 1, 128, 128, "f32"),
    (4, 1, 8, 600, 32, 128, "bf16"),
    (2, 1, 17, 140, 96, 64, "bf16"),     # two blocks of query heads
    (2, 1, 40, 300, 128, 32, "f32"),
    (1, 2, 2, 3000, 128, 128, "bf16"),
    (1, 1, 16, 2500, 16, 8, "f32"),
    (2, 4, 2, 70, 7, 1, "bf16"),
]


@pytest.mark.parametrize("case", STEPS, ids=str)
def test_token(sata, case):
    B, H, G, cap, dk, dv, dtype = case
    print("token", case, file=sys.stderr, flush=True)
    gen = torch.Generator().manual_seed(cap + dk + G)
    dt = _dtype(dtype)
    old = [torch.randn(B, H, cap, d, generator=gen).to(dt) for d in (dk, dv)]
    q, k, v = (torch.randn(B, h, d, generator=gen).to(dt) for h, d in ((H * G, dk), (H, dk), (H, dv)))
    K, V = _cache(sata, B, H, cap, dk), _cache(sata, B, H, cap, dv)
    sata.packed_write(K, V, None, old[0].cuda(), old[1].cuda())
    # sequences of all kinds: full but for the new row, one old row, none, some
    ends = [cap - 1, 0, cap // 2, min(cap - 1, 1)][:B]
    lengths = torch.tensor(ends, dtype=torch.int32)
    for b, e in enumerate(ends):  # rows behind a sequence's are not used: NaN groups
        K[b, :, e:], V[b, :, e:] = 0xFF, 0xFF
    before = K.clone(), V.clone()
    y = sata.softmax_step_packed(K, V, lengths.cuda(), q.cuda(), k.cuda(), v.cuda())
    for C, was, x, row in ((K, before[0], old[0], k), (V, before[1], old[1], v)):
        want = was.cpu().numpy()
        for b, e in enumerate(ends):
            want[b, :, e] = ref.pack(row[b].float().numpy())[0]
            x[b, :, e] = row[b]
        assert np.array_equal(C.cpu().numpy(), want)
    want, tol = _attend(_stands(old[0]), _stands(old[1]), q, [e + 1 for e in ends], dtype)
    err = (y.double().cpu() - want).abs()
    assert (err <= tol).all(), (err / tol).max()


def test_idle_and_empty_sequences(sata):
    B, H, G, cap, d = 4, 2, 2, 50, 32
    gen = torch.Generator().manual_seed(3)
    K, V = _cache(sata, B, H, cap, d), _cache(sata, B, H, cap, d)
    lengths = torch.tensor([-1, cap, 0, 2 ** 31 - 1], dtype=torch.int32)
    q, k, v = (torch.randn(B, h, d, generator=gen) for h in (H * G, H, H))
    y = sata.softmax_step_packed(K, V, lengths.cuda(), q.cuda(), k.cuda(), v.cuda()).cpu()
    assert (y[[0, 1, 3]] == 0).all()
    assert (K[[0, 1, 3]] == 0xA5).all() and (V[[0, 1, 3]] == 0xA5).all()
    # the first token sees itself alone
    want = torch.from_numpy(ref.pack(v[2].numpy())[1]).repeat_interleave(G, dim=0)
    assert (y[2] - want).abs().max() <= 64 * 2.0 ** -24 * 4


def test_bad_rows_stay_in_their_sequences_and_heads(sata):
    """A row that stands for NaN makes NaN of its own head's outputs: of all columns by a key, of its group's by a value."""
    B, H, cap, d = 2, 2, 200, 64
    gen = torch.Generator().manual_seed(4)
    k, v = torch.randn(2, B, H, cap, d, generator=gen)
    k[0, 0, 150, 3] = math.nan
    v[1, 1, 20, 40] = math.inf
    K, V = _cache(sata, B, H, cap, d), _cache(sata, B, H, cap, d)
    sata.packed_write(K, V, None, k.cuda(), v.cuda())
    lengths = torch.tensor([199, 199], dtype=torch.int32).cuda()
    q, kn, vn = torch.randn(3, B, H, d, generator=gen).cuda()
    y = sata.softmax_step_packed(K, V, lengths, q, kn, vn).cpu()
    bad = torch.zeros(B, H, d, dtype=torch.bool)
    bad[0, 0] = True
    bad[1, 1, 32:] = True
    assert torch.equal(torch.isnan(y), bad)


def test_many_sequences(sata):
    """More sequences than the card's stretches are cut by: 400 of one head, lengths of all sizes."""
    B, cap, d = 400, 900, 32
    gen = torch.Generator().manual_seed(5)
    old = torch.randn(2, B, 1, cap, d, generator=gen)
    K, V = _cache(sata, B, 1, cap, d), _cache(sata, B, 1, cap, d)
    sata.packed_write(K, V, None, old[0].cuda(), old[1].cuda())
    lengths = torch.arange(B, dtype=torch.int32) * 2
    q, k, v = torch.randn(3, B, 1, d, generator=gen)
    y = sata.softmax_step_packed(K, V, lengths.cuda(), q.cuda(), k.cuda(), v.cuda()).cpu().double()
    pick = [0, 1, 64, 201, 399]
    K64, V64 = (x[pick].clone() for x in old)
    for i, b in enumerate(pick):
        K64[i, :, lengths[b]], V64[i, :, lengths[b]] = k[b], v[b]
    want, tol = _attend(_stands(K64), _stands(V64), q[pick], [int(lengths[b]) + 1 for b in pick], "f32")
    assert ((y[pick] - want).abs() <= tol).all()


def test_captured_with_lengths_that_change(sata):
    """One graph for all tokens; replayed, each gives what the call gives."""
    B, H, G, cap, d = 2, 2, 2, 600, 64
    gen = torch.Generator().manual_seed(6)
    old = torch.randn(2, B, H, cap, d, generator=gen).bfloat16().cuda()
    K, V = _cache(sata, B, H, cap, d), _cache(sata, B, H, cap, d)
    sata.packed_write(K, V, None, old[0], old[1])
    q, k, v = (torch.randn(B, h, d, generator=gen).bfloat16().cuda() for h in (H * G, H, H))
    lengths = torch.tensor([3, 500], dtype=torch.int32, device="cuda")
    y = torch.empty_like(q)
    sata.softmax_step_packed(K, V, lengths, q, k, v, y=y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sata.softmax_step_packed(K, V, lengths, q, k, v, y=y)
    for i in range(4):
        q.mul_(0.9)
        k.add_(0.01)
        lengths.add_(7)
        other = K.clone(), V.clone()
        graph.replay()
        want = sata.softmax_step_packed(*other, lengths, q, k, v)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(K, other[0]) and torch.equal(V, other[1])


def test_other_stream(sata):
    s = torch.cuda.Stream()
    x = torch.randn(1, 2, 300, 128, generator=torch.Generator().manual_seed(7)).cuda()
    K = _cache(sata, 1, 2, 300, 128)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        sata.packed_write(K, None, None, x, None)
        y = sata.packed_read(K, None, 300, 128, torch.float32)
    s.synchronize()
    assert torch.equal(y.cpu(), torch.from_numpy(ref.pack(x.cpu().numpy())[1]))


def test_refusals(sata):
    K = _cache(sata, 1, 2, 10, 64)
    q, k = torch.zeros(1, 2, 64, device="cuda"), torch.zeros(1, 2, 64, device="cuda")
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(sata.SataError):
        sata.softmax_step_packed(K, K, at, q, k, k)
    with pytest.raises(ValueError):
        sata.softmax_step_packed(K, _cache(sata, 1, 2, 11, 64), at, q, k, k)
    with pytest.raises(ValueError):
        sata.softmax_step_packed(K, _cache(sata, 1, 2, 10, 32), at, q, k, k)
    with pytest.raises(TypeError):
        sata.softmax_step_packed(K.char(), K.char(), at, q, k, k)
    with pytest.raises(ValueError):
        sata.packed_write(K, None, None, torch.zeros(1, 2, 3, 65, device="cuda"), None)
    with pytest.raises(ValueError):
        sata.packed_read(K, None, -1, 64, torch.float32)
    with pytest.raises(ValueError):
        sata.packed_row_bytes(129)
    buf = torch.zeros(1 + K.numel(), dtype=torch.uint8, device="cuda")
    odd = buf[1:].view(K.shape)
    with pytest.raises(sata.SataError):
        sata.packed_read(odd, None, 1, 64, torch.float32)
