"""Decayed linear attention and softmax attention on the CPU: the float64
references against recurrences, autograd of another formulation and differences,
and what the calls refuse."""
import ctypes
import math

import pytest

import pair_ref
from paper_2602_00294_amd import _binding as bnd

torch = pytest.importorskip("torch")

NULL = ctypes.c_void_p(None)
FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first


def _inputs(seed, B, H, G, n, dk, dv):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    return (r(B, H * G, n, dk), r(B, H, n, dk), r(B, H, n, dv), r(B, H * G, n, dv), r(B, H, dk, dv), r(B, H, dk, dv),
            -torch.rand(H, generator=g, dtype=torch.float64))


@pytest.fixture(autouse=True)
def _f64(monkeypatch):
    for table in (pair_ref.HALF, pair_ref.WEIGHT):
        monkeypatch.setitem(table, torch.float64, 2.0 ** -50)


def _recurrence(q, k, v, g, S, end):
    """Token by token, differentiable."""
    G = q.shape[0]
    rows = []
    for t in range(end):
        S = torch.exp(g) * S + k[t][:, None] * v[t][None, :]
        rows.append((q[:, t] @ S) / math.sqrt(q.shape[-1]))
    n = q.shape[1]
    y = torch.stack(rows, 1) if rows else q.new_zeros(G, 0, v.shape[-1])
    return torch.cat([y, y.new_zeros(G, n - end, v.shape[-1])], 1), S


@pytest.mark.parametrize("n,lengths", [(7, None), (6, [0, 1, 6])])
def test_decay_reference(n, lengths):
    B, H, G, dk, dv = (len(lengths) if lengths else 1), 2, 2, 3, 4
    q, k, v, dy, S0, dS, g = _inputs(1, B, H, G, n, dk, dv)
    leaves = [x.clone().requires_grad_() for x in (q, k, v, S0)]
    ends = lengths or [n] * B
    ys, Ss = [], []
    for b in range(B):
        for h in range(H):
            y, S = _recurrence(leaves[0][b, h * G:(h + 1) * G], leaves[1][b, h], leaves[2][b, h], g[h], leaves[3][b, h],
                               ends[b])
            ys.append(y)
            Ss.append(S)
    y, S = torch.cat(ys).view(B, H * G, n, dv), torch.stack(Ss).view(B, H, dk, dv)
    grads = torch.autograd.grad((y * dy).sum() + (S * dS).sum(), leaves)
    ry, rS = pair_ref.decay_prefill(q, k, v, g, lengths, S0)
    assert torch.allclose(ry[0], y, atol=1e-12) and torch.allclose(rS[0], S, atol=1e-12)
    for got, want in zip(pair_ref.decay_backward(q, k, v, g, dy, lengths, S0, dS), grads):
        assert torch.allclose(got[0], want, atol=1e-12)
    # one token more, by the step
    (y1, _), (S1, _) = pair_ref.decay_step(S, q[:, :, 0], k[:, :, 0], v[:, :, 0], g)
    for b in range(B):
        for h in range(H):
            a, c = _recurrence(q[b, h * G:(h + 1) * G, :1], k[b, h, :1], v[b, h, :1], g[h], S[b, h], 1)
            assert torch.allclose(y1[b, h * G:(h + 1) * G], a[:, 0]) and torch.allclose(S1[b, h], c)


def test_decay_of_minus_infinity():
    q, k, v, _, S0, _, _ = _inputs(2, 1, 1, 1, 5, 3, 2)
    g = torch.tensor([-math.inf])
    (y, _), (S, _) = pair_ref.decay_prefill(q, k, v, g, None, S0)
    assert torch.allclose(y, (q * k).sum(-1, keepdim=True) * v / math.sqrt(3))
    assert torch.allclose(S[0, 0], k[0, 0, 4][:, None] * v[0, 0, 4])


@pytest.mark.parametrize("lengths", [None, [0, 1, 6]])
def test_softmax_reference(lengths):
    B, H, G, n, dk, dv = (len(lengths) if lengths else 1), 2, 2, 6, 3, 4
    q, k, v, dy, *_ = _inputs(3, B, H, G, n, dk, dv)
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    ends = lengths or [n] * B
    y = torch.zeros(B, H * G, n, dv, dtype=torch.float64)
    for b in range(B):
        for i in range(H * G):
            for t in range(ends[b]):
                s = leaves[1][b, i // G, :t + 1] @ leaves[0][b, i, t] / math.sqrt(dk)
                y[b, i, t] = torch.softmax(s, 0) @ leaves[2][b, i // G, :t + 1]
    grads = torch.autograd.grad((y * dy).sum(), leaves)
    (ry, _), (lse, _) = pair_ref.softmax_prefill(q, k, v, lengths)
    assert torch.allclose(ry, y, atol=1e-12)
    for b in range(B):
        assert torch.isinf(lse[b, :, ends[b]:]).all() and torch.isfinite(lse[b, :, :ends[b]]).all()
    for got, want in zip(pair_ref.softmax_backward(q, k, v, ry, lse, dy, lengths), grads):
        assert torch.allclose(got[0], want, atol=1e-12)
    # the last token of each sequence, by the step
    K, V = k.clone(), v.clone()
    at = torch.tensor([e - 1 for e in ends], dtype=torch.int32)
    pick = lambda x: torch.stack([x[b, :, max(e - 1, 0)] for b, e in enumerate(ends)])  # noqa: E731
    (y1, _), _, _ = pair_ref.softmax_step(K, V, at, pick(q), pick(k), pick(v))
    for b, e in enumerate(ends):
        assert torch.allclose(y1[b], y[b, :, e - 1].detach() if e else torch.zeros(H * G, dv, dtype=torch.float64))


@pytest.mark.parametrize("which", ["decay", "softmax"])
def test_gradients_by_differences(which):
    B, H, G, n, dk, dv = 1, 1, 2, 5, 3, 2
    q, k, v, dy, S0, dS, g = _inputs(4, B, H, G, n, dk, dv)
    if which == "decay":
        def loss(q, k, v, S0):
            (y, _), (S, _) = pair_ref.decay_prefill(q, k, v, g, None, S0)
            return ((y * dy).sum() + (S * dS).sum()).item()
        args, grads = [q, k, v, S0], [x[0] for x in pair_ref.decay_backward(q, k, v, g, dy, None, S0, dS)]
    else:
        def loss(q, k, v):
            return (pair_ref.softmax_prefill(q, k, v)[0][0] * dy).sum().item()
        (y, _), (lse, _) = pair_ref.softmax_prefill(q, k, v)
        args, grads = [q, k, v], [x[0] for x in pair_ref.softmax_backward(q, k, v, y, lse, dy)]
    step = 1e-5  # the differences are off by step^2 times a third derivative, and by 2^-52 / step
    for at, (x, gx) in enumerate(zip(args, grads)):
        for j in range(x.numel()):
            moved = []
            for sign in (1, -1):
                y = x.clone()
                y.view(-1)[j] += sign * step
                moved.append(loss(*args[:at], y, *args[at + 1:]))
            assert abs((moved[0] - moved[1]) / (2 * step) - gx.reshape(-1)[j].item()) < 1e-7, (which, at, j)


@pytest.mark.parametrize("n,d", [(600, 128), (600, 64), (300, 32)])
def test_bfloat16_bounds_feel_every_pair(n, d):
    """With one entry a row the bounds of bfloat16 results tell a key lost, or one seen too early, at any place of
    any row: for dv every pair of a query and a key, for the others all but a few, where a row's few keys hold nearly the
    same as the one lost or added, or a pair's term is nearly zero."""
    q, k, v, dy = pair_ref.one_entry_a_row(1, n, d, d)
    (y, y_bound), (lse, _) = pair_ref.softmax_prefill(q, k, v)
    grads = pair_ref.softmax_backward(q, k, v, y.bfloat16(), lse.float(), dy)
    Q, K, V, Y = (x[0, 0].double() for x in (q, k, v, dy))
    t, c = torch.arange(n), 1 / math.sqrt(d)
    col = t % d
    p = torch.exp(Q @ K.T * c - lse[0, 0][:, None])
    # a row without its key s, or with one behind it: the weights of the others change with it
    was, add = y[0, 0][:, col], V[t, col]
    now = torch.where(t[:, None] >= t[None, :], (was - p * add) / (1 - p), (was + p * add) / (1 + p))
    now[0, 0] = math.inf  # (a row without its only key)
    assert ((now - was).abs() > y_bound[0, 0][:, col]).double().mean() > 0.9999
    e = c * p * (Y @ V.T - (Y * y[0, 0]).sum(1, keepdim=True))
    felt = [((term.abs() > bound[0, 0][:, col]).double().mean().item())
            for term, (_, bound) in zip((e * K[t, col], e.T * Q[t, col], p.T * Y[t, col]), grads)]
    assert felt[0] > 0.999 and felt[1] > 0.96 and felt[2] == 1.0, felt


# ------------------------------------------------------------------ refusals

SIZES = [  # (dtype, B, H_kv, G, n, d_k, d_v), status
    ((7, 1, 1, 1, 8, 4, 4), -1), ((0, 0, 1, 1, 8, 4, 4), -1), ((0, 1, 0, 1, 8, 4, 4), -1), ((0, 1, 1, 0, 8, 4, 4), -1),
    ((0, 1, 1, 1, -1, 4, 4), -1), ((0, 1, 1, 1, 8, 0, 4), -1), ((0, 1, 1, 1, 8, 4, 0), -1),
    ((0, 1, 1, 1, 8, 129, 4), -2), ((1, 1, 1, 1, 8, 4, 129), -2), ((1, 64, 128, 8, 8, 4, 4), -3),
    ((0, 2 ** 30, 2 ** 30, 2 ** 30, 8, 4, 4), -3), ((0, 1, 1, 1, 2 ** 21 + 1, 4, 4), -3),
]


@pytest.fixture(scope="module")
def lib():
    return bnd.load_library()


@pytest.mark.parametrize("sizes,code", SIZES)
def test_sizes_refused(lib, sizes, code):
    dt, B, H, G, n, dk, dv = sizes
    F = FAKE
    calls = [lib.sata_decay_prefill(F, F, F, F, *sizes, NULL, NULL, F, NULL, F, NULL),
             lib.sata_decay_backward(F, F, F, F, F, *sizes, NULL, NULL, NULL, F, F, F, NULL, F, NULL),
             lib.sata_softmax_prefill(F, F, F, *sizes, NULL, F, F, NULL),
             lib.sata_softmax_backward(F, F, F, F, F, F, *sizes, NULL, F, F, F, F, NULL),
             lib.sata_softmax_step(F, F, n, F, F, F, F, dt, B, H, G, dk, dv, F, F, NULL)]
    if n == 8:
        calls.append(lib.sata_decay_step(F, F, F, F, F, dt, B, H, G, dk, dv, F, NULL))
    assert calls == [code] * len(calls)
    assert lib.sata_last_error().decode() != ""


def test_pointers_refused(lib):
    F, N = FAKE, NULL
    ok = (0, 1, 1, 1, 8, 4, 4)
    for at in range(4):
        p = [F] * 4
        p[at] = N
        assert lib.sata_decay_prefill(*p, *ok, N, N, F, N, F, N) == -1
    assert lib.sata_decay_prefill(F, F, F, F, *ok, N, N, N, N, F, N) == -1
    assert lib.sata_decay_prefill(F, F, F, F, *ok, N, F, F, F, F, N) == -1      # S_out is S_in
    for at in range(5):
        p = [F] * 5
        p[at] = N
        assert lib.sata_decay_backward(*p, *ok, N, N, N, F, F, F, N, F, N) == -1
    assert lib.sata_decay_backward(F, F, F, F, F, *ok, N, N, F, F, F, F, F, F, N) == -1  # dS_in is dS
    assert lib.sata_decay_backward(F, F, F, F, F, *ok, N, N, N, F, N, F, N, F, N) == -1
    for at in range(5):
        p = [F] * 5
        p[at] = N
        assert lib.sata_decay_step(*p, 0, 1, 1, 1, 4, 4, F, N) == -1
    assert lib.sata_softmax_prefill(F, N, F, *ok, N, F, N, N) == -1
    for at in range(6):
        p = [F] * 6
        p[at] = N
        assert lib.sata_softmax_backward(*p, *ok, N, F, F, F, F, N) == -1
    assert lib.sata_softmax_backward(F, F, F, F, F, F, *ok, N, F, F, N, F, N) == -1
    assert lib.sata_softmax_step(F, F, 8, N, F, F, F, 0, 1, 1, 1, 4, 4, F, F, N) == -1
    assert lib.sata_softmax_step(F, F, 0, F, F, F, F, 0, 1, 1, 1, 4, 4, F, F, N) == -1
    # no tokens: nothing to do without a state
    empty = (0, 1, 1, 1, 0, 4, 4)
    assert lib.sata_decay_prefill(N, N, N, F, *empty, N, N, N, N, N, N) == 0
    assert lib.sata_decay_backward(N, N, N, F, N, *empty, N, N, N, N, N, N, N, N, N) == 0
    assert lib.sata_softmax_prefill(N, N, N, *empty, N, N, N, N) == 0
    assert lib.sata_softmax_backward(N, N, N, N, N, N, *empty, N, N, N, N, N, N) == 0


def test_more_tokens_than_a_launch_holds(lib):
    """A launch has fewer than 2^32 threads; softmax prompts take two a query and gradients four a key."""
    F, N = FAKE, NULL
    big = 2 ** 21
    prompt = lambda B, H, G, n: lib.sata_softmax_prefill(F, F, F, 1, B, H, G, n, 1, 1, N, N if n == 0 else F, F, N)  # noqa: E731
    # (null scratch: refused next, so that nothing is launched)
    grads = lambda B, H, G, n: lib.sata_softmax_backward(F, F, F, F, F, F, 1, B, H, G, n, 1, 1, N, F, F, F, N, N)  # noqa: E731
    too_large = lambda got: got == -3 and "tokens" in lib.sata_last_error().decode()  # noqa: E731
    for B, H, G, n in ((1, 954, 1, big), (2, 10, 100, 1000001), (65535, 1, 1, 30519), (5, 1, 13107, 32768)):
        assert B * H * G * n > 2 * 10 ** 9 and too_large(prompt(B, H, G, n)) and too_large(grads(B, H, G, n))
        assert lib.sata_softmax_backward_scratch(B, H, G, n) == -1
    for B, H, G, n in ((1, 477, 1, big), (500, 2, 2, 1000001), (65535, 1, 1, 15260)):
        assert B * H * n > 10 ** 9 and too_large(grads(B, H, G, n))
        assert lib.sata_softmax_backward_scratch(B, H, G, n) == -1
    for B, H, G, n in ((1, 476, 2, big), (1, 1, 953, big), (65535, 1, 1, 15258)):
        assert B * H * n <= 10 ** 9 and B * H * G * n <= 2 * 10 ** 9
        assert grads(B, H, G, n) == -1 and "scratch" in lib.sata_last_error().decode()
        assert lib.sata_softmax_backward_scratch(B, H, G, n) == 4 * B * H * G * n


def test_states_that_alias(lib):
    """One workgroup would write dS_in while another reads S_in or dS."""
    F, N = FAKE, NULL
    A, B, C = (ctypes.c_void_p(0x1000 * i) for i in (2, 3, 4))
    for sizes in ((0, 1, 1, 1, 8, 4, 4), (1, 2, 3, 2, 4096, 64, 32)):
        assert lib.sata_decay_backward(F, F, F, F, F, *sizes, N, A, B, F, F, F, A, F, N) == -1
        assert "S_in" in lib.sata_last_error().decode()
        assert lib.sata_decay_backward(F, F, F, F, F, *sizes, N, A, B, F, F, F, B, F, N) == -1
    # (other states: only the missing scratch is in the way)
    assert lib.sata_decay_backward(F, F, F, F, F, *sizes, N, A, B, F, F, F, C, N, N) == -1
    assert "scratch" in lib.sata_last_error().decode()


def test_scratch(lib):
    F, N = FAKE, NULL
    odd = ctypes.c_void_p(0x1008)
    # long heads and few of them work in parts, and long caches in stretches, whose sums need room
    assert lib.sata_decay_scratch(1, 2, 1, 4096, 64, 32) > 0 and lib.sata_decay_scratch(64, 64, 1, 4096, 64, 32) == 0
    assert lib.sata_softmax_backward_scratch(2, 3, 4, 5) == 4 * 2 * 3 * 4 * 5
    assert lib.sata_softmax_step_scratch(1, 2, 4, 8192, 64) > 0 and lib.sata_softmax_step_scratch(64, 64, 1, 256, 64) == 0
    for bad in ((0, 1, 1, 1, 1, 1), (1, 1, 1, -1, 1, 1), (1, 1, 1, 1, 129, 1), (1, 65536, 1, 1, 1, 1), (1, 1, 0, 1, 1, 1)):
        assert lib.sata_decay_scratch(*bad) == -1
    assert lib.sata_softmax_backward_scratch(1, 1, 0, 5) == -1
    assert lib.sata_softmax_step_scratch(1, 1, 1, 0, 5) == -1
    sizes = (0, 1, 2, 1, 4096, 64, 32)
    for s in (N, odd):
        assert lib.sata_decay_prefill(F, F, F, F, *sizes, N, N, F, N, s, N) == -1
        assert lib.sata_decay_backward(F, F, F, F, F, *sizes, N, N, N, F, F, F, N, s, N) == -1
        assert lib.sata_softmax_backward(F, F, F, F, F, F, *sizes, N, F, F, F, s, N) == -1
        assert lib.sata_softmax_step(F, F, 8192, F, F, F, F, 0, 1, 2, 1, 64, 64, F, s, N) == -1
        assert "scratch" in lib.sata_last_error().decode()


class TestBindingRefuses:
    """Types and shapes are checked before the device, which CPU tensors fail last."""

    def t(self, *shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=dtype)

    def prompt(self):
        return self.t(2, 6, 8, 4), self.t(2, 3, 8, 4), self.t(2, 3, 8, 5)

    def test_prompts(self):
        q, k, v = self.prompt()
        g, i32, bf = self.t(3), torch.int32, torch.bfloat16
        dy, y, lse = self.t(2, 6, 8, 5), self.t(2, 6, 8, 5), self.t(2, 6, 8)
        st = self.t(2, 3, 4, 5)
        for call, extra in ((lambda *a, **x: bnd.decay_prefill(*a, g, **x), {}),
                            (lambda *a, **x: bnd.decay_backward(*a, g, dy, **x), {}),
                            (bnd.softmax_prefill, {}),
                            (lambda *a, **x: bnd.softmax_backward(*a, y, lse, dy, **x), {})):
            with pytest.raises(TypeError):
                call(q, k.to(bf), v)
            with pytest.raises(TypeError):
                call(q.half(), k.half(), v.half())
            with pytest.raises(ValueError):
                call(q[:, :5], k, v)
            with pytest.raises(ValueError):
                call(q, k[:, :, :7], v)
            with pytest.raises(ValueError):
                call(q[0], k, v)
            with pytest.raises(TypeError):
                call(q, k, v, lengths=self.t(2))
            with pytest.raises(ValueError):
                call(q, k, v, lengths=self.t(3, dtype=i32))
            with pytest.raises(ValueError, match="GPU"):
                call(q, k, v, lengths=self.t(2, dtype=i32))
        with pytest.raises(ValueError):
            bnd.decay_prefill(q, k, v, self.t(2))
        with pytest.raises(TypeError):
            bnd.decay_prefill(q, k, v, g.double())
        with pytest.raises(ValueError):
            bnd.decay_prefill(q, k, v, g, S_in=self.t(2, 3, 5, 4))
        with pytest.raises(TypeError):
            bnd.decay_prefill(q, k, v, g, S=st.to(bf))
        with pytest.raises(ValueError):
            bnd.decay_prefill(q, k, v, g, y=self.t(2, 3, 8, 5))
        with pytest.raises(ValueError):
            bnd.decay_backward(q, k, v, g, dy[:, :, :7])
        with pytest.raises(ValueError):
            bnd.decay_backward(q, k, v, g, dy, dS=self.t(2, 6, 4, 5))
        with pytest.raises(ValueError):
            bnd.softmax_backward(q, k, v, y, lse[:, :3], dy)
        with pytest.raises(TypeError):
            bnd.softmax_backward(q, k, v, y, lse.to(bf), dy)
        with pytest.raises(TypeError):
            bnd.softmax_backward(q, k, v, y.to(bf), lse, dy)

    def test_tokens(self):
        q, k, v, g = self.t(2, 6, 4), self.t(2, 3, 4), self.t(2, 3, 5), self.t(3)
        S, K, V, at = self.t(2, 3, 4, 5), self.t(2, 3, 9, 4), self.t(2, 3, 9, 5), self.t(2, dtype=torch.int32)
        with pytest.raises(ValueError):
            bnd.decay_step(S[:, :, :3], q, k, v, g)
        with pytest.raises(TypeError):
            bnd.decay_step(S.double(), q, k, v, g)
        with pytest.raises(ValueError):
            bnd.decay_step(S, q[:, :4], k, v, g)
        with pytest.raises(ValueError):
            bnd.decay_step(S, q, k, v, g, y=self.t(2, 3, 5))
        with pytest.raises(ValueError, match="GPU"):
            bnd.decay_step(S, q, k, v, g)
        with pytest.raises(ValueError):
            bnd.softmax_step(K, V[:, :, :8], at, q, k, v)
        with pytest.raises(TypeError):
            bnd.softmax_step(K.bfloat16(), V, at, q, k, v)
        with pytest.raises(TypeError):
            bnd.softmax_step(K, V, at.long(), q, k, v)
        with pytest.raises(ValueError):
            bnd.softmax_step(K[0], V, at, q, k, v)
        with pytest.raises(ValueError, match="GPU"):
            bnd.softmax_step(K, V, at, q, k, v)

    def test_sizes_beyond_32_bits(self):
        """They would reach the library cut to their low 32 bits: 2^32 + 4 tokens would be taken for 4."""
        far = 2 ** 32 + 4
        long = lambda *s: torch.zeros(1, dtype=torch.bfloat16).expand(*s)  # noqa: E731
        f32 = lambda *s: torch.zeros(1).expand(*s)  # noqa: E731
        at = torch.zeros(1, dtype=torch.int32)
        sizes = [(1, 1, far, 1, 1), (1, far, 1, 1, 1), (1, 1, 1, far, 1), (1, 1, 1, 1, far), (far, 1, 1, 1, 1)]
        for B, H, n, dk, dv in sizes:
            q, k, v, y = long(B, H, n, dk), long(B, H, n, dk), long(B, H, n, dv), long(B, H, n, dv)
            g, lse = f32(H), f32(B, H, n)
            for call in (lambda: bnd.decay_prefill(q, k, v, g), lambda: bnd.decay_backward(q, k, v, g, y),
                         lambda: bnd.softmax_prefill(q, k, v), lambda: bnd.softmax_backward(q, k, v, y, lse, y)):
                with pytest.raises(ValueError, match="32 bits"):
                    call()
            if n == 1:
                t = [x[:, :, 0] for x in (q, k, v)]
                with pytest.raises(ValueError, match="32 bits"):
                    bnd.decay_step(f32(B, H, dk, dv), *t, g)
                with pytest.raises(ValueError, match="32 bits"):
                    bnd.softmax_step(long(B, H, 9, dk), long(B, H, 9, dv), at.expand(B), *t)
        with pytest.raises(ValueError, match="32 bits"):
            bnd.softmax_step(long(1, 1, far, 4), long(1, 1, far, 4), at, *(long(1, 1, 4) for _ in range(3)))


def test_the_stream_without_torchs_private_function(monkeypatch):
    """The current stream's handle is the same whether or not this torch has the function that gives it directly."""
    class Stream:
        def __init__(self, device):
            self.cuda_stream = 1000 + device

    handed = []

    class Library:
        def call(self, *args):
            handed.append(args)
            return 0

    monkeypatch.setattr(torch.cuda, "current_stream", Stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(bnd, "load_library", Library)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 2000 + index, raising=False)
    bnd._invoke("call", torch.device("cuda", 3), 7)
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    bnd._invoke("call", torch.device("cuda", 3), 7)
    assert handed == [(7, 2003), (7, 1003)]
