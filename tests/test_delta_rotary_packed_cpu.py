"""Host side of the delta rule, rotary positions and 4-bit caches: frequencies, sizes, refusals, and the references that
the GPU tests compare with."""
import ctypes
import math

import numpy as np
import pytest
import torch

import delta_ref as ref
from paper_2602_00294_amd import _binding as bnd

INVALID, UNSUPPORTED, LARGE = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    return bnd.load_library()


P = ctypes.c_void_p(4096)  # an address that no refused call reads
NULL = None


# ------------------------------------------------------------------ frequencies

def test_plain_and_linear_frequencies():
    f, s = bnd.rotary_frequencies(4, 10000.0, device="cpu")
    assert s == 1.0 and np.array_equal(f.numpy(), np.float32([1.0, 0.1, 0.01, 0.001]))
    f, s = bnd.rotary_frequencies(3, 8.0, "linear", 4.0, device="cpu")
    assert s == 1.0 and np.allclose(f.numpy(), [0.25, 0.125, 0.0625], rtol=2.0 ** -23)


@pytest.mark.parametrize("pairs", [2, 5, 64])
def test_scaled_base(pairs):
    """The fastest pair stays, the slowest is divided by the factor."""
    plain, _ = bnd.rotary_frequencies(pairs, 10000.0, device="cpu")
    f, s = bnd.rotary_frequencies(pairs, 10000.0, "base", 8.0, device="cpu")
    assert s == 1.0 and f[0] == 1.0
    assert math.isclose(f[-1] * 8.0, plain[-1], rel_tol=2.0 ** -22)


def test_by_turns():
    pairs, original, factor = 64, 4096.0, 16.0
    plain, _ = bnd.rotary_frequencies(pairs, 10000.0, device="cpu")
    f, s = bnd.rotary_frequencies(pairs, 10000.0, "by_turns", factor, original, device="cpu")
    assert math.isclose(s, 0.1 * math.log(16.0) + 1.0, rel_tol=2.0 ** -23)
    turns = original * plain.double() / (2 * math.pi)
    assert torch.equal(f[turns >= 32.1], plain[turns >= 32.1])
    slow = turns <= 0.99
    assert slow.any() and torch.allclose(f[slow] * factor, plain[slow], rtol=2.0 ** -22)
    mid = ~slow & (turns < 32.1)
    assert mid.any() and (f[mid] <= plain[mid]).all() and (f[mid] >= plain[mid] / factor).all()
    r = (f / plain).double()
    assert (r[:-1] - r[1:] >= -1e-6).all()  # the slower, the more


@pytest.mark.parametrize("args", [(0,), (65,), (4, 1.0), (4, math.inf), (4, math.nan), (4, 1e4, "linear", 0.5),
                                  (4, 1e4, "by_turns", 2.0, 0.0), (1, 1e4, "base", 2.0), (4, 1e4, "linear", math.nan)])
def test_refused_frequencies(args):
    with pytest.raises(bnd.SataError):
        bnd.rotary_frequencies(*args, device="cpu")


def test_unknown_scaling():
    with pytest.raises(ValueError):
        bnd.rotary_frequencies(4, 1e4, "other", device="cpu")


# ------------------------------------------------------------------ sizes and refusals

def test_row_bytes():
    assert [bnd.packed_row_bytes(d) for d in (1, 32, 33, 64, 65, 96, 128)] == [20, 20, 40, 40, 80, 80, 80]
    for d in (0, -1, 129):
        with pytest.raises(ValueError):
            bnd.packed_row_bytes(d)


def test_scratch_queries(lib):
    assert lib.sata_delta_scratch(0, 1, 1, 1, 1, 100, 64, 64) >= 0
    assert lib.sata_softmax_step_packed_scratch(2, 2, 4, 1000, 64) >= 0
    for B, H, G in ((0, 1, 1), (1, 0, 1), (1, 1, 0)):
        assert lib.sata_delta_scratch(0, 1, B, H, G, 5, 64, 64) == -1
    assert lib.sata_delta_scratch(0, 1, 1, 1, 1, -1, 64, 64) == -1
    assert lib.sata_delta_scratch(1, 1, 1, 1, 1, 5, 129, 64) == -1
    assert lib.sata_delta_scratch(1, 7, 1, 1, 1, 5, 64, 64) == -1
    assert lib.sata_delta_scratch(1, 1, 65535, 1, 1, 1 << 21, 64, 64) == -1
    assert lib.sata_softmax_step_packed_scratch(1, 1, 1, 0, 64) == -1
    assert lib.sata_softmax_step_packed_scratch(1, 1, 1, (1 << 21) + 1, 64) == -1


def _prefill(lib, q=P, k=P, v=P, g=P, beta=P, dt=1, B=1, H=1, G=1, n=4, dk=8, dv=8, S_in=NULL, y=P, S=NULL):
    return lib.sata_delta_prefill(q, k, v, g, beta, dt, B, H, G, n, dk, dv, NULL, S_in, y, S, NULL, NULL)


@pytest.mark.parametrize("change,status", [
    (dict(q=NULL), INVALID), (dict(beta=NULL), INVALID), (dict(y=NULL), INVALID), (dict(dt=5), INVALID),
    (dict(B=0), INVALID), (dict(H=0), INVALID), (dict(G=-1), INVALID), (dict(n=-1), INVALID), (dict(dk=0), INVALID),
    (dict(dk=129), UNSUPPORTED), (dict(dv=129), UNSUPPORTED), (dict(B=65536), LARGE), (dict(B=256, H=256), LARGE),
    (dict(B=2 ** 30, H=2 ** 30, G=2 ** 30), LARGE), (dict(n=(1 << 21) + 1), LARGE), (dict(B=500, n=1 << 21), LARGE),
    (dict(S_in=P, S=P), INVALID)])
def test_refused_prompts(lib, change, status):
    assert _prefill(lib, **change) == status
    assert lib.sata_last_error()


def test_refused_delta_gradients_and_tokens(lib):
    def back(dq=P, dS=NULL, S_in=NULL, dS_in=NULL, n=4, dbeta=P, dv=8):
        return lib.sata_delta_backward(P, P, P, P, P, P, 1, 1, 1, 1, n, 8, dv, NULL, S_in, dS, dq, P, P, P, dbeta, dS_in, NULL,
                                       NULL)
    assert back(dq=NULL) == INVALID and back(dbeta=NULL) == INVALID
    assert back(dS=P, dS_in=P) == INVALID and back(S_in=P, dS_in=P) == INVALID
    assert back(n=-1) == INVALID and back(dv=200) == UNSUPPORTED
    assert lib.sata_delta_step(NULL, P, P, P, P, P, 1, 1, 1, 1, 8, 8, P, NULL) == INVALID
    assert lib.sata_delta_step(P, P, P, P, P, NULL, 1, 1, 1, 1, 8, 8, P, NULL) == INVALID
    assert lib.sata_delta_step(P, P, P, P, P, P, 1, 1, 1, 1, 8, 200, P, NULL) == UNSUPPORTED


def test_refused_rotary(lib):
    def call(q=P, k=NULL, pos=P, f=P, dt=1, B=1, Hq=1, Hk=0, n=4, d=8, pairs=4, qo=P, ko=NULL):
        return lib.sata_rotary(q, k, pos, f, dt, B, Hq, Hk, n, d, pairs, 0, 1.0, 0, qo, ko, NULL)
    other, third = ctypes.c_void_p(8192), ctypes.c_void_p(12288)
    assert call(q=NULL) == INVALID and call(pos=NULL) == INVALID and call(f=NULL) == INVALID and call(qo=NULL) == INVALID
    assert call(dt=9) == INVALID and call(B=0) == INVALID and call(Hq=0) == INVALID and call(Hk=-1) == INVALID
    assert call(n=-1) == INVALID and call(pairs=0) == INVALID and call(pairs=5) == INVALID and call(d=130) == UNSUPPORTED
    assert call(B=2, Hq=40000) == LARGE and call(n=(1 << 21) + 1) == LARGE
    assert call(Hk=1, k=NULL, ko=other) == INVALID and call(Hk=1, k=other, ko=NULL) == INVALID
    assert call(Hk=1, k=other, qo=third, ko=third) == INVALID  # one output for both
    assert call(Hk=1, k=other, qo=other, ko=third) == INVALID  # q's output in k's place
    assert call(n=0) == 0


def test_refused_packed(lib):
    def write(K=P, V=ctypes.c_void_p(8192), cap=4, k=P, v=P, dt=1, B=1, H=1, n=4, dk=64, dv=64):
        return lib.sata_packed_write(K, V, cap, NULL, k, v, NULL, dt, B, H, n, dk, dv, NULL)
    assert write(K=NULL) == INVALID and write(V=NULL) == INVALID and write(v=NULL) == INVALID and write(V=P) == INVALID
    assert write(cap=0) == INVALID and write(n=-1) == INVALID and write(dk=129) == UNSUPPORTED and write(dt=4) == INVALID
    assert write(cap=(1 << 21) + 1) == LARGE and write(K=ctypes.c_void_p(4100)) == INVALID and write(n=0) == 0

    def read(C=P, cap=4, dt=0, n=1, d=128, x=P):
        return lib.sata_packed_read(C, cap, NULL, dt, 1, 1, n, d, x, NULL)
    assert read(C=NULL) == INVALID and read(x=NULL) == INVALID and read(cap=-1) == INVALID and read(d=0) == INVALID
    assert read(C=ctypes.c_void_p(4104)) == INVALID and read(n=0) == 0

    def step(K=P, V=ctypes.c_void_p(8192), cap=4, L=P, q=P, d=64, y=P, G=1):
        return lib.sata_softmax_step_packed(K, V, cap, L, q, P, P, 1, 1, 1, G, d, d, y, NULL, NULL)
    assert step(K=NULL) == INVALID and step(V=P) == INVALID and step(L=NULL) == INVALID and step(y=NULL) == INVALID
    assert step(cap=0) == INVALID and step(d=200) == UNSUPPORTED and step(G=0) == INVALID
    assert step(cap=1 << 20) == INVALID  # (scratch is missing)


# ------------------------------------------------------------------ the references

def test_delta_reference_replaces_and_decays():
    """With beta 1 and keys of length one a key reads back the value that it was last written with."""
    d = 6
    k = torch.eye(d, dtype=torch.float64)[[0, 1, 0, 2]][None, None]
    v = torch.randn(1, 1, 4, 3, dtype=torch.float64)
    one, zero = torch.ones(1, 1, 4, dtype=torch.float64), torch.zeros(1, 1, 4, dtype=torch.float64)
    _, S, _ = ref.delta(k, k, v, zero, one)
    assert torch.allclose(S[0, 0, 0], v[0, 0, 2]) and torch.allclose(S[0, 0, 1], v[0, 0, 1])
    g = torch.full((1, 1, 4), math.log(0.5), dtype=torch.float64)
    _, S, _ = ref.delta(k, k, v, g, one)
    assert torch.allclose(S[0, 0, 1], v[0, 0, 1] / 4) and torch.allclose(S[0, 0, 2], v[0, 0, 3])


def test_delta_reference_without_rates_is_linear_attention():
    q, k, v, g, beta, _ = ref.draw(3, 1, 2, 1, 9, 5, 4, "f32")
    q, k, v = ref.to64(q, k, v)
    tiny = torch.full((1, 2, 9), 1e-9, dtype=torch.float64)
    y, _, _ = ref.delta(q, k, v, torch.zeros(1, 2, 9, dtype=torch.float64), tiny)
    want = ((q @ k.transpose(-1, -2)).tril() @ v) / math.sqrt(5) * 1e-9
    assert torch.allclose(y, want, rtol=1e-6)


def test_delta_gradients_by_differences():
    """The reference's gradients against central differences of the recurrence, along random directions."""
    x = ref.to64(*ref.draw(7, 2, 1, 2, 12, 5, 4, "f32", state=True))
    gen = torch.Generator().manual_seed(8)
    w, wS = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((2, 2, 12, 4), (2, 2, 5, 4)))

    def loss(q, k, v, g, beta, S):
        y, S, _ = ref.delta(q, k, v, g, beta, torch.tensor([12, 7]), S)
        return (y * w).sum() + (S * wS).sum()

    leaves = [a.clone().requires_grad_() for a in x]
    grads = torch.autograd.grad(loss(*leaves), leaves)
    for i, grad in enumerate(grads):
        e = torch.randn(x[i].shape, generator=gen, dtype=torch.float64)
        at = lambda s: loss(*(a + s * e if j == i else a for j, a in enumerate(x)))  # noqa: E731
        slope = (at(1e-5) - at(-1e-5)) / 2e-5
        assert math.isclose(slope.item(), (grad * e).sum().item(), rel_tol=1e-7, abs_tol=1e-8)


def test_packed_reference_by_hand():
    """0, 1 .. 15 twice: scale 1, least value 0, codes as they are; a byte holds entries a and 16 + a."""
    x = np.float32(np.arange(32) % 16)
    rows, values = ref.pack(x)
    assert np.array_equal(values, x)
    assert np.array_equal(rows[:16], [i | i << 4 for i in range(16)])
    assert np.array_equal(rows[16:], [0x80, 0x3F, 0, 0])
    rows, values = ref.pack(np.float32([3.0] * 40))
    assert rows.shape == (40,) and np.array_equal(values, np.float32([3.0] * 40)) and not rows[:32].any()
    x = np.random.default_rng(1).standard_normal((50, 128)).astype(np.float32)
    _, values = ref.pack(x)
    # half a step, what rounding the ends to bfloat16 adds, of a group's range and least value
    group = x.reshape(50, 4, 32)
    most = (group.max(-1) - group.min(-1)) / 30 + 2.0 ** -8 * np.abs(group).max(-1) * 3
    assert (np.abs(values - x).reshape(50, 4, 32) <= most[..., None]).all()
