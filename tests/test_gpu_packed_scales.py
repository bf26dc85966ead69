"""Scales of 4-bit rows where their rounding to bfloat16 hangs on the last bit of what is rounded."""
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


def _ends():
    """(least, most) pairs, float32: half their distance times the nearest float32 to 1 / 7.5, and divided by 7.5, round to
    different bfloat16 numbers."""
    rng = np.random.default_rng(5)
    low, high = -np.abs(rng.standard_normal((2, 4_000_000))).astype(np.float32)
    high = -high
    half = np.float32(0.5) * high - np.float32(0.5) * low
    there = ref.bf16(half * np.float32(1 / 7.5)) != ref.bf16(half / np.float32(7.5))
    return low[there], high[there]


def test_scales_are_products_with_the_inverse_of_7_5(sata):
    """As a program forms them that divides a tensor by 7.5 with torch on the GPU, which multiplies: in one group of some
    100 000 the scale is not the one of a division."""
    low, high = _ends()
    assert len(low) >= 20
    x = np.ascontiguousarray(np.linspace(low, high, 32, axis=-1), dtype=np.float32)
    x[:, 0], x[:, -1] = low, high
    want = ref.bf16((np.float32(0.5) * high - np.float32(0.5) * low) * np.float32(1 / 7.5))
    t = torch.from_numpy(x)[None, None].cuda()
    K = torch.zeros(1, 1, len(low), 20, dtype=torch.uint8, device="cuda")
    sata.packed_write(K, None, None, t, None)
    got = K[0, 0, :, 16:18].contiguous().view(torch.bfloat16).float().cpu().numpy()[:, 0]
    assert np.array_equal(got, want)
    # a token's row has the same bits
    C, D = (torch.zeros(len(low), 1, 1, 20, dtype=torch.uint8, device="cuda") for _ in range(2))
    rows = t[0, 0, :, None].contiguous()
    sata.softmax_step_packed(C, D, torch.zeros(len(low), dtype=torch.int32, device="cuda"), rows, rows, rows)
    assert torch.equal(C[:, 0, 0], K[0, 0]) and torch.equal(D[:, 0, 0], K[0, 0])
