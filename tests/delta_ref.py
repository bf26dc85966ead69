"""The gated delta rule, rows of 4 bits an entry and rotary positions from their definitions, in float64 on the CPU."""
import math

import numpy as np
import torch


def delta(q, k, v, g, beta, lengths=None, S_in=None):
    """(y, S, states): q, k [B, H, n, d_k], v [B, G*H, n, d_v], g, beta [B, G*H, n] -> y as v, the last states, and the
    states behind every token [n, B, G*H, d_k, d_v].  Differentiable."""
    B, Hk, n, dk = k.shape
    H, dv = v.shape[1], v.shape[-1]
    q, k = (x.repeat_interleave(H // Hk, dim=1) for x in (q, k))
    S = torch.zeros(B, H, dk, dv, dtype=torch.float64) if S_in is None else S_in
    ys, states = [], []
    for t in range(n):
        live = torch.ones(B, dtype=torch.bool) if lengths is None else t < lengths
        live = live[:, None, None, None]
        Sp = torch.exp(g[:, :, t])[..., None, None] * S
        u = beta[:, :, t, None] * (v[:, :, t] - (k[:, :, t, :, None] * Sp).sum(-2))
        new = Sp + k[:, :, t, :, None] * u[..., None, :]
        S = torch.where(live, new, S)
        y = (q[:, :, t, :, None] * S).sum(-2) / math.sqrt(dk)
        ys.append(torch.where(live[..., 0], y, 0.0))
        states.append(S)
    y = torch.stack(ys, 2) if n else torch.zeros(B, H, 0, dv, dtype=torch.float64)
    return y, S, states


def draw(seed, B, Hk, G, n, dk, dv, dtype, decay=0.05, state=False, unit=True):
    """Inputs as a layer makes them: keys of length one, beta in (0, 1), g below zero; values exact in dtype."""
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    q, k, v = r(B, Hk, n, dk), r(B, Hk, n, dk), r(B, Hk * G, n, dv)
    if unit:
        q, k = (x / x.norm(dim=-1, keepdim=True).clamp(min=1e-3) for x in (q, k))
    g = -decay * torch.nn.functional.softplus(r(B, Hk * G, n))
    beta = torch.sigmoid(r(B, Hk * G, n))
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v = (x.to(dt) for x in (q, k, v))
    out = [q, k, v, g.float(), beta.float()]
    return out + ([r(B, Hk * G, dk, dv).float()] if state else [None])


def to64(*xs):
    return [x.double().cpu() if x is not None else None for x in xs]


# ------------------------------------------------------------------ rows of 4 bits an entry

def bf16(x):
    """float32 array -> the nearest bfloat16, as float32."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def pack(x):
    """[..., d] float32 -> (rows [..., bytes] uint8, the values they stand for [..., d] float32), entry by entry."""
    x = np.asarray(x, dtype=np.float32)
    d = x.shape[-1]
    groups = 1 if d <= 32 else 2 if d <= 64 else 4
    flat = x.reshape(-1, d)
    rows = np.zeros((flat.shape[0], 20 * groups), dtype=np.uint8)
    values = np.zeros_like(flat)
    half, one = np.float32(0.5), np.float32(7.5)
    with np.errstate(all="ignore"):
        for g in range(0, (d + 31) // 32):
            part = flat[:, 32 * g:32 * g + 32]
            fine = (np.abs(part) <= np.float32(2.0 ** 120)).all(-1)
            least, most = part.min(-1), part.max(-1)
            scale, low = bf16((half * most - half * least) / one), bf16(least)
            scale, low = (np.where(fine, a, np.float32(np.nan)) for a in (scale, low))
            step = (half * scale)[:, None]
            code = np.rint((half * part - (half * low)[:, None]) / np.where(step > 0, step, np.float32(1)))
            code = np.where(step > 0, np.clip(code, 0, 15), 0)
            values[:, 32 * g:32 * g + 32] = (low[:, None].astype(np.float64) + scale[:, None].astype(np.float64) * code)
            code = np.nan_to_num(code).astype(np.uint8)
            for i in range(part.shape[1]):
                rows[:, (i % 16) * groups + g] |= code[:, i] << (4 * (i // 16))
            for j, a in enumerate((scale, low)):
                bits = torch.from_numpy(a.copy()).to(torch.bfloat16).view(torch.int16).numpy().astype(np.uint16)
                bits = np.where(fine, bits, 0x7fc0)
                rows[:, 16 * groups + 4 * g + 2 * j] = bits & 255
                rows[:, 16 * groups + 4 * g + 2 * j + 1] = bits >> 8
    return rows.reshape(*x.shape[:-1], -1), values.reshape(x.shape)


# ------------------------------------------------------------------ rotary positions

def rotary(x, positions, freq, interleaved, scale, back=False):
    """x [B, H, n, d] float64, positions [B, n], freq [R] -> turned, one pair after the other."""
    R = len(freq)
    y = x.clone()
    for i in range(R):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, R + i)
        angle = positions.double()[:, None, :] * float(freq[i]) * (-1.0 if back else 1.0)
        y[..., a] = scale * (x[..., a] * torch.cos(angle) - x[..., b] * torch.sin(angle))
        y[..., b] = scale * (x[..., b] * torch.cos(angle) + x[..., a] * torch.sin(angle))
    return y
