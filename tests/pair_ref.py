"""Decayed linear attention and exact softmax attention from their definitions, in
float64 on the CPU, with bounds on what a computation in float32 (and, where it
says so, with one operand of a product rounded to bfloat16) may be off by.

Each function returns (value, bound) pairs.  A bound counts, with h the relative
half step of the output's type (2^-8 bfloat16, 2^-24 float32):
  h |value|                         the rounding of the output;
  r sum |w| |x|                     one rounding of the weights w to the operands' type,
                                    r = 2^-8 for bfloat16 inputs, 2^-22 for float32 ones
                                    (three bfloat16 numbers carry 24 bits; their product
                                    leaves out partial products below 2^-24, three of them);
  r sum |a| |R|                     one rounding of the entries of a state R to the operands' type
                                    where it is read out, at the start of a chunk of 32 tokens
                                    (from the other end in the gradients of k and v);
  N 2^-23 sum |terms|               float32 sums of N terms and the factors of a term.
A weight inside a chunk is carried as two bfloat16 numbers (2^-17), for which r is more than enough.
"""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
WEIGHT = {torch.float32: 2.0 ** -22, torch.bfloat16: 2.0 ** -8}
CHUNK = 32


def _ends(lengths, B, n):
    return [n] * B if lengths is None else [min(max(int(x), 0), n) for x in lengths]


def _power(g, e):
    """exp(g)^e for exponents e >= 0 (0 below); a decay of minus infinity keeps e = 0."""
    w = torch.where(e > 0, torch.exp(e.clamp(min=1) * g), torch.ones_like(e))
    return torch.where(e >= 0, w, torch.zeros_like(e))


def _pairs(g, n):
    t = torch.arange(n, dtype=torch.float64)
    return _power(g, t[:, None] - t[None, :])


def _readout(a, b, w, g, R, c, reverse=False):
    """sum |a| |R| of each row: R the state before (reverse: behind) the row's chunk, by whole chunks.
    a, b [e, i], w [e, j], in reverse R already times exp(g) (as the state behind the last token is given)."""
    e = a.shape[0]
    out = torch.zeros(e, w.shape[1], dtype=torch.float64)
    starts = list(range(0, e, CHUNK))
    for p in reversed(starts) if reverse else starts:
        q = min(e, p + CHUNK)
        t = torch.arange(q - p, dtype=torch.float64)
        far = (q - p - 1 - t) if reverse else t + 1
        out[p:q] = (a[p:q].abs() * _power(g, far)[:, None]) @ R.abs() * c
        late = t + 1 if reverse else q - p - 1 - t
        R = _power(g, torch.tensor(float(q - p), dtype=torch.float64)) * R + (b[p:q] * _power(g, late)[:, None]).T @ w[p:q]
    return out


def _bounded(value, dtype, weights, terms, count):
    """weights: sum |w| |x| of the rounded weights and sum |a| |R| of the rounded states; terms: sum of all
    factors' sizes."""
    f = HALF[dtype] * value.abs() + 1.01 * WEIGHT[dtype] * weights + count * 2.0 ** -23 * terms
    return value, f + 1e-30


def decay_prefill(q, k, v, log_decay, lengths=None, S_in=None):
    """((y, bound), (S, bound))"""
    dt = q.dtype
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    B, Hq, n, dk = q.shape
    H, dv = k.shape[1], v.shape[-1]
    c = 1.0 / math.sqrt(dk)
    out = [torch.zeros(B, Hq, n, dv, dtype=torch.float64) for _ in range(3)]
    st = [torch.zeros(B, H, dk, dv, dtype=torch.float64) for _ in range(2)]
    for b, e in enumerate(_ends(lengths, B, n)):
        for h in range(H):
            g = log_decay[h].double().cpu()
            D = _pairs(g, e)
            t = torch.arange(e, dtype=torch.float64)
            K, V = k[b, h, :e], v[b, h, :e]
            S0 = S_in[b, h].double().cpu() if S_in is not None else torch.zeros(dk, dv, dtype=torch.float64)
            first = _power(g, t + 1)[:, None]
            for m in range(Hq // H):
                i = h * (Hq // H) + m
                Q = q[b, i, :e]
                w = Q @ K.T * D * c
                out[0][b, i, :e] = w @ V + (Q * first) @ S0 * c
                out[1][b, i, :e] = w.abs() @ V.abs() + _readout(Q, K, V, g, S0, c)
                out[2][b, i, :e] = (Q.abs() @ K.abs().T * D * c) @ V.abs() + (Q.abs() * first) @ S0.abs() * c
            late = _power(g, e - 1 - t)[:, None]
            last = _power(g, torch.tensor(float(e), dtype=torch.float64))
            st[0][b, h] = (K * late).T @ V + last * S0
            st[1][b, h] = (K.abs() * late).T @ V.abs() + last * S0.abs()
    count = n + dk + dv + 16
    return _bounded(out[0], dt, out[1], out[2], count), (st[0], (n + 16) * 2.0 ** -23 * st[1] + 1e-30)


def decay_backward(q, k, v, log_decay, dy, lengths=None, S_in=None, dS=None):
    """((dq, bound), (dk, bound), (dv, bound), (dS_in, bound))"""
    dt = q.dtype
    q, k, v, dy = (x.double().cpu() for x in (q, k, v, dy))
    B, Hq, n, dk = q.shape
    H, dv = k.shape[1], v.shape[-1]
    c, G = 1.0 / math.sqrt(dk), Hq // H
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
    gq, gk, gv, gS = ([zero(B, Hq, n, dk) for _ in range(3)], [zero(B, H, n, dk) for _ in range(3)],
                      [zero(B, H, n, dv) for _ in range(3)], [zero(B, H, dk, dv) for _ in range(2)])
    for b, e in enumerate(_ends(lengths, B, n)):
        for h in range(H):
            g = log_decay[h].double().cpu()
            D = _pairs(g, e)
            t = torch.arange(e, dtype=torch.float64)
            K, V = k[b, h, :e], v[b, h, :e]
            S0 = S_in[b, h].double().cpu() if S_in is not None else zero(dk, dv)
            Ue = dS[b, h].double().cpu() if dS is not None else zero(dk, dv)
            first, late = _power(g, t + 1)[:, None], _power(g, e - 1 - t)[:, None]
            last = _power(g, torch.tensor(float(e), dtype=torch.float64))
            gk[0][b, h, :e] += (V @ Ue.T) * late
            gk[2][b, h, :e] += (V.abs() @ Ue.abs().T) * late
            gv[0][b, h, :e] += (K @ Ue) * late
            gv[2][b, h, :e] += (K.abs() @ Ue.abs()) * late
            gS[0][b, h] += last * Ue
            gS[1][b, h] += last * Ue.abs()
            for m in range(G):
                i = h * G + m
                Q, Y = q[b, i, :e], dy[b, i, :e]
                a, w = Y @ V.T * D * c, Q @ K.T * D * c
                aa, ww = Y.abs() @ V.abs().T * D * c, Q.abs() @ K.abs().T * D * c
                gq[0][b, i, :e] = a @ K + (Y * first) @ S0.T * c
                gq[1][b, i, :e] = a.abs() @ K.abs() + _readout(Y, V, K, g, S0.T, c)
                gq[2][b, i, :e] = aa @ K.abs() + (Y.abs() * first) @ S0.abs().T * c
                gk[0][b, h, :e] += a.T @ Q
                gk[1][b, h, :e] += a.abs().T @ Q.abs() + _readout(V, Y * c, Q, g, Ue.T / G, 1.0, True)
                gk[2][b, h, :e] += aa.T @ Q.abs()
                gv[0][b, h, :e] += w.T @ Y
                gv[1][b, h, :e] += w.abs().T @ Y.abs() + _readout(K, Q * c, Y, g, Ue / G, 1.0, True)
                gv[2][b, h, :e] += ww.T @ Y.abs()
                gS[0][b, h] += (Q * first).T @ Y * c
                gS[1][b, h] += (Q.abs() * first).T @ Y.abs() * c
    count = G * n + dk + dv + 16
    return (*(_bounded(x[0], dt, x[1], x[2], count) for x in (gq, gk, gv)),
            (gS[0], (G * n + 16) * 2.0 ** -23 * gS[1] + 1e-30))


def decay_step(S, q, k, v, log_decay):
    """((y, bound), (S, bound)) of one token from the state S."""
    dt = q.dtype
    S0, q, k, v = S.double().cpu(), q.double().cpu(), k.double().cpu(), v.double().cpu()
    B, H, dk = k.shape
    lam = torch.exp(log_decay.double().cpu())[:, None, None]
    S1 = lam * S0 + k[..., None] * v[..., None, :]
    Sa = lam * S0.abs() + k.abs()[..., None] * v.abs()[..., None, :]
    Q = q.view(B, H, -1, dk) / math.sqrt(dk)
    y, ya = (Q @ S1).flatten(1, 2), (Q.abs() @ Sa).flatten(1, 2)
    return (y, HALF[dt] * y.abs() + (dk + 8) * 2.0 ** -23 * ya + 1e-30), (S1, 4 * 2.0 ** -24 * Sa + 1e-30)


def _scores(Q, K, c):
    """Scores with later keys out, and how far a score in float32 may be off: the product's sum and the
    factors, and the exponential's argument (both ends of the subtraction)."""
    s = (Q @ K.T * c).masked_fill_(torch.ones(len(Q), len(K), dtype=torch.bool).triu_(1), -math.inf)
    off = (Q.shape[1] + 8) * 2.0 ** -23 * (Q.abs() @ K.abs().T * c).tril()
    return s, off


def softmax_prefill(q, k, v, lengths=None):
    """((y, bound), (lse, bound))"""
    dt = q.dtype
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    B, Hq, n, dk = q.shape
    H, dv = k.shape[1], v.shape[-1]
    c = 1.0 / math.sqrt(dk)
    y, yb = (torch.zeros(B, Hq, n, dv, dtype=torch.float64) for _ in range(2))
    lse, lb = torch.full((B, Hq, n), -math.inf, dtype=torch.float64), torch.zeros(B, Hq, n, dtype=torch.float64)
    for b, e in enumerate(_ends(lengths, B, n)):
        for i in range(Hq if e else 0):
            h = i // (Hq // H)
            s, off = _scores(q[b, i, :e], k[b, h, :e], c)
            z = torch.logsumexp(s, -1)
            p = torch.exp(s - z[:, None])
            V = v[b, h, :e]
            y[b, i, :e], lse[b, i, :e] = p @ V, z
            # a weight: its score's error, the exponential (2^-22), the sum of all weights; then its rounding
            rel = 2 * off + 2 * (p * off).sum(1, keepdim=True) + (n + 32) * 2.0 ** -23
            yb[b, i, :e] = HALF[dt] * y[b, i, :e].abs() + (p * (1.01 * WEIGHT[dt] + rel)) @ V.abs() + 1e-30
            lb[b, i, :e] = 2.0 ** -22 * z.abs() + (p * off).sum(1) + (n + 16) * 2.0 ** -23
    return (y, yb), (lse, lb)


def softmax_backward(q, k, v, y, lse, dy, lengths=None):
    """((dq, bound), (dk, bound), (dv, bound)), the probabilities from the exact lse: what the given y and lse
    (rounded results of the forward) are off by goes into the bounds."""
    dt = q.dtype
    given = y.double().cpu()
    z_given = lse.double().cpu()
    q, k, v, dy = (x.double().cpu() for x in (q, k, v, dy))
    B, Hq, n, dk = q.shape
    H, dv = k.shape[1], v.shape[-1]
    c, G = 1.0 / math.sqrt(dk), Hq // H
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
    g = [[zero(B, Hq, n, dk), zero(B, H, n, dk), zero(B, H, n, dv)] for _ in range(2)]
    for b, e in enumerate(_ends(lengths, B, n)):
        for i in range(Hq if e else 0):
            h = i // G
            Q, K, V, Y = q[b, i, :e], k[b, h, :e], v[b, h, :e], dy[b, i, :e]
            s, off = _scores(Q, K, c)
            z = torch.logsumexp(s, -1, keepdim=True)
            p = torch.exp(s - z)
            o = p @ V
            d = (Y @ V.T - (Y * o).sum(1, keepdim=True)).tril()
            x = c * p * d
            # p: its score, the given lse, the exponential
            rel = 2 * off + (z_given[b, i, :e, None] - z).abs() + 2.0 ** -23 * (z.abs() + s.masked_fill(p == 0, 0.0).abs() + 16)
            # dy.v - dy.y: float32 sums, and the given y's distance from the exact one
            diff = ((dv + 4) * 2.0 ** -23 * (Y.abs() @ V.abs().T + (Y.abs() * o.abs()).sum(1, keepdim=True))
                    + (Y.abs() * (given[b, i, :e] - o).abs()).sum(1, keepdim=True))
            wb = p * (1.01 * WEIGHT[dt] + rel + (G * n + 16) * 2.0 ** -23)
            xb = x.abs() * (1.01 * WEIGHT[dt] + rel + (G * n + 16) * 2.0 ** -23) + 1.01 * c * p * diff
            g[0][0][b, i, :e], g[1][0][b, i, :e] = x @ K, xb @ K.abs()
            g[0][1][b, h, :e] += x.T @ Q
            g[1][1][b, h, :e] += xb.T @ Q.abs()
            g[0][2][b, h, :e] += p.T @ Y
            g[1][2][b, h, :e] += wb.T @ Y.abs()
    return tuple((a, HALF[dt] * a.abs() + w + 1e-30) for a, w in zip(*g))


def softmax_step(K, V, lengths, q, k, v):
    """((y, bound), K, V): the cache after the call."""
    dt = q.dtype
    K, V = K.clone().cpu(), V.clone().cpu()
    B, H, cap, dk = K.shape
    G, dv = q.shape[1] // H, V.shape[-1]
    y, yb = (torch.zeros(B, H * G, dv, dtype=torch.float64) for _ in range(2))
    for b in range(B):
        e = int(lengths[b])
        if not 0 <= e < cap:
            continue
        K[b, :, e], V[b, :, e] = k[b].cpu(), v[b].cpu()
        for i in range(H * G):
            x, kk, vv = q[b, i].double().cpu(), K[b, i // G, :e + 1].double(), V[b, i // G, :e + 1].double()
            s = kk @ x / math.sqrt(dk)
            off = (dk + 8) * 2.0 ** -23 * (kk.abs() @ x.abs()) / math.sqrt(dk)
            p = torch.softmax(s, 0)
            y[b, i] = p @ vv
            rel = 2 * off + 2 * (p * off).sum() + (e + 32) * 2.0 ** -23
            yb[b, i] = HALF[dt] * y[b, i].abs() + (p * (1.01 * WEIGHT[dt] + rel)) @ vv.abs() + 1e-30
    return (y, yb), K, V


def one_entry_a_row(seed, n, dk, dv):
    """q, k, v, dy [1, 1, n, d] in bfloat16 with one entry a row, in column t % d, so that an element of a result is a sum of
    about n / d terms.  q and dy grow with t as the weights shrink, so that all terms of a sum are of
    like size: one that is left out, or one too many, is then well beyond 2^-8 of their sum."""
    g = torch.Generator().manual_seed(seed)
    t = torch.arange(n)

    def make(d, low, high, grow):
        a = (torch.rand(n, generator=g) * (high - low) + low) * (torch.randint(0, 2, (n,), generator=g) * 2 - 1)
        x = torch.zeros(n, d)
        x[t, t % d] = a * (t + 1) / grow if grow else a
        return x.bfloat16()[None, None]

    return make(dk, 0.5, 1.0, 16), make(dk, 0.125, 0.25, 0), make(dv, 0.5, 2.0, 0), make(dv, 0.5, 2.0, 64)


def check(got, ref, label=""):
    """Every element of a result within its bound (infinities equal)."""
    value, bound = ref
    got = got.double().cpu()
    assert got.shape == value.shape, f"{label}: {tuple(got.shape)} instead of {tuple(value.shape)}"
    fine = torch.isfinite(value)
    assert torch.equal(got[~fine], value[~fine]), f"{label}: infinities differ"
    off = (got - value)[fine].abs()
    worst = (off / bound[fine].clamp(min=1e-30)).max().item() if off.numel() else 0.0  # (exact where there is nothing to sum)
    assert not math.isnan(worst) and worst <= 1.0, f"{label}: {worst:.3g} times the bound"
    return worst
