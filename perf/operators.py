"""Decayed linear attention and exact softmax attention, as measurable cases.

Each case is one call that a serving or training program makes of one of the
six entry points: a prompt (decay_prefill, softmax_prefill), one token of every
sequence (decay_step, softmax_step) and the gradients of a prompt
(decay_backward, softmax_backward).  With c = 1 / sqrt(d_k) and lam = exp(log_decay)
of the key/value head,

    decay:    S_t = lam S_{t-1} + k_t (x) v_t,   y_t = c q_t S_t
    softmax:  y_t = sum_{s<=t} exp(c q_t.k_s - lse_t) v_s

over the tokens below a sequence's length; rows from there on give zeros (lse:
minus infinity).  Queries, keys, values and gradients are N(0, 1); the decays
run from 1 - 2^-2 to 1 - 2^-12 over the heads.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def listed():
    return [
        # a batch of long prompts through one layer of large heads, the states kept for generation
        dict(name="decay_prompt_batch", op="decay_prefill", B=8, H=16, G=1, n=8192, dk=128, dv=128, dtype="bf16",
             lengths=False, state=True),
        # a few short float32 prompts of odd sizes in a padded batch, going on from earlier states
        dict(name="decay_prompt_ragged", op="decay_prefill", B=3, H=2, G=2, n=777, dk=24, dv=40, dtype="f32",
             lengths=True, state=True),
        # one token of one sequence: launch latency
        dict(name="decay_token_one", op="decay_step", B=1, H=16, G=1, dk=64, dv=64, dtype="bf16"),
        # one token of a serving batch, four query heads to each state: 268 MB of state read and written
        dict(name="decay_token_batch", op="decay_step", B=128, H=16, G=4, dk=128, dv=128, dtype="bf16"),
        # the gradients of a training batch
        dict(name="decay_gradients_batch", op="decay_backward", B=8, H=32, G=1, n=2048, dk=64, dv=64, dtype="bf16",
             lengths=False, state=False),
        # float32 gradients at odd sizes in a padded batch, with the gradients of both states
        dict(name="decay_gradients_ragged", op="decay_backward", B=2, H=4, G=2, n=1111, dk=48, dv=32, dtype="f32",
             lengths=True, state=True),
        # a long prompt with grouped query heads
        dict(name="softmax_prompt_long", op="softmax_prefill", B=1, H=8, G=4, n=8192, dk=128, dv=128, dtype="bf16",
             lengths=False),
        # short float32 prompts of odd sizes in a padded batch
        dict(name="softmax_prompt_ragged", op="softmax_prefill", B=4, H=3, G=1, n=333, dk=40, dv=40, dtype="f32",
             lengths=True),
        # one token of one sequence with a short cache: launch latency
        dict(name="softmax_token_one", op="softmax_step", B=1, H=8, G=1, n=1000, dk=64, dv=64, dtype="bf16"),
        # one token of a serving batch with sequences of many lengths, four query heads to each cached head
        dict(name="softmax_token_batch", op="softmax_step", B=16, H=8, G=4, n=8192, dk=128, dv=128, dtype="bf16"),
        # the gradients of a training batch
        dict(name="softmax_gradients_batch", op="softmax_backward", B=2, H=16, G=1, n=4096, dk=128, dv=128,
             dtype="bf16", lengths=False),
        # gradients at odd sizes in a padded batch with grouped query heads
        dict(name="softmax_gradients_ragged", op="softmax_backward", B=3, H=4, G=2, n=1001, dk=64, dv=56,
             dtype="bf16", lengths=True),
    ]


# ------------------------------------------------------------------ drawn cases

def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """One more case of these ranges: 1 to 8192 tokens, heads of 8 to 128, every type, direction and form."""
    op = rng.choice(["decay_prefill", "decay_step", "decay_backward", "softmax_prefill", "softmax_step",
                     "softmax_backward"])
    while True:
        dk = rng.choice([16, 32, 64, 64, 96, 128, 128, rng.randint(8, 128)])
        dv = dk if rng.random() < 0.7 else rng.choice([16, 32, 64, 128, rng.randint(8, 128)])
        case = dict(op=op, B=_log_int(rng, 1, 16), H=rng.choice([1, 2, 4, 8, 16, rng.randint(1, 16)]),
                    G=rng.choice([1, 1, 2, 4, 8, rng.randint(1, 8)]), dk=dk, dv=dv,
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
        if op == "decay_step":
            case["B"] = _log_int(rng, 1, 128)
        else:
            case["n"] = _log_int(rng, 1, 8192)
        if op not in ("decay_step", "softmax_step"):
            case["lengths"] = rng.random() < 0.5
        if op in ("decay_prefill", "decay_backward"):
            case["state"] = rng.random() < 0.5
        w = work(case)
        rows = case["B"] * case["H"] * case["G"] * case.get("n", 1)
        if w["bytes"] > 1.1e9 or (op.startswith("softmax") and w["flops"] > (5e11 if case["dtype"] == "bf16" else 6e10)):
            continue
        if rows * max(dk, dv) > 70_000_000 or (op in ("softmax_prefill", "softmax_backward")
                                               and rows * case["n"] > 2_200_000_000):
            continue
        return case


# ------------------------------------------------------------------ inputs

def _lengths_of(case):
    """Tokens of each sequence: all, or from none in the first to all in the last."""
    B, n = case["B"], case.get("n", 1)
    if case["op"] == "softmax_step":  # tokens in the cache before the call
        return [(n - 1) * (b + 1) // B for b in range(B)]
    if not case.get("lengths"):
        return [n] * B
    return [n * b // max(1, B - 1) if B > 1 else (n + 1) // 2 for b in range(B)]


def _draw_inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    dt = DTYPES[case["dtype"]]
    op, B, H, G, dk, dv = (case[k] for k in ("op", "B", "H", "G", "dk", "dv"))

    def normal(*shape, dtype=dt):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)

    t = {}
    if op.startswith("decay"):
        x = torch.linspace(2.0, 12.0, H, dtype=torch.float64) if H > 1 else torch.tensor([6.0], dtype=torch.float64)
        t["log_decay"] = torch.log1p(-torch.exp2(-x)).float().cuda()
    if op in ("decay_step", "softmax_step"):
        t.update(q=normal(B, H * G, dk), k=normal(B, H, dk), v=normal(B, H, dv))
        if op == "decay_step":
            t["S"] = normal(B, H, dk, dv, dtype=torch.float32) * 4.0
        else:
            t.update(K=normal(B, H, case["n"], dk), V=normal(B, H, case["n"], dv))
            t["lengths"] = torch.tensor(_lengths_of(case), dtype=torch.int32, device="cuda")
        return t
    n = case["n"]
    t.update(q=normal(B, H * G, n, dk), k=normal(B, H, n, dk), v=normal(B, H, n, dv))
    t["lengths"] = torch.tensor(_lengths_of(case), dtype=torch.int32, device="cuda") if case["lengths"] else None
    if op.endswith("backward"):
        t["dy"] = normal(B, H * G, n, dv)
    if op.startswith("decay") and case["state"]:
        t["S_in"] = normal(B, H, dk, dv, dtype=torch.float32) * 4.0
        if op == "decay_backward":
            t["dS"] = normal(B, H, dk, dv, dtype=torch.float32) * 4.0
    return t


def prepare(case, seed):
    t = _draw_inputs(case, seed)
    if case["op"] == "softmax_backward":  # what the forward pass has left
        t["y"], t["lse"] = _softmax_forward(t["q"], t["k"], t["v"], t["lengths"])
    t["case"] = case
    return t


# ------------------------------------------------------------------ one pass

def run(state):
    case, t = state["case"], state
    op = case["op"]
    if own:
        import paper_2602_00294_amd as sata
        if op == "decay_prefill":
            y, S = sata.decay_prefill(t["q"], t["k"], t["v"], t["log_decay"], lengths=t["lengths"], S_in=t.get("S_in"),
                                      want_state=case["state"])
            return [y] + ([S] if case["state"] else [])
        if op == "decay_step":
            return [sata.decay_step(t["S"], t["q"], t["k"], t["v"], t["log_decay"]), t["S"]]
        if op == "decay_backward":
            dq, dk, dv, dS_in = sata.decay_backward(t["q"], t["k"], t["v"], t["log_decay"], t["dy"],
                                                    lengths=t["lengths"], S_in=t.get("S_in"), dS=t.get("dS"))
            return [dq, dk, dv] + ([dS_in] if case["state"] else [])
        if op == "softmax_prefill":
            return list(sata.softmax_prefill(t["q"], t["k"], t["v"], lengths=t["lengths"]))
        if op == "softmax_step":
            return [sata.softmax_step(t["K"], t["V"], t["lengths"], t["q"], t["k"], t["v"]), t["K"], t["V"]]
        return list(sata.softmax_backward(t["q"], t["k"], t["v"], t["y"], t["lse"], t["dy"], lengths=t["lengths"]))
    if op == "decay_prefill":
        y, S = _decay_forward(t["q"], t["k"], t["v"], t["log_decay"], t["lengths"], t.get("S_in"), case["state"])
        return [y] + ([S] if case["state"] else [])
    if op == "decay_step":
        return [_decay_token(t["S"], t["q"], t["k"], t["v"], t["log_decay"]), t["S"]]
    if op == "decay_backward":
        return _decay_gradients(t["q"], t["k"], t["v"], t["log_decay"], t["dy"], t["lengths"], t.get("S_in"),
                                t.get("dS"))
    if op == "softmax_prefill":
        return list(_softmax_forward(t["q"], t["k"], t["v"], t["lengths"]))
    if op == "softmax_step":
        return [_softmax_token(t["K"], t["V"], t["lengths"], t["q"], t["k"], t["v"]), t["K"], t["V"]]
    return list(_softmax_gradients(t["q"], t["k"], t["v"], t["y"], t["lse"], t["dy"], t["lengths"]))


# ------------------------------------------------------------------ the plain forms, in 32 bits

def _grouped(x, H):
    """[B, H G, n, d] -> [B, H, G, n, d] in 32 bits."""
    B, HG = x.shape[:2]
    return x.float().reshape(B, H, HG // H, *x.shape[2:])


def _alive(lengths, B, n, device):
    """[B, n]: whether a position is below its sequence's length, and the lengths."""
    at = torch.arange(n, device=device)
    ends = torch.full((B,), n, device=device) if lengths is None else lengths.long()
    return at[None, :] < ends[:, None], ends


def _powers(log_decay, exponent):
    """lam^exponent for exponents [...] -> [H, ...], the angle of far positions in 64 bits; zero for negative exponents."""
    e = exponent.double()
    g = log_decay.double().reshape(-1, *([1] * e.dim()))
    return torch.where(e >= 0, torch.exp(e.clamp(min=0) * g), 0.0).float()


def _mix(a, b, v, log_decay, S_in):
    """sum_{s<=t} lam^(t-s) (a_t.b_s) v_s + lam^(t+1) a_t S_in for a [B,H,G,n,i], b [B,H,G',n,i], v [B,H,G',n,j]
    (G' = 1 or G), in chunks: pairs inside a chunk, and the chunks' sums carried by their powers."""
    B, H, G, n, i = a.shape
    j, C = v.shape[-1], 128
    c = (n + C - 1) // C
    pad = lambda x: torch.nn.functional.pad(x, (0, 0, 0, c * C - n)).reshape(*x.shape[:3], c, C, x.shape[-1])  # noqa: E731
    a, b, v = pad(a), pad(b), pad(v)
    at = torch.arange(C, device=a.device)
    pairs = torch.matmul(a, b.transpose(-1, -2)) * _powers(log_decay, at[:, None] - at[None, :])[None, :, None, None]
    out = torch.matmul(pairs, v)
    late = _powers(log_decay, C - 1 - at)[None, :, None, None, :, None]
    sums = torch.matmul((b * late).transpose(-1, -2), v)                     # [B,H,G',c,i,j]
    ch = torch.arange(c, device=a.device)
    carry = _powers(log_decay, C * (ch[:, None] - 1 - ch[None, :]))          # [H,c,c], zero from the chunk itself on
    S = torch.matmul(carry[None, :, None], sums.reshape(*sums.shape[:4], i * j)).reshape(sums.shape)
    if S_in is not None:
        S = S + _powers(log_decay, C * ch)[None, :, None, :, None, None] * S_in[:, :, None, None]
    out = out + torch.matmul(a, S) * _powers(log_decay, at + 1)[None, :, None, None, :, None]
    return out.reshape(B, H, G, c * C, j)[..., :n, :]


def _to_end(b, v, log_decay, ends, S_in):
    """sum_s lam^(end-1-s) b_s (x) v_s + lam^end S_in over the members of each group."""
    n = b.shape[3]
    far = ends[:, None] - 1 - torch.arange(n, device=b.device)[None, :]      # [B,n]
    w = _powers(log_decay, far).transpose(0, 1)                              # [B,H,n]
    S = torch.matmul((b * w[:, :, None, :, None]).transpose(-1, -2), v).sum(2)
    return S if S_in is None else S + _powers(log_decay, ends).transpose(0, 1)[:, :, None, None] * S_in


def _decay_forward(q, k, v, log_decay, lengths, S_in, want_state):
    B, H, n, dk = k.shape
    alive, ends = _alive(lengths, B, n, q.device)
    m = alive[:, None, None, :, None]
    qf, kf, vf = (torch.where(m, _grouped(x, H), 0.0) for x in (q, k, v))
    y = _mix(qf, kf, vf, log_decay, S_in) / math.sqrt(dk)
    S = _to_end(kf, vf, log_decay, ends, S_in) if want_state else None
    return torch.where(m, y, 0.0).reshape(B, -1, n, v.shape[-1]).to(q.dtype), S


def _decay_token(S, q, k, v, log_decay):
    B, H, dk = k.shape
    S.mul_(_powers(log_decay, torch.ones((), device=S.device))[None, :, None, None])
    S.add_(k.float()[..., None] * v.float()[..., None, :])
    y = torch.matmul(q.float().reshape(B, H, -1, dk), S) / math.sqrt(dk)
    return y.reshape(B, -1, v.shape[-1]).to(q.dtype)


def _decay_gradients(q, k, v, log_decay, dy, lengths, S_in, dS):
    B, H, n, dk = k.shape
    alive, ends = _alive(lengths, B, n, q.device)
    m = alive[:, None, None, :, None]
    qf, kf, vf, df = (torch.where(m, _grouped(x, H), 0.0) for x in (q, k, v, dy))
    back = lambda x: x.flip(3)  # noqa: E731
    scale = 1.0 / math.sqrt(dk)
    dq = _mix(df, vf, kf, log_decay, None if S_in is None else S_in.transpose(-1, -2)) * scale
    G = qf.shape[2]
    wide = lambda x: x.expand(-1, -1, G, -1, -1)  # noqa: E731
    gk = back(_mix(back(wide(vf)), back(df), back(qf), log_decay, None)).sum(2, keepdim=True) * scale
    gv = back(_mix(back(wide(kf)), back(qf), back(df), log_decay, None)).sum(2, keepdim=True) * scale
    gS = None
    if dS is not None:
        far = _powers(log_decay, ends[:, None] - 1 - torch.arange(n, device=q.device)[None, :]).transpose(0, 1)
        gk = gk + torch.matmul(vf, dS.transpose(-1, -2)[:, :, None]) * far[:, :, None, :, None]
        gv = gv + torch.matmul(kf, dS[:, :, None]) * far[:, :, None, :, None]
    if S_in is not None:
        early = _powers(log_decay, torch.arange(n, device=q.device) + 1)[None, :, None, :, None]
        gS = torch.matmul((qf * early).transpose(-1, -2), df).sum(2) * scale
        gS = gS + _powers(log_decay, ends).transpose(0, 1)[:, :, None, None] * dS
    out = [torch.where(m, x, 0.0).reshape(B, -1, n, x.shape[-1]).to(q.dtype) for x in (dq, gk, gv)]
    return out + ([gS] if gS is not None else [])


def _seen(lengths, B, n, device):
    """[B, 1, 1, n, n]: whether a query (row) sees a key (column)."""
    alive, _ = _alive(lengths, B, n, device)
    at = torch.arange(n, device=device)
    return ((at[:, None] >= at[None, :])[None] & alive[:, :, None])[:, None, None]


def _softmax_forward(q, k, v, lengths):
    B, H, n, dk = k.shape
    qf, kf, vf = _grouped(q, H), _grouped(k, H), _grouped(v, H)
    s = torch.matmul(qf, kf.transpose(-1, -2)).div_(math.sqrt(dk))
    s = s.masked_fill_(~_seen(lengths, B, n, q.device), -math.inf)
    top = s.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    y = torch.matmul(p, vf) / total.clamp(min=1e-38)
    lse = (torch.log(total) + top)[..., 0]
    return y.reshape(B, -1, n, v.shape[-1]).to(q.dtype), lse.reshape(B, -1, n)


def _softmax_gradients(q, k, v, y, lse, dy, lengths):
    B, H, n, dk = k.shape
    qf, kf, vf, yf, df = (_grouped(x, H) for x in (q, k, v, y, dy))
    alive, _ = _alive(lengths, B, n, q.device)
    df = torch.where(alive[:, None, None, :, None], df, 0.0)
    s = torch.matmul(qf, kf.transpose(-1, -2)).div_(math.sqrt(dk))
    s = s.masked_fill_(~_seen(lengths, B, n, q.device), -math.inf)
    p = s.sub_(lse.reshape(B, H, -1, n, 1).clamp(min=-3e38)).exp_()
    dv = torch.matmul(p.transpose(-1, -2), df).sum(2, keepdim=True)
    g = torch.matmul(df, vf.transpose(-1, -2)).sub_((df * yf).sum(-1, keepdim=True)).mul_(p).div_(math.sqrt(dk))
    dq = torch.matmul(g, kf)
    dkk = torch.matmul(g.transpose(-1, -2), qf).sum(2, keepdim=True)
    return tuple(x.reshape(B, -1, n, x.shape[-1]).to(q.dtype) for x in (dq, dkk, dv))


def _softmax_token(K, V, lengths, q, k, v):
    B, H, n, dk = K.shape
    b, at = torch.arange(B, device=K.device), lengths.long()
    K[b, :, at] = k
    V[b, :, at] = v
    s = torch.matmul(q.float().reshape(B, H, -1, dk), K.float().transpose(-1, -2)) / math.sqrt(dk)
    seen = torch.arange(n, device=K.device)[None, :] <= at[:, None]
    s = s.masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    y = torch.matmul(p, V.float()) / p.sum(-1, keepdim=True)
    return y.reshape(B, -1, V.shape[-1]).to(q.dtype)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """Bytes: each input (the tokens that count) read once, each output written
    once.  Flops: two products of a token with the state for the recurrences;
    the pairs' products for softmax (two forward, five backward)."""
    op, B, H, G, dk, dv, size = (*(case[k] for k in ("op", "B", "H", "G", "dk", "dv")), SIZE[case["dtype"]])
    if op == "decay_step":
        return {"bytes": B * H * (8.0 * dk * dv + size * (dk + dv) * (G + 1)), "flops": B * H * 2.0 * dk * dv * (G + 1)}
    ends = _lengths_of(case)
    n = case["n"]
    if op == "softmax_step":
        tokens = float(sum(x + 1 for x in ends))
        return {"bytes": H * size * (tokens * (dk + dv) + B * (dk + dv) * (G + 1)),
                "flops": H * G * tokens * 2.0 * (dk + dv)}
    tokens, pairs = float(sum(ends)), float(sum(x * (x + 1) // 2 for x in ends))
    state = B * H * 4.0 * dk * dv
    if op == "decay_prefill":
        return {"bytes": H * size * (tokens * (dk * (G + 1) + dv) + B * n * dv * G) + (2 * state if case["state"] else 0.0),
                "flops": H * tokens * 2.0 * dk * dv * (G + 1)}
    if op == "decay_backward":
        return {"bytes": H * size * (tokens * (dk + dv) * (G + 1) + B * n * (dk * (G + 1) + dv))
                + (3 * state if case["state"] else 0.0),
                "flops": H * tokens * 2.0 * dk * dv * (2 * G + 3)}
    if op == "softmax_prefill":
        return {"bytes": H * size * (tokens * (dk * (G + 1) + dv) + B * n * dv * G) + 4.0 * B * H * G * n,
                "flops": H * G * pairs * 2.0 * (dk + dv)}
    return {"bytes": H * size * (tokens * (dk * (G + 1) + dv * (2 * G + 1)) + B * n * (dk * (G + 1) + dv))
            + 4.0 * H * G * tokens,
            "flops": H * G * pairs * 2.0 * (3 * dk + 2 * dv)}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    def decay_head(q, k, v, g, S, end):
        """One sequence of one head: rows of c q_t S_t and the state, 512 tokens at a time (q [G, n, i])."""
        out = torch.zeros(*q.shape[:2], v.shape[1], dtype=torch.float64, device=q.device)
        for r0 in range(0, end, 512):
            r1 = min(end, r0 + 512)
            i = torch.arange(r1 - r0, dtype=torch.float64, device=q.device)
            d = i[:, None] - i[None, :]
            w = torch.where(d >= 0, torch.exp(g * d.clamp(min=0)), 0.0)
            out[:, r0:r1] = ((q[:, r0:r1] @ k[r0:r1].T) * w) @ v[r0:r1] + (q[:, r0:r1] @ S) * torch.exp(g * (i + 1))[:, None]
            S = S * torch.exp(g * (r1 - r0)) + (k[r0:r1] * torch.exp(g * (r1 - r0 - 1 - i))[:, None]).T @ v[r0:r1]
        return out, S

    t = _draw_inputs(case, seed)
    op, B, H, G, dk, dv = (case[k] for k in ("op", "B", "H", "G", "dk", "dv"))
    f = {name: x.double() for name, x in t.items() if x is not None}
    ends, scale = _lengths_of(case), 1.0 / math.sqrt(dk)
    zeros = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")  # noqa: E731
    if op == "decay_step":
        S = f["S"] * torch.exp(f["log_decay"])[:, None, None] + f["k"][..., None] * f["v"][..., None, :]
        y = (f["q"].view(B, H, G, dk) @ S) * scale
        return [y.reshape(B, H * G, dv), S]
    if op == "softmax_step":
        K, V, y = t["K"].clone(), t["V"].clone(), zeros(B, H * G, dv)
        for b, e in enumerate(ends):
            K[b, :, e], V[b, :, e] = t["k"][b], t["v"][b]
            for h in range(H):
                p = torch.softmax(f["q"][b, h * G:(h + 1) * G] @ K[b, h, :e + 1].double().T * scale, -1)
                y[b, h * G:(h + 1) * G] = p @ V[b, h, :e + 1].double()
        return [y, K, V]
    n = case["n"]
    q = f["q"].view(B, H, G, n, dk)
    if op == "decay_prefill":
        y, S = zeros(B, H, G, n, dv), zeros(B, H, dk, dv)
        for b in range(B):
            for h in range(H):
                S0 = f["S_in"][b, h] if case["state"] else S[b, h]
                y[b, h], S[b, h] = decay_head(q[b, h], f["k"][b, h], f["v"][b, h], f["log_decay"][h], S0, ends[b])
        return [y.view(B, H * G, n, dv) * scale] + ([S] if case["state"] else [])
    if op == "decay_backward":
        # c q_t S_t . dy_t by halves: dq from the states, dk and dv from the states of the reversed sequence
        dy = f["dy"].view(B, H, G, n, dv)
        gq, gk, gv, gS = zeros(B, H, G, n, dk), zeros(B, H, n, dk), zeros(B, H, n, dv), zeros(B, H, dk, dv)
        for b in range(B):
            e = ends[b]
            for h in range(H):
                g, k, v = f["log_decay"][h], f["k"][b, h], f["v"][b, h]
                S0 = f["S_in"][b, h] if case["state"] else gS[b, h]
                gq[b, h] = decay_head(dy[b, h], v, k, g, S0.T, e)[0] * scale
                rk, rv = k[:e].flip(0), v[:e].flip(0)
                late = torch.exp(g * torch.arange(e, dtype=torch.float64, device="cuda"))[:, None]
                U = f["dS"][b, h] if case["state"] else gS[b, h]
                if case["state"]:
                    gk[b, h, :e] = ((rv @ U.T) * late).flip(0)
                    gv[b, h, :e] = ((rk @ U) * late).flip(0)
                total = U * torch.exp(g * (e - 1))
                for m in range(G):
                    rq, rd = q[b, h, m, :e].flip(0), dy[b, h, m, :e].flip(0)
                    gv[b, h, :e] += decay_head(rk[None], rq, rd, g, zeros(dk, dv), e)[0][0].flip(0) * scale
                    x, last = decay_head(rv[None], rd, rq, g, zeros(dv, dk), e)
                    gk[b, h, :e] += x[0].flip(0) * scale
                    total = total + last.T * scale
                gS[b, h] = total * torch.exp(g)
        out = [gq.view(B, H * G, n, dk), gk, gv]
        return out + ([gS] if case["state"] else [])
    y, lse = zeros(B, H, G, n, dv), zeros(B, H, G, n) - math.inf
    out = [zeros(B, H, G, n, dk), zeros(B, H, n, dk), zeros(B, H, n, dv)]
    for b in range(B):
        for h in range(H):
            k, v = f["k"][b, h], f["v"][b, h]
            for m in range(G):
                for r0 in range(0, ends[b], 2048):
                    r1 = min(ends[b], r0 + 2048)
                    s = q[b, h, m, r0:r1] @ k[:r1].T * scale
                    s.masked_fill_(torch.ones_like(s, dtype=torch.bool).triu_(r0 + 1), -math.inf)
                    z = torch.logsumexp(s, -1, keepdim=True)
                    p = s.sub_(z).exp_()
                    o = p @ v[:r1]
                    if op == "softmax_prefill":
                        y[b, h, m, r0:r1], lse[b, h, m, r0:r1] = o, z[:, 0]
                        continue
                    d = f["dy"].view(B, H, G, n, dv)[b, h, m, r0:r1]
                    g = p * (d @ v[:r1].T - (d * o).sum(-1, keepdim=True)) * scale
                    out[0][b, h, m, r0:r1] = g @ k[:r1]
                    out[1][b, h, :r1] += g.T @ q[b, h, m, r0:r1]
                    out[2][b, h, :r1] += p.T @ d
    if op == "softmax_prefill":
        return [y.view(B, H * G, n, dv), lse.view(B, H * G, n)]
    return [out[0].view(B, H * G, n, dk)] + out[1:]
