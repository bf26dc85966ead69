"""The gated delta rule, rotary positions and attention over a 4-bit cache, as measurable cases.

Each case is one call that a serving or training program makes of the entry
points: a prompt through a delta-rule layer (delta_prefill), one token of every
sequence (delta_step), the gradients of a prompt (delta_backward); queries and
keys turned by their positions (rotary) and gradients turned back
(rotary_backward); one token of every sequence over caches of 4 bits an entry
(softmax_step_packed), and a prompt's keys and values put into such caches and
read back (packed_write, packed_read).  With c = 1 / sqrt(d_k),

    delta:   S' = exp(g_t) S_{t-1},  u_t = beta_t (v_t - k_t S'),  S_t = S' + k_t (x) u_t,  y_t = c q_t S_t
             for every value head; G of them share the queries and keys of one head
    rotary:  (a, b) -> s (a cos x - b sin x, b cos x + a sin x), x = position times the pair's frequency
    packed:  32 entries of a row share a scale and a least value in bfloat16; an entry stands for
             least + scale * code, code in 0..15

Keys of the delta rule have length one, as such layers make them; beta is in (0, 1) and
the mean decay runs from 2^-2 to 2^-10 a token over the heads.  What else is not said is N(0, 1).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def listed():
    return [
        # a batch of prompts through one layer of large heads, the states kept for generation
        dict(name="delta_prompt_batch", op="delta_prefill", B=8, H=16, G=1, n=4096, dk=128, dv=128, dtype="bf16",
             lengths=False, state=True),
        # a few short float32 prompts of odd sizes in a padded batch, going on from earlier states
        dict(name="delta_prompt_ragged", op="delta_prefill", B=3, H=2, G=2, n=777, dk=24, dv=40, dtype="f32",
             lengths=True, state=True),
        # one token of one sequence: launch latency
        dict(name="delta_token_one", op="delta_step", B=1, H=16, G=1, dk=64, dv=64, dtype="bf16"),
        # one token of a serving batch, two value heads to each key head: 268 MB of state read and written
        dict(name="delta_token_batch", op="delta_step", B=64, H=16, G=2, dk=128, dv=128, dtype="bf16"),
        # the gradients of a training batch
        dict(name="delta_gradients_batch", op="delta_backward", B=4, H=16, G=1, n=2048, dk=128, dv=128, dtype="bf16",
             lengths=False, state=False),
        # float32 gradients at odd sizes in a padded batch, with the gradients of both states
        dict(name="delta_gradients_ragged", op="delta_backward", B=2, H=3, G=2, n=555, dk=48, dv=32, dtype="f32",
             lengths=True, state=True),
        # the queries and keys of a batch of prompts with grouped query heads
        dict(name="rotary_prompt", op="rotary", B=4, H=8, G=4, n=4096, d=128, pairs=64, interleaved=False, dtype="bf16"),
        # one token of a serving batch, a quarter of the head turned, neighbours paired: launch latency
        dict(name="rotary_token", op="rotary", B=16, H=8, G=1, n=1, d=64, pairs=8, interleaved=True, dtype="f32"),
        # gradients of a batch of odd sizes, neighbours paired, most of the head turned
        dict(name="rotary_gradients", op="rotary_backward", B=3, H=4, G=2, n=2111, d=80, pairs=30, interleaved=True,
             dtype="bf16"),
        # one token of one sequence with a short cache: launch latency
        dict(name="packed_token_one", op="softmax_step_packed", B=1, H=8, G=1, n=1000, dk=64, dv=64, dtype="bf16"),
        # one token of a serving batch with sequences of many lengths, four query heads to each cached head
        dict(name="packed_token_batch", op="softmax_step_packed", B=16, H=8, G=4, n=16384, dk=128, dv=128,
             dtype="bf16"),
        # the keys and values of a padded batch of prompts put into the caches, and read back for a prompt that follows
        dict(name="packed_prompt", op="packed", B=4, H=8, n=4000, dk=128, dv=128, dtype="bf16"),
    ]


# ------------------------------------------------------------------ drawn cases

def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """One more case of these ranges: 1 to 16384 tokens, heads of 8 to 128, every type, direction and form."""
    op = rng.choice(["delta_prefill", "delta_prefill", "delta_step", "delta_backward", "delta_backward", "rotary",
                     "rotary_backward", "softmax_step_packed", "softmax_step_packed", "packed"])
    while True:
        case = dict(op=op, B=_log_int(rng, 1, 16), H=rng.choice([1, 2, 4, 8, 16, rng.randint(1, 16)]))
        if op != "packed":
            case["G"] = rng.choice([1, 1, 2, 4, rng.randint(1, 8)])
        dk = rng.choice([16, 32, 64, 64, 96, 128, 128, rng.randint(8, 128)])
        if op.startswith("rotary"):
            case["n"] = rng.choice([1, _log_int(rng, 1, 8192)])
            case["d"] = dk = max(2, dk)
            case["pairs"] = rng.choice([dk // 2, dk // 2, max(1, dk // 8), rng.randint(1, dk // 2)])
            case["interleaved"] = rng.random() < 0.5
        else:
            case["dk"], case["dv"] = dk, dk if rng.random() < 0.7 else rng.choice([16, 32, 64, 128, rng.randint(8, 128)])
        case["dtype"] = rng.choice(["bf16", "bf16", "f32"])
        if op == "delta_step":
            case["B"] = _log_int(rng, 1, 64)
        elif op == "softmax_step_packed":
            case["n"] = _log_int(rng, 1, 16384)
        elif op == "packed":
            case["n"] = _log_int(rng, 1, 8192)
        elif op.startswith("delta"):
            case["n"] = _log_int(rng, 1, 4096)
            case["lengths"] = rng.random() < 0.5
            case["state"] = rng.random() < 0.5
        w = work(case)
        if w["bytes"] > 3.4e8 or (op == "softmax_step_packed" and w["bytes"] > 1.6e8):
            continue
        if op in ("delta_prefill", "delta_backward"):
            heads = case["B"] * case["H"] * case["G"]
            most = 8 * 16 * 4096 if op == "delta_prefill" else 4 * 16 * 2048
            if heads * case["n"] > most or heads * case["n"] * case["dk"] * case["dv"] > most * 128 * 128:
                continue
        return case


# ------------------------------------------------------------------ inputs

def _lengths_of(case):
    """Tokens of each sequence: all, or from few in the first to all in the last; of a cache, those before the call."""
    B, n = case["B"], case.get("n", 1)
    if case["op"] == "softmax_step_packed":
        return [(n - 1) * (b + 1) // B for b in range(B)]
    if case["op"] != "packed" and not case.get("lengths"):
        return [n] * B
    return [n * b // max(1, B - 1) if B > 1 else (n + 1) // 2 for b in range(B)]


def _starts_of(case):
    """The positions (rotary) or cache rows (packed) that sequences start at: prompts that follow on others."""
    return [(37 * b) % 101 if case["op"] == "packed" else (5003 * b) % 30011 for b in range(case["B"])]


def _draw_inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    dt = DTYPES[case["dtype"]]
    op, B, H, G, n = case["op"], case["B"], case["H"], case.get("G", 1), case.get("n", 1)

    def normal(*shape, dtype=dt, unit=False):
        x = torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)
        return (x / x.square().sum(-1, keepdim=True).sqrt() if unit else x).to(dtype)

    def whole(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    if op.startswith("rotary"):
        q, k = normal(B, H * G, n, case["d"]), normal(B, H, n, case["d"])
        at = whole(_starts_of(case))[:, None] + torch.arange(n, dtype=torch.int32, device="cuda")
        pairs = case["pairs"]
        freq = (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float().cuda()
        return dict(q=q, k=k, positions=at.contiguous(), freq=freq, scale=1.0 if case["interleaved"] else 1.125)
    dk, dv = case["dk"], case["dv"]
    if op == "packed":
        return dict(k=normal(B, H, n, dk), v=normal(B, H, n, dv), first=whole(_starts_of(case)),
                    counts=whole(_lengths_of(case)))
    if op == "softmax_step_packed":
        return dict(q=normal(B, H * G, dk), k=normal(B, H, dk), v=normal(B, H, dv), oldK=normal(B, H, n, dk),
                    oldV=normal(B, H, n, dv), lengths=whole(_lengths_of(case)))
    rows = () if op == "delta_step" else (n,)
    t = dict(q=normal(B, H, *rows, dk, unit=True), k=normal(B, H, *rows, dk, unit=True), v=normal(B, H * G, *rows, dv))
    rate = torch.exp2(-torch.linspace(2.0, 10.0, H * G)) if H * G > 1 else torch.tensor([2.0 ** -6])
    size = torch.nn.functional.softplus(normal(B, H * G, *rows, dtype=torch.float32))
    t["g"] = -size * rate.cuda().reshape(1, -1, *([1] * len(rows)))
    t["beta"] = torch.sigmoid(normal(B, H * G, *rows, dtype=torch.float32))
    state = lambda: normal(B, H * G, dk, dv, dtype=torch.float32)  # noqa: E731
    if op == "delta_step":
        t["S"] = state()
        return t
    t["lengths"] = whole(_lengths_of(case)) if case["lengths"] else None
    if op == "delta_backward":
        t["dy"] = normal(B, H * G, n, dv)
    if case["state"]:
        t["S_in"] = state()
        if op == "delta_backward":
            t["dS"] = state()
    return t


def prepare(case, seed):
    t = _draw_inputs(case, seed)
    t["case"] = case
    if case["op"] == "softmax_step_packed":  # what earlier tokens have left in the caches
        t["K"], t["V"] = _pack(t.pop("oldK")), _pack(t.pop("oldV"))
    if case["op"] == "packed":
        rows = case["n"] + 128
        t["K"], t["V"] = (torch.zeros(case["B"], case["H"], rows, _row_bytes(case[d]), dtype=torch.uint8, device="cuda")
                          for d in ("dk", "dv"))
    return t


# ------------------------------------------------------------------ one pass

def run(state):
    case, t = state["case"], state
    op = case["op"]
    if own:
        import paper_2602_00294_amd as sata
        if op == "delta_prefill":
            y, S = sata.delta_prefill(t["q"], t["k"], t["v"], t["g"], t["beta"], lengths=t["lengths"],
                                      S_in=t.get("S_in"), want_state=case["state"])
            return [y] + ([S] if case["state"] else [])
        if op == "delta_step":
            return [sata.delta_step(t["S"], t["q"], t["k"], t["v"], t["g"], t["beta"]), t["S"]]
        if op == "delta_backward":
            out = sata.delta_backward(t["q"], t["k"], t["v"], t["g"], t["beta"], t["dy"], lengths=t["lengths"],
                                      S_in=t.get("S_in"), dS=t.get("dS"))
            return list(out[:5]) + ([out[5]] if case["state"] else [])
        if op.startswith("rotary"):
            turn = sata.rotary if op == "rotary" else sata.rotary_backward
            return list(turn(t["q"], t["k"], t["positions"], t["freq"], interleaved=case["interleaved"],
                             scale=t["scale"]))
        if op == "softmax_step_packed":
            y = sata.softmax_step_packed(t["K"], t["V"], t["lengths"], t["q"], t["k"], t["v"])
            # (the rows that the call has added, as the values they stand for)
            return [y] + [sata.packed_read(t[c], t["lengths"], 1, case[d], torch.float32) for c, d in (("K", "dk"), ("V", "dv"))]
        sata.packed_write(t["K"], t["V"], t["first"], t["k"], t["v"], counts=t["counts"])
        return [sata.packed_read(t[c], t["first"], case["n"], case[d], t["k"].dtype) for c, d in (("K", "dk"), ("V", "dv"))]
    if op == "delta_prefill":
        y, S = _delta_forward(t, want_state=case["state"])
        return [y] + ([S] if case["state"] else [])
    if op == "delta_step":
        return [_delta_token(t), t["S"]]
    if op == "delta_backward":
        return _delta_gradients(t)
    if op.startswith("rotary"):
        return [_turned(x, t["positions"], t["freq"], case["interleaved"], t["scale"], op != "rotary")
                for x in (t["q"], t["k"])]
    if op == "softmax_step_packed":
        return _packed_token(t)
    return _packed_prompt(t)


# ------------------------------------------------------------------ the plain forms, in 32 bits

CHUNK = 64


def _inverse(A):
    """(I + A)^-1 of strictly lower triangular matrices [..., C, C]: blocks of 1, 2, 4.. on the diagonal."""
    C = A.shape[-1]
    at = torch.arange(C, device=A.device)
    T = torch.eye(C, device=A.device).expand(A.shape)
    s = 1
    while s < C:
        below = ((at[:, None] // s) % 2 == 1) & (at[:, None] // s - 1 == at[None, :] // s)
        T = T - torch.matmul(torch.matmul(T, A * below), T)
        s *= 2
    return T


def _delta_parts(t):
    """Tokens in chunks of 64 ([B, H, chunks, 64, d]; padding leaves a state alone), and what each chunk's pairs are."""
    q, k, v = t["q"], t["k"], t["v"]
    B, Hk, n, dk = k.shape
    H, dv = v.shape[1], v.shape[-1]
    c = (n + CHUNK - 1) // CHUNK
    ends = torch.full((B,), n, device=q.device) if t["lengths"] is None else t["lengths"].long()
    alive = torch.arange(n, device=q.device)[None, :] < ends[:, None]

    def cut(x, wide):
        x = torch.where(alive.reshape(B, 1, n, *([1] * (x.dim() - 3))), x.float(), 0.0)
        x = x.repeat_interleave(H // Hk, dim=1) if wide else x
        pad = [0, 0] * (x.dim() - 3) + [0, c * CHUNK - n]
        return torch.nn.functional.pad(x, pad).reshape(B, H, c, CHUNK, *x.shape[3:])

    p = dict(q=cut(q, True), k=cut(k, True), v=cut(v, False), beta=cut(t["beta"], False)[..., None], alive=alive)
    sums = cut(t["g"], False).double().cumsum(-1)
    at = torch.arange(CHUNK, device=q.device)
    later = at[:, None] >= at[None, :]
    D = torch.where(later, torch.exp(torch.where(later, sums[..., :, None] - sums[..., None, :], 0.0)), 0.0).float()
    p["early"] = torch.exp(sums).float()[..., None]
    p["late"] = torch.exp(sums[..., -1:] - sums).float()[..., None]
    p["whole"] = torch.exp(sums[..., -1]).float()[..., None, None]
    kt = p["k"].transpose(-1, -2)
    p["scale"] = 1.0 / math.sqrt(dk)
    p["D"], p["before"] = D, at[:, None] > at[None, :]
    p["L"] = torch.matmul(p["k"], kt) * D * p["before"]
    p["P"] = torch.matmul(p["q"], kt) * D * p["scale"]
    p["T"] = _inverse(p["beta"] * p["L"])
    S = t.get("S_in")
    p["S"] = torch.zeros(B, H, dk, dv, device=q.device) if S is None else S
    return p


def _delta_states(p):
    """The states before every chunk and after the last, and the tokens' updates u."""
    values = torch.matmul(p["T"], p["beta"] * p["v"])
    keys = torch.matmul(p["T"], p["beta"] * p["early"] * p["k"])
    late = (p["late"] * p["k"]).transpose(-1, -2)
    S, states, updates = p["S"], [p["S"]], []
    for c in range(p["k"].shape[2]):
        u = values[:, :, c] - torch.matmul(keys[:, :, c], S)
        S = p["whole"][:, :, c] * S + torch.matmul(late[:, :, c], u)
        states.append(S)
        updates.append(u)
    return torch.stack(states, 2), torch.stack(updates, 2)


def _tokens(x, n):
    """[B, H, chunks, 64, ...] -> [B, H, n, ...]"""
    return x.reshape(*x.shape[:2], -1, *x.shape[4:])[:, :, :n]


def _delta_forward(t, want_state):
    p = _delta_parts(t)
    S, u = _delta_states(p)
    y = p["scale"] * p["early"] * torch.matmul(p["q"], S[:, :, :-1]) + torch.matmul(p["P"], u)
    y = torch.where(p["alive"][:, None, :, None], _tokens(y, t["q"].shape[2]), 0.0)
    return y.to(t["q"].dtype), S[:, :, -1].contiguous() if want_state else None


def _delta_token(t):
    S, G = t["S"], t["v"].shape[1] // t["k"].shape[1]
    k, q = (t[x].float().repeat_interleave(G, dim=1) for x in ("k", "q"))
    S.mul_(torch.exp(t["g"])[..., None, None])
    u = t["beta"][..., None] * (t["v"].float() - torch.matmul(k[..., None, :], S)[..., 0, :])
    S.add_(k[..., None] * u[..., None, :])
    return (torch.matmul(q[..., None, :], S)[..., 0, :] / math.sqrt(k.shape[-1])).to(t["q"].dtype)


def _delta_gradients(t):
    p = _delta_parts(t)
    S, u = _delta_states(p)
    B, H, c, C, dv = u.shape
    n = t["q"].shape[2]
    dy = torch.where(p["alive"][:, None, :, None], t["dy"].float(), 0.0)
    dy = torch.nn.functional.pad(dy, (0, 0, 0, c * C - n)).reshape(B, H, c, C, dv)
    flip = lambda x: x.transpose(-1, -2)  # noqa: E731
    q, k, early, late, beta = p["q"], p["k"], p["early"], p["late"], p["beta"]
    dS = t.get("dS")
    dS = torch.zeros_like(S[:, :, 0]) if dS is None else dS
    own_pairs, turned = torch.matmul(flip(p["P"]), dy), flip(p["T"])
    into = torch.matmul(flip(p["scale"] * early * q), dy)
    back, behind, z = flip(early * k), [], []
    for i in reversed(range(c)):
        behind.append(dS)
        x = torch.matmul(turned[:, :, i], own_pairs[:, :, i] + late[:, :, i] * torch.matmul(k[:, :, i], dS))
        dS = p["whole"][:, :, i] * dS + into[:, :, i] - torch.matmul(back[:, :, i], beta[:, :, i] * x)
        z.append(x)
    behind, z = torch.stack(behind[::-1], 2), torch.stack(z[::-1], 2)
    before, after = S[:, :, :-1], S[:, :, 1:]
    miss = p["v"] - early * torch.matmul(k, before) - torch.matmul(p["L"], u)
    dbeta = (z * miss).sum(-1)
    dv_ = beta * z
    one = torch.matmul(dy, flip(u)) * p["D"] * p["scale"]
    two = torch.matmul(-dv_, flip(u)) * p["D"] * p["before"]
    dq = p["scale"] * early * torch.matmul(dy, flip(before)) + torch.matmul(one, k)
    asked = torch.matmul(two, k) - early * torch.matmul(dv_, flip(before))
    kept = torch.matmul(flip(one), q) + torch.matmul(flip(two), k) + late * torch.matmul(u, flip(behind))
    at = (q.double() * dq + k.double() * asked - k.double() * kept).sum(-1)
    dg = at.flip(-1).cumsum(-1).flip(-1) + (behind.double() * after).sum((-1, -2))[..., None]
    G = H // t["k"].shape[1]
    dk = asked + kept
    out = []
    for x, shared in ((dq, True), (dk, True), (dv_, False), (dg.float(), False), (dbeta, False)):
        x = _tokens(x, n)
        x = torch.where(p["alive"].reshape(B, 1, n, *([1] * (x.dim() - 3))), x, 0.0)
        x = x.reshape(B, H // G, G, *x.shape[2:]).sum(2) if shared else x
        out.append(x.to(t["q"].dtype) if x.dim() == 4 else x.contiguous())
    return out + ([dS] if t.get("dS") is not None else [])


def _turned(x, positions, freq, interleaved, scale, back):
    """Pairs of the first 2 len(freq) entries turned by positions times freq; the angles in 64 bits."""
    R, d = freq.shape[0], x.shape[-1]
    angle = positions.double()[:, None, :, None] * freq.double()
    cos, sin = (scale * torch.cos(angle)).float(), (scale * torch.sin(angle)).float()
    sin = -sin if back else sin
    f = x[..., :2 * R].float()
    a, b = (f[..., 0::2], f[..., 1::2]) if interleaved else (f[..., :R], f[..., R:])
    a, b = a * cos - b * sin, b * cos + a * sin
    f = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((f.to(x.dtype), x[..., 2 * R:]), -1) if 2 * R < d else f.to(x.dtype)


# A packed row: 16 bytes of codes for each 32 entries (of 1, 2 or 4 groups), byte a * groups + g holding entries
# 32 g + a (low four bits) and 32 g + 16 + a; then each group's scale and least value in bfloat16.

def _groups(d):
    return 1 if d <= 32 else 2 if d <= 64 else 4


def _row_bytes(d):
    return 20 * _groups(d)


def _pack(x):
    """[..., d] -> [..., row bytes]: scale (max - min) / 15 and min of 32 entries in bfloat16, the nearest codes."""
    d, g = x.shape[-1], _groups(x.shape[-1])
    f = torch.nn.functional.pad(x.float(), (0, 32 * g - d)).reshape(*x.shape[:-1], g, 32)
    there = (torch.arange(32 * g, device=x.device) < d).reshape(g, 32)
    least = torch.where(there, f, math.inf).amin(-1)
    most = torch.where(there, f, -math.inf).amax(-1)
    used = there.any(-1)
    least, most = torch.where(used, least, 0.0), torch.where(used, most, 0.0)
    scale = ((0.5 * most - 0.5 * least) / 7.5).bfloat16()
    low = least.bfloat16()
    half = 0.5 * scale.float()[..., None]
    code = ((0.5 * f - 0.5 * low.float()[..., None]) / torch.where(half > 0, half, 1.0)).round().clamp(0, 15)
    code = torch.where(there & (half > 0), code, 0.0).to(torch.uint8).transpose(-1, -2)   # [..., 32, g]
    both = (code[..., :16, :] | (code[..., 16:, :] << 4)).flatten(-2)
    return torch.cat((both, torch.stack((scale, low), -1).flatten(-2).view(torch.uint8)), -1)


def _unpack(rows, d):
    """[..., row bytes] -> the values [..., d] in 32 bits."""
    g = _groups(d)
    both = rows[..., :16 * g].unflatten(-1, (16, g)).transpose(-1, -2)
    code = torch.cat((both & 15, both >> 4), -1).float()                                 # [..., g, 32]
    p = rows[..., 16 * g:].contiguous().view(torch.bfloat16).float().unflatten(-1, (g, 2))
    return (p[..., 1:] + p[..., :1] * code).flatten(-2)[..., :d]


def _packed_token(t):
    K, V, q, k, v = (t[x] for x in ("K", "V", "q", "k", "v"))
    B, H, n = K.shape[:3]
    dk, dv = k.shape[-1], v.shape[-1]
    b, at = torch.arange(B, device=K.device), t["lengths"].long()
    rows = _pack(k), _pack(v)
    K[b, :, at], V[b, :, at] = rows
    s = torch.matmul(q.float().reshape(B, H, -1, dk), _unpack(K, dk).transpose(-1, -2)) / math.sqrt(dk)
    seen = torch.arange(n, device=K.device)[None, :] <= at[:, None]
    s = s.masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    y = torch.matmul(p, _unpack(V, dv)) / p.sum(-1, keepdim=True)
    return [y.reshape(B, -1, dv).to(q.dtype)] + [_unpack(x, d)[:, :, None] for x, d in zip(rows, (dk, dv))]


def _packed_prompt(t):
    B, H, n = t["k"].shape[:3]
    at = t["first"].long()[:, None] + torch.arange(n, device=t["k"].device)              # [B, n]
    live = torch.arange(n, device=at.device)[None, :] < t["counts"].long()[:, None]
    out = []
    for cache, x in ((t["K"], t["k"]), (t["V"], t["v"])):
        index = at[:, None, :, None].expand(-1, H, -1, cache.shape[-1])
        rows = torch.where(live[:, None, :, None], _pack(x), cache.gather(2, index))
        cache.scatter_(2, index, rows)
        out.append(_unpack(cache.gather(2, index), x.shape[-1]).to(x.dtype))
    return out


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """Bytes: each input (the tokens that count) read once, each output written
    once.  Flops: the products of a token with its state (three forward, nine for
    gradients, the forward's two among them); the cached rows' two products; six operations a turned pair."""
    op, B, H, G, size = case["op"], case["B"], case["H"], case.get("G", 1), SIZE[case["dtype"]]
    n, ends = case.get("n", 1), _lengths_of(case)
    if op.startswith("rotary"):
        rows = B * n * H * (G + 1)
        return {"bytes": 2.0 * size * rows * case["d"] + 4.0 * B * n, "flops": 6.0 * rows * case["pairs"]}
    dk, dv = case["dk"], case["dv"]
    if op == "packed":
        rows, kept = float(B * H * n), float(H * sum(ends))
        bits = _row_bytes(dk) + _row_bytes(dv)
        return {"bytes": kept * (size * (dk + dv) + bits) + rows * (bits + size * (dk + dv)), "flops": 6.0 * kept * (dk + dv)}
    if op == "softmax_step_packed":
        tokens = float(sum(x + 1 for x in ends))
        return {"bytes": H * (tokens * (_row_bytes(dk) + _row_bytes(dv)) + B * (size * (dk + dv) * (G + 1) + 4 * (dk + dv))),
                "flops": H * G * tokens * 2.0 * (dk + dv)}
    if op == "delta_step":
        return {"bytes": B * H * G * (8.0 * dk * dv + 2 * size * dv + 8) + B * H * 2.0 * size * dk,
                "flops": B * H * G * 7.0 * dk * dv}
    tokens, state = float(sum(ends)), B * H * G * 4.0 * dk * dv
    rows = H * size * tokens * (2 * dk + G * dv) + 8.0 * H * G * tokens
    if op == "delta_prefill":
        return {"bytes": rows + size * B * H * G * n * dv + (2 * state if case["state"] else 0.0),
                "flops": H * G * tokens * 6.0 * dk * dv}
    return {"bytes": rows + size * H * G * tokens * dv + B * H * n * (size * (2 * dk + G * dv) + 8.0 * G)
            + (3 * state if case["state"] else 0.0),
            "flops": H * G * tokens * 18.0 * dk * dv}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    t = _draw_inputs(case, seed)
    op, B, H, G, n = case["op"], case["B"], case["H"], case.get("G", 1), case.get("n", 1)

    def values_of(x):
        """What a row's entries stand for, group by group: bfloat16 scale and least value, codes to the nearest."""
        out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
        for g in range(0, x.shape[-1], 32):
            f = x[..., g:g + 32].float()
            lo, hi = f.min(-1, keepdim=True).values, f.max(-1, keepdim=True).values
            step = ((hi / 2 - lo / 2) / 7.5).bfloat16().double()
            lo = lo.bfloat16().double()
            code = torch.where(step > 0, (f.double() - lo) / torch.where(step > 0, step, 1.0), 0.0).round().clamp(0, 15)
            out[..., g:g + 32] = lo + step * code
        return out

    if op.startswith("rotary"):
        R, out = case["pairs"], []
        angle = t["positions"].double()[:, None, :, None] * t["freq"].double()
        spin = t["scale"] * torch.polar(torch.ones_like(angle), -angle if op != "rotary" else angle)
        for x in (t["q"].double(), t["k"].double()):
            i = torch.arange(R, device=x.device)
            a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R)
            z = torch.complex(x[..., a], x[..., b]) * spin
            x = x.clone()
            x[..., a], x[..., b] = z.real, z.imag
            out.append(x)
        return out
    dk, dv = case["dk"], case["dv"]
    if op == "packed":
        out = []
        for x in (t["k"], t["v"]):
            w = values_of(x)
            for b, count in enumerate(_lengths_of(case)):
                w[b, :, count:] = 0.0
            out.append(w)
        return out
    if op == "softmax_step_packed":
        y, k, v = torch.zeros(B, H * G, dv, dtype=torch.float64, device="cuda"), values_of(t["k"]), values_of(t["v"])
        for b, e in enumerate(_lengths_of(case)):
            for h in range(H):
                K = torch.cat((values_of(t["oldK"][b, h, :e]), k[b, h, None]))
                V = torch.cat((values_of(t["oldV"][b, h, :e]), v[b, h, None]))
                y[b, h * G:(h + 1) * G] = torch.softmax(t["q"][b, h * G:(h + 1) * G].double() @ K.T / math.sqrt(dk), -1) @ V
        return [y, k[:, :, None], v[:, :, None]]

    # the delta rule, token by token; heads [B, H, G] with the shared queries and keys [B, H, 1]
    c = 1.0 / math.sqrt(dk)
    f = {x: t[x].double() for x in ("q", "k", "v", "g", "beta")}
    if op == "delta_step":
        S = t["S"].double().view(B, H, G, dk, dv) * torch.exp(f["g"]).view(B, H, G, 1, 1)
        k, q = f["k"].view(B, H, 1, dk, 1), f["q"].view(B, H, 1, dk, 1)
        u = f["beta"].view(B, H, G, 1) * (f["v"].view(B, H, G, dv) - (k * S).sum(-2))
        S = S + k * u[..., None, :]
        return [(q * S).sum(-2).view(B, H * G, dv) * c, S.view(B, H * G, dk, dv)]
    live = torch.arange(n, device="cuda")[None, :] < torch.tensor(_lengths_of(case), device="cuda")[:, None]  # [B, n]
    live = live.double().view(B, 1, 1, n)
    q, k = f["q"].view(B, H, 1, n, dk), f["k"].view(B, H, 1, n, dk)
    v = f["v"].view(B, H, G, n, dv)
    decay, beta = torch.exp(f["g"].view(B, H, G, n) * live), f["beta"].view(B, H, G, n) * live
    first = t["S_in"].double().view(B, H, G, dk, dv) if case["state"] else torch.zeros(B, H, G, dk, dv, dtype=torch.float64, device="cuda")
    back = op == "delta_backward"
    if back:
        kept = torch.empty(n, *first.shape, dtype=torch.float64, device="cuda")  # exp(g_t) S_{t-1}
    S, y = first, torch.zeros(B, H, G, n, dv, dtype=torch.float64, device="cuda")
    err = torch.zeros_like(y)
    for i in range(n):
        S = S * decay[..., i, None, None]
        if back:
            kept[i] = S
        err[..., i, :] = v[..., i, :] - (k[..., i, None, :] @ S)[..., 0, :]
        S = S + k[..., i, :, None] * (beta[..., i, None] * err[..., i, :])[..., None, :]
        if not back:
            y[..., i, :] = (q[..., i, None, :] @ S)[..., 0, :] * (c * live[..., i, None])
    if not back:
        return [y.view(B, H * G, n, dv)] + ([S.view(B, H * G, dk, dv)] if case["state"] else [])
    dy = t["dy"].double().view(B, H, G, n, dv) * live[..., None]
    dS = t["dS"].double().view(B, H, G, dk, dv) if case["state"] else torch.zeros_like(first)
    gq, gk = torch.zeros(B, H, G, n, dk, dtype=torch.float64, device="cuda"), torch.zeros(B, H, G, n, dk, dtype=torch.float64, device="cuda")
    gv, gg, gb = torch.zeros_like(y), torch.zeros_like(beta), torch.zeros_like(beta)
    for i in reversed(range(n)):
        before, ki, qi, d = kept[i], k[..., i, :], q[..., i, :], dy[..., i, :]
        u = beta[..., i, None] * err[..., i, :]
        gq[..., i, :] = c * ((before @ d[..., None])[..., 0] + ki * (u * d).sum(-1, keepdim=True))
        dS = dS + c * qi[..., None] * d[..., None, :]
        du = (ki[..., None, :] @ dS)[..., 0, :]
        gb[..., i] = (du * err[..., i, :]).sum(-1)
        gv[..., i, :] = beta[..., i, None] * du
        gk[..., i, :] = (dS @ u[..., None])[..., 0] - (before @ gv[..., i, :, None])[..., 0]
        dS = dS - ki[..., None] * gv[..., i, None, :]
        gg[..., i] = (dS * before).sum((-1, -2))
        dS = dS * decay[..., i, None, None]
    gk, gg, gb = gk * live[..., None], gg * live, gb * live
    out = [gq.sum(2), gk.sum(2), gv.view(B, H * G, n, dv), gg.view(B, H * G, n), gb.view(B, H * G, n)]
    return out + ([dS.view(B, H * G, dk, dv)] if case["state"] else [])
