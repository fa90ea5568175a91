"""The operators of a causal history encoder, as cases to be timed: norms and position rotation of query and key heads, attention
over packed user histories, and the softmax cross entropy over an item catalogue, each with its gradients.

`run` computes an operator in its plain form (elementary torch operations in fp32) or, where `own` is set, with the calls of
`paper_2510_18239_amd.binding`.  `exact` computes it in fp64, user by user and head by head.

Widths and lengths are those of `synth.CONFIGS` (d = 128 and 256 with four heads, histories of up to 16384 items, ragged
batches of 16 and 32 users) and generic ones between them (grouped heads, head widths that are no power of two, odd row counts).
Values: queries and keys have unit variance per element (they come out of a norm), so that with scale dh^-1/2 the logits of a
row have a standard deviation near one; lengths are spread over a stated range; targets follow a long-tailed popularity.
"""

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp32": 4}
EPS, BASE = 1e-6, 10000.0


# ------------------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one new event for each of 32 users, before its attention: all launch latency
        dict(name="rotary one event", op="rotary", rows=32, hq=4, hk=2, dh=64, dtype="bf16", train=False),
        # a training batch of 65536 events of the d = 256, four-head model, forward and gradients
        dict(name="rotary train", op="rotary", rows=65536, hq=4, hk=4, dh=64, dtype="bf16", train=True),
        # reference-precision training of a small model with heads of an odd width
        dict(name="rotary train fp32 odd", op="rotary", rows=10007, hq=3, hk=1, dh=48, dtype="fp32", train=True),
        # serving: one new event for each of 32 users against its cached history (padded slots, ragged lengths)
        dict(name="attention one event", op="attention", B=32, Nq=1, Nk=4096, lo=1, hq=8, hk=2, dh=64, dtype="bf16", slots=True, train=False),
        # serving: four users with very long histories, all query heads on one key head
        dict(name="attention one event long", op="attention", B=4, Nq=1, Nk=131072, lo=65536, hq=8, hk=1, dh=128, dtype="bf16", slots=True, train=False),
        # encoding many short histories from scratch, d = 128 with four heads, packed
        dict(name="attention short histories", op="attention", B=64, Nq=256, Nk=256, lo=16, hq=4, hk=4, dh=32, dtype="bf16", slots=False, train=False),
        # a session's 64 new events at once against the cached history
        dict(name="attention extend", op="attention", B=8, Nq=64, Nk=8192, lo=1000, hq=4, hk=2, dh=64, dtype="bf16", slots=True, train=False),
        # training on ragged histories of up to 4096 items, d = 256 with four heads on two key heads
        dict(name="attention train", op="attention", B=16, Nq=4096, Nk=4096, lo=2048, hq=4, hk=2, dh=64, dtype="bf16", slots=False, train=True),
        # reference-precision training of a small model, odd widths and lengths
        dict(name="attention train fp32 odd", op="attention", B=5, Nq=501, Nk=501, lo=1, hq=6, hk=3, dh=40, dtype="fp32", slots=False, train=True),
        # a small batch against a small catalogue, some rows without a target: latency
        dict(name="loss small", op="loss", rows=200, items=5003, d=64, dtype="bf16", unlabelled=0.1, train=True),
        # next-item training of the d = 256 model over a catalogue of 131072 items
        dict(name="loss train", op="loss", rows=8192, items=131072, d=256, dtype="bf16", unlabelled=0.0, train=True),
        # reference-precision training, odd sizes, padded batch
        dict(name="loss train fp32 odd", op="loss", rows=1003, items=20011, d=96, dtype="fp32", unlabelled=0.3, train=True),
    ]


def _log(rng, lo, hi):
    """A size spread evenly over the logarithm of [lo, hi], odd as often as even."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    op = rng.choice(["rotary", "attention", "attention", "attention", "loss", "loss"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    if op == "rotary":
        hq, hk, dh = rng.choice([(4, 4, 32), (4, 2, 64), (8, 1, 128), (3, 1, 48), (6, 2, 80), (1, 1, 20)])
        return dict(op=op, rows=_log(rng, 1, 33554432 // ((hq + hk) * dh)), hq=hq, hk=hk, dh=dh, dtype=dtype, train=rng.random() < 0.5)
    if op == "loss":
        d = rng.choice([32, 64, 96, 128, 200, 256])
        items = _log(rng, 100, 131072 if dtype == "bf16" else 40000)
        rows = _log(rng, 1, min(65536, (1 << 30 if dtype == "bf16" else 1 << 26) // items))
        return dict(op=op, rows=rows, items=items, d=d, dtype=dtype, unlabelled=rng.choice([0.0, 0.1, 0.5]), train=rng.random() < 0.7)
    hq, hk = rng.choice([(1, 1), (4, 4), (4, 2), (8, 2), (8, 1), (6, 2), (5, 1)])
    dh = rng.choice([16, 32, 40, 64, 64, 80, 128])
    kind = rng.choice(["event", "extend", "histories", "train"])
    if kind == "event":
        Nk = _log(rng, 1, 131072)
        B = _log(rng, 1, min(256, 1 + 524288 // Nk))
        return dict(op=op, B=B, Nq=1, Nk=Nk, lo=_log(rng, 1, Nk), hq=hq, hk=hk, dh=dh, dtype=dtype, slots=True, train=False)
    if kind == "extend":
        Nk = _log(rng, 256, 16384)
        Nq = _log(rng, 2, min(256, Nk))
        return dict(op=op, B=_log(rng, 1, min(32, 65536 // Nk)), Nq=Nq, Nk=Nk, lo=_log(rng, Nq, Nk), hq=hq, hk=hk, dh=dh, dtype=dtype, slots=True,
                    train=False)
    most = 64000000 if dtype == "bf16" else 8000000  # pairs of a query and a key, without the heads
    N = _log(rng, 2, 4096 if dtype == "bf16" else 1500)
    B = _log(rng, 1, max(1, min(64, most // (N * N))))
    return dict(op=op, B=B, Nq=N, Nk=N, lo=_log(rng, 1, N), hq=hq, hk=hk, dh=dh, dtype=dtype, slots=rng.random() < 0.3, train=kind == "train")


# ------------------------------------------------------------------------------------------------------------ the inputs
def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    normal = lambda *shape, std=1.0, mean=0.0: (torch.randn(shape, generator=g, device=dev) * std + mean).to(dt)  # noqa: E731
    whole = lambda lo, hi, n: torch.randint(lo, hi + 1, (n,), generator=g, device=dev, dtype=torch.int32)  # noqa: E731
    s = dict(case)
    if case["op"] == "rotary":
        rows, hq, hk, dh = (case[k] for k in ("rows", "hq", "hk", "dh"))
        # the two head blocks are columns of one fused projection of the events
        qkv = normal(rows, hq + 2 * hk, dh, std=0.8)
        s.update(Q=qkv[:, :hq], K=qkv[:, hq:hq + hk], gq=normal(dh, std=0.2, mean=1.0), gk=normal(dh, std=0.2, mean=1.0),
                 positions=whole(0, 16383, rows))
        if case["train"]:
            s.update(dQ=normal(rows, hq, dh), dK=normal(rows, hk, dh))
        return s
    if case["op"] == "loss":
        rows, items, d = (case[k] for k in ("rows", "items", "d"))
        popular = torch.rand(rows, generator=g, device=dev, dtype=torch.float64).pow(3.0)
        targets = (popular * items).long().clamp_(max=items - 1).int()
        targets = torch.where(torch.rand(rows, generator=g, device=dev) < case["unlabelled"], torch.full_like(targets, -1), targets)
        weight = torch.rand(rows, generator=g, device=dev) + 0.5
        s.update(X=normal(rows, d), W=normal(items, d, std=1.5), targets=targets, dloss=weight / rows, scale=d ** -0.5)
        return s
    B, Nq, Nk, hq, hk, dh = (case[k] for k in ("B", "Nq", "Nk", "hq", "hk", "dh"))
    # evenly spread over [lo, Nk], the longest among them, in another order for each seed
    k_lens = Nk - (torch.arange(B, device=dev) * (Nk - case["lo"]) // max(1, B - 1)).int()
    k_lens = k_lens[torch.randperm(B, generator=g, device=dev)]
    q_lens = k_lens if Nq == Nk else torch.clamp(k_lens, max=Nq)
    count = lambda n: torch.arange(B + 1, device=dev, dtype=torch.int32) * n  # noqa: E731
    packed = lambda lens: torch.cat([lens.new_zeros(1), lens.cumsum(0, dtype=torch.int32)])  # noqa: E731
    s["scale"], s["q_lens"], s["k_lens"] = dh ** -0.5, None, None
    if case["slots"]:  # a slot of Nk rows for each user, the first of them in use
        s.update(q_offsets=count(Nq), k_offsets=count(Nk), k_lens=k_lens, q_lens=q_lens if Nq > 1 else None)
        q_rows, k_rows = B * Nq, B * Nk
    else:
        s.update(q_offsets=packed(q_lens), k_offsets=packed(k_lens))
        q_rows, k_rows = int(s["q_offsets"][-1]), int(s["k_offsets"][-1])
    s.update(Q=normal(q_rows, hq, dh), K=normal(k_rows, hk, dh), V=normal(k_rows, hk, dh))
    if case["train"]:
        s["dO"] = normal(q_rows, hq, dh)
    return s


# ------------------------------------------------------------------------------------------------------------ the calls
def run(s):
    if own:
        return _own(s)
    return {"rotary": _plain_rotary, "attention": _plain_attention, "loss": _plain_loss}[s["op"]](s)


def _own(s):
    from paper_2510_18239_amd import binding as b

    if s["op"] == "rotary":
        out = b.lime_norm_rotary(s["Q"], s["K"], s["gq"], s["gk"], s["positions"], BASE, EPS)
        if s["train"]:
            out = out + b.lime_norm_rotary_backward(s["dQ"], s["dK"], s["Q"], s["K"], s["gq"], s["gk"], s["positions"], BASE, EPS)
        return out
    if s["op"] == "loss":
        loss, lse = b.lime_catalogue_loss(s["X"], s["W"], s["targets"], s["scale"])
        if not s["train"]:
            return (loss,)
        return (loss,) + b.lime_catalogue_loss_backward(s["dloss"], s["X"], s["W"], s["targets"], lse, s["scale"])
    where = (s["q_offsets"], s["k_offsets"], s["Nq"], s["Nk"], s["scale"])
    O, lse = b.lime_sequence_attention(s["Q"], s["K"], s["V"], *where, q_lens=s["q_lens"], k_lens=s["k_lens"])
    if not s["train"]:
        return O, lse
    return (O, lse) + b.lime_sequence_attention_backward(s["dO"], s["Q"], s["K"], s["V"], O, lse, *where, q_lens=s["q_lens"], k_lens=s["k_lens"])


# ------------------------------------------------------------------------------------------------------------ the plain forms
def _angles(positions, dh):
    """cos and sin [rows, 1, dh / 2] of position * BASE^(-2 i / dh), the angles in fp64."""
    i = torch.arange(dh // 2, device=positions.device, dtype=torch.float64)
    angle = positions.double()[:, None] * torch.exp(i * (-2.0 / dh * math.log(BASE)))
    return torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]


def _plain_rotary(s):
    dt, dh = s["Q"].dtype, s["dh"]
    cos, sin = _angles(s["positions"], dh)
    out, gradients, weights = [], [], []
    for x, gamma, dy in ((s["Q"], s["gq"], s.get("dQ")), (s["K"], s["gk"], s.get("dK"))):
        x, gamma = x.float(), gamma.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        n = x * r
        a, b = (n * gamma).chunk(2, -1)
        out.append(torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(dt))
        if s["train"]:
            a, b = dy.float().chunk(2, -1)
            dz = torch.cat([a * cos + b * sin, b * cos - a * sin], -1)
            weights.append((dz * n).sum((0, 1)).to(dt))
            dn = dz * gamma
            gradients.append((r * (dn - n * (dn * n).mean(-1, keepdim=True))).to(dt))
    return tuple(out + gradients + weights)


def _of_rows(offsets, lens, rows):
    """For each of `rows` packed rows: its user, its place in the user's slot, and whether it is in use."""
    row = torch.arange(rows, device=offsets.device)
    user = torch.searchsorted(offsets[1:].contiguous(), row.int(), right=True)
    place = row - offsets[user]
    used = lens if lens is not None else offsets[1:] - offsets[:-1]
    return user, place, place < used[user]


def _padded(x, offsets, lens, n):
    """[B, n, heads, dh] fp32 of packed rows, zeros past a user's length."""
    at = torch.arange(n, device=x.device)[None]
    live = at < (lens if lens is not None else offsets[1:] - offsets[:-1])[:, None]
    return torch.where(live[..., None, None], x[(offsets[:-1, None] + at).clamp(max=x.shape[0] - 1)].float(), 0.0), live


def _plain_attention(s):
    dt, hq, hk, dh, Nq, Nk = s["Q"].dtype, s["hq"], s["hk"], s["dh"], s["Nq"], s["Nk"]
    g = hq // hk
    q, q_live = _padded(s["Q"], s["q_offsets"], s["q_lens"], Nq)
    k, k_live = _padded(s["K"], s["k_offsets"], s["k_lens"], Nk)
    v, _ = _padded(s["V"], s["k_offsets"], s["k_lens"], Nk)
    B = q.shape[0]
    q = q.view(B, Nq, hk, g, dh).permute(0, 2, 3, 1, 4).reshape(B, hk, g * Nq, dh)
    k, v = k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()  # [B, hk, Nk, dh]
    last = torch.arange(Nq, device=q.device)[None] + (k_live.sum(1) - q_live.sum(1))[:, None]  # the last key a query sees
    seen = (torch.arange(Nk, device=q.device)[None, None] <= last[..., None]) & k_live[:, None] & q_live[..., None]
    seen = seen[:, None, None].expand(B, hk, g, Nq, Nk).reshape(B, hk, g * Nq, Nk)
    logits = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"]).masked_fill_(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp_(logits.sub_(torch.where(top == -math.inf, 0.0, top)))
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[..., 0]  # -inf for a row that sees nothing
    p = p.div_(torch.where(total == 0, 1.0, total))
    o = torch.matmul(p, v)

    def rows(x, offsets, lens, n, like, heads):  # [B, hk, heads / hk * n, .] back to packed rows
        user, place, used = _of_rows(offsets, lens, like.shape[0])
        x = x.view(B, hk, heads // hk, n, -1).permute(0, 3, 1, 2, 4).reshape(B, n, heads, -1)
        return x[user, place.clamp(max=n - 1)], used[:, None, None]

    of_queries = (s["q_offsets"], s["q_lens"], Nq, s["Q"], hq)
    of_keys = (s["k_offsets"], s["k_lens"], Nk, s["K"], hk)
    O, used = rows(o, *of_queries)
    L, _ = rows(lse, *of_queries)
    out = (torch.where(used, O, 0.0).to(dt), torch.where(used, L, -math.inf)[..., 0])
    if not s["train"]:
        return out
    do, _ = _padded(s["dO"], s["q_offsets"], s["q_lens"], Nq)
    do = do.view(B, Nq, hk, g, dh).permute(0, 2, 3, 1, 4).reshape(B, hk, g * Nq, dh)
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    back = []
    for x, where in ((dq, of_queries), (dk, of_keys), (dv, of_keys)):
        x, used = rows(x, *where)
        back.append(torch.where(used, x, 0.0).to(dt))
    return out + tuple(back)


def _plain_loss(s):
    dt, x, w, t = s["X"].dtype, s["X"].float(), s["W"].float(), s["targets"].long()
    labelled = (t >= 0) & (t < w.shape[0])
    t = torch.where(labelled, t, 0)
    logits = torch.matmul(x, w.t()).mul_(s["scale"])
    top = logits.amax(1, keepdim=True)
    chosen = logits.gather(1, t[:, None])
    p = torch.exp_(logits.sub_(top))
    total = p.sum(1, keepdim=True)
    loss = torch.where(labelled, (top + torch.log(total) - chosen)[:, 0], 0.0)
    if not s["train"]:
        return (loss,)
    p.div_(total)
    p.scatter_add_(1, t[:, None], torch.full_like(chosen, -1.0))
    p.mul_((torch.where(labelled, s["dloss"], 0.0) * s["scale"])[:, None])
    return loss, torch.matmul(p, w).to(dt), torch.matmul(p.t(), x).to(dt)


# ------------------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "attention": _exact_attention, "loss": _exact_loss}[case["op"]](s)


def _exact_rotary(s):
    """Pairs (i, i + dh / 2) of a normalised head as complex numbers, turned by e^(i angle)."""
    half = s["dh"] // 2
    frequency = torch.tensor([BASE ** (-2.0 * i / s["dh"]) for i in range(half)], dtype=torch.float64, device=s["Q"].device)
    turn = torch.exp(1j * (s["positions"].double().unsqueeze(1) * frequency)).unsqueeze(1)
    out, dx, dgamma = [], [], []
    for name, gamma in (("Q", s["gq"].double()), ("K", s["gk"].double())):
        x = s[name].double()
        norm = ((x ** 2).sum(-1, keepdim=True) / s["dh"] + EPS).sqrt()
        unit = x / norm
        z = unit * gamma
        y = torch.complex(z[..., :half], z[..., half:]) * turn
        out.append(torch.cat((y.real, y.imag), -1))
        if s["train"]:
            dy = s["d" + name].double()
            back = torch.complex(dy[..., :half], dy[..., half:]) * turn.conj()
            back = torch.cat((back.real, back.imag), -1)
            dgamma.append((back * unit).flatten(0, 1).sum(0))
            du = back * gamma
            dx.append(du / norm - x * ((du * x).sum(-1, keepdim=True) / (s["dh"] * norm ** 3)))
    return tuple(out + dx + dgamma)


def _exact_attention(s):
    q_at, k_at = s["q_offsets"].tolist(), s["k_offsets"].tolist()
    q_n = s["q_lens"].tolist() if s["q_lens"] is not None else [b - a for a, b in zip(q_at, q_at[1:])]
    k_n = s["k_lens"].tolist() if s["k_lens"] is not None else [b - a for a, b in zip(k_at, k_at[1:])]
    Q, K, V = s["Q"].double(), s["K"].double(), s["V"].double()
    O, L = torch.zeros_like(Q), Q.new_full(Q.shape[:2], -math.inf)
    dO = s["dO"].double() if s["train"] else None
    dQ, dK, dV = torch.zeros_like(Q), torch.zeros_like(K), torch.zeros_like(V)
    group = s["hq"] // s["hk"]
    for u in range(s["B"]):
        nq, nk = q_n[u], k_n[u]
        if nq == 0 or nk == 0:
            continue
        rq, rk = slice(q_at[u], q_at[u] + nq), slice(k_at[u], k_at[u] + nk)
        hidden = torch.ones(nq, nk, dtype=torch.bool, device=Q.device).triu(nk - nq + 1)
        for h in range(s["hq"]):
            q, k, v = Q[rq, h], K[rk, h // group], V[rk, h // group]
            z = (s["scale"] * (q @ k.T)).masked_fill(hidden, -math.inf)
            L[rq, h] = torch.logsumexp(z, 1)
            a = torch.where(hidden, 0.0, torch.exp(z - L[rq, h, None]))
            O[rq, h] = a @ v
            if s["train"]:
                go = dO[rq, h]
                e = a * (go @ v.T - (go * O[rq, h]).sum(1, keepdim=True)) * s["scale"]
                dQ[rq, h] = e @ k
                dK[rk, h // group] += e.T @ q
                dV[rk, h // group] += a.T @ go
    return (O, L, dQ, dK, dV) if s["train"] else (O, L)


def _exact_loss(s):
    X, W, t = s["X"].double(), s["W"].double(), s["targets"]
    loss = torch.zeros(X.shape[0], dtype=torch.float64, device=X.device)
    dX, dW = torch.zeros_like(X), torch.zeros_like(W)
    live = torch.nonzero((t >= 0) & (t < W.shape[0])).flatten()
    for rows in live.split(1024):
        x, label, each = X[rows], t[rows].long(), torch.arange(len(rows), device=X.device)
        z = s["scale"] * (x @ W.T)
        lse = torch.logsumexp(z, 1)
        loss[rows] = lse - z[each, label]
        if s["train"]:
            e = torch.exp(z - lse[:, None])
            e[each, label] -= 1.0
            e *= (s["dloss"].double()[rows] * s["scale"])[:, None]
            dX[rows] = e @ W
            dW += e.T @ x
    return (loss, dX, dW) if s["train"] else (loss,)


# ------------------------------------------------------------------------------------------------------------ the work
def work(case):
    """Inputs read once, outputs written once, and the products of the visible pairs (for the mean of the lengths)."""
    e = BYTES[case["dtype"]]
    if case["op"] == "rotary":
        heads = case["rows"] * (case["hq"] + case["hk"]) * case["dh"]
        passes = 5 if case["train"] else 2  # x in, y out; dy in, x in again for a call of its own, dx out
        return {"bytes": heads * e * passes + 4 * case["rows"] + 4 * case["dh"] * e, "flops": heads * (22 if case["train"] else 8)}
    if case["op"] == "loss":
        rows, items, d = case["rows"] * (1 - case["unlabelled"]), case["items"], case["d"]
        sides = (rows + items) * d * e
        return {"bytes": sides * (2 if case["train"] else 1) + 16 * case["rows"], "flops": 2 * rows * items * d * (3 if case["train"] else 1)}
    B, Nq, Nk, lo, hq, hk, dh = (case[k] for k in ("B", "Nq", "Nk", "lo", "hq", "hk", "dh"))
    mean = (lo + Nk) / 2
    if Nq == Nk:
        n, pairs = mean, ((lo * lo + lo * Nk + Nk * Nk) / 3 + mean) / 2
    else:
        n = min(Nq, mean)
        pairs = n * max(mean - (n - 1) / 2, 1)
    passes = 2 if case["train"] else 1
    q_bytes, k_bytes = B * n * hq * (2 * dh * e + 4), B * mean * hk * 2 * dh * e
    return {"bytes": passes * (q_bytes + k_bytes), "flops": B * hq * pairs * dh * 2 * (2 + (5 if case["train"] else 0))}
