"""The history encoder's operators against their formulas in 64 bits, at the sizes, layouts and contents where they can go wrong.

Tolerances: the oracle's bounds, element by element.  A rounding to the storage type is off by at most half a step (u = 2^-8 for
bf16, 2^-24 for fp32) of the value; fp32 sums and the hardware's exp2 and log2 (one unit in the last place each) by a number of
2^-24 steps of the sum of magnitudes that the bounds count."""

import numpy as np
import pytest
import torch

from oracle import encoder_oracle as enc
from paper_2510_18239_amd import binding

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
U = {"bf16": 2.0**-8, "fp32": 2.0**-24}
F = 2.0**-24


def make(shape, dtype, seed, std=1.0, mean=0.0):
    """Values of the storage type: (device tensor, fp64 array)."""
    x = torch.from_numpy(np.random.default_rng(seed).standard_normal(shape) * std + mean).to(DT[dtype])
    return x.cuda(), x.double().numpy()


def within(got, want, tolerance, what):
    got = got.detach().double().cpu().numpy()
    assert got.shape == want.shape, what
    assert np.isfinite(got).all(), f"{what}: not finite"
    off = np.abs(got - want) - tolerance - 1e-37
    worst = np.unravel_index(off.argmax(), off.shape) if off.size else None
    assert off.size == 0 or off.max() <= 0, f"{what}: {got[worst]} for {want[worst]} at {worst}, allowed {tolerance[worst]}"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def strided(x, before, after):
    """The same [rows, heads, dh] tensor as columns of a wider one whose other columns are NaN."""
    rows, heads, dh = x.shape
    wide = torch.full((rows, before + heads * dh + after), float("nan"), dtype=x.dtype, device=x.device)
    view = wide[:, before:before + heads * dh].unflatten(1, (heads, dh))
    view.copy_(x)
    return wide, view


# ------------------------------------------------------------------------------------------------- norms and rotation
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,hq,hk,dh,before,turned", [
    (1, 1, 1, 2, 0, True), (1, 4, 2, 64, 0, True), (7, 3, 1, 48, 8, True), (33, 8, 1, 128, 16, True), (9, 2, 2, 20, 0, True), (9, 2, 2, 20, 3, True),
    (5, 1, 0, 256, 0, True), (17, 5, 3, 254, 1, True), (12, 6, 2, 80, 0, False), (2049, 4, 4, 32, 0, True), (8195, 2, 1, 16, 0, True), (16395, 3, 1, 24, 0, True), (16385, 1, 1, 48, 8, True),
])
def test_norm_rotary(dtype, rows, hq, hk, dh, before, turned):
    u, eps, base = U[dtype], 1e-6, 10000.0
    (q, Q), (k, K) = make((rows, hq, dh), dtype, 1, 0.7), make((rows, max(hk, 1), dh), dtype, 2, 3.0)
    (gq, Gq), (gk, Gk) = make((dh,), dtype, 3, 0.3, 1.0), make((dh,), dtype, 4, 0.3, 1.0)
    (dyq, DYq), (dyk, DYk) = make((rows, hq, dh), dtype, 5), make((rows, max(hk, 1), dh), dtype, 6)
    pos = np.random.default_rng(7).integers(-(2**31), 2**31, rows) if rows > 4 else np.arange(rows) * 1000003
    positions = ints(pos) if turned else None
    pos = pos if turned else None
    if before:
        q, k, dyq, dyk = (strided(x, before, 5)[1] for x in (q, k, dyq, dyk))
    qo, ko = binding.lime_norm_rotary(q, k if hk else None, gq, gk if hk else None, positions, base, eps)
    grads = binding.lime_norm_rotary_backward(dyq, dyk if hk else None, q, k if hk else None, gq, gk if hk else None, positions, base, eps)
    for x, X, g, G, y, DY, dx, dg in ((q, Q, gq, Gq, qo, DYq, grads[0], grads[2]), (k, K, gk, Gk, ko, DYk, grads[1], grads[3]))[: 2 if hk else 1]:
        want, size = enc.norm_rotary(X, G, pos, base, eps)
        within(y, want, u * abs(want) + F * (dh + 24) * size, "y")  # norm: dh terms; angle, sine, products: 24 steps
        (wx, wg), (sx, sg) = enc.norm_rotary_backward(DY, X, G, pos, base, eps)
        within(dx, wx, u * abs(wx) + F * (3 * dh + 40) * sx, "dx")
        within(dg, wg, u * abs(wg) + F * (dh + 40 + rows * X.shape[1]) * sg, "dgamma")
    assert hk or (ko is None and grads[1] is None and grads[3] is None)


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 20), ("fp32", 40)])
def test_norm_rotary_in_place_and_without_gamma(dtype, dh):
    (q, _), (k, _), (dy, _) = make((37, 4, dh), dtype, 1), make((37, 2, dh), dtype, 2), make((37, 4, dh), dtype, 3)
    pos = ints(np.arange(37) * 5)
    want = binding.lime_norm_rotary(q, k, None, None, pos)
    back = binding.lime_norm_rotary_backward(dy, k, q, k, None, None, pos)
    assert back[2] is None and back[3] is None
    wide, view = strided(q, 16, 7)
    got = binding.lime_norm_rotary(view, k, None, None, pos, QO=view, KO=k)
    assert got[0].data_ptr() == view.data_ptr()
    # (rows that are not whole 16-byte pieces have their squares summed in another order: fp32 sums of dh terms, each then rounded)
    bar = 2 * (U[dtype] + F * (dh + 24)) * 8.0  # no y is larger than sqrt(dh) < 8
    for a, b in zip((view, k), want):
        assert float((a.float() - b.float()).abs().max()) <= bar
    assert wide[:, :16].isnan().all() and wide[:, 16 + 4 * dh:].isnan().all()  # the columns beside the heads
    (k, _) = make((37, 2, dh), dtype, 2)
    grad = dy.clone()
    binding.lime_norm_rotary_backward(grad, k, q, k, None, None, pos, dQ=grad)
    assert torch.equal(grad, back[0])


def test_norm_rotary_of_rows_that_are_not_finite_or_zero():
    (q, _) = make((6, 2, 64), "bf16", 1)
    want, _ = binding.lime_norm_rotary(q, None, positions=ints(range(6)))
    bad = q.clone()
    bad[2, 1], bad[4, 0] = float("nan"), float("inf")
    got, _ = binding.lime_norm_rotary(bad, None, positions=ints(range(6)))
    other = torch.ones(6, 2, dtype=torch.bool, device="cuda")
    other[2, 1] = other[4, 0] = False
    assert torch.equal(got[other], want[other]) and got[2, 1].isnan().all()
    zero, _ = binding.lime_norm_rotary(torch.zeros_like(q), None, positions=ints(range(6)))
    assert (zero == 0).all()


# ------------------------------------------------------------------------------------------------- attention
def packed(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(int)


def attention_case(dtype, q_lens, k_lens, hq, hk, dh, causal=True, slots=None, scale=None, std=1.0, before=0, gradients=True, seed=0):
    """One call of each direction against the oracle; slots: (rows of a query slot, of a key slot), the rest of a slot NaN."""
    u, scale = U[dtype], dh**-0.5 if scale is None else scale
    B = len(q_lens)
    qo, ko = (packed(q_lens), packed(k_lens)) if slots is None else (np.arange(B + 1) * slots[0], np.arange(B + 1) * slots[1])
    extra = 3  # rows behind the last slot
    (q, Q), (k, K), (v, V), (g, G) = (make((n + extra, h, dh), dtype, seed + i, s) for i, (n, h, s) in
                                      enumerate(((qo[-1], hq, std), (ko[-1], hk, std), (ko[-1], hk, 1.0), (qo[-1], hq, 1.0))))
    qs, ks = enc.spans(qo, q_lens, None), enc.spans(ko, k_lens, None)
    q_used, k_used = np.zeros(len(Q), bool), np.zeros(len(K), bool)
    q_slot, k_slot = np.arange(len(Q)) < qo[-1], np.arange(len(K)) < ko[-1]
    for spans, used in ((qs, q_used), (ks, k_used)):
        for a, _, n in spans:
            used[a:a + n] = True
    for x, used in ((q, q_used), (g, q_used), (k, k_used), (v, k_used)):  # what is not in use may hold anything
        x[torch.from_numpy(~used).cuda()] = float("nan")
    max_q, max_k = (max(q_lens), max(k_lens)) if slots is None else slots
    kw = {} if slots is None else dict(q_lens=ints(q_lens), k_lens=ints(k_lens))
    if before:
        q, k, v = (strided(x, before, 1)[1] for x in (q, k, v))
    O = torch.full((len(Q), hq, dh), 7.0, dtype=DT[dtype], device="cuda")
    lse = torch.full((len(Q), hq), 7.0, device="cuda")
    where = (ints(qo), ints(ko), int(max_q), int(max_k), scale)
    binding.lime_sequence_attention(q, k, v, *where, causal=causal, O=O, lse=lse, **kw)
    wO, wl, inside = enc.sequence_attention(Q, K, V, qs, ks, scale, causal)
    tO, tl, tQ, tK, tV = enc.sequence_attention_bounds(Q, K, V, G if gradients else None, wO, inside, scale, u, causal)
    out = ~q_slot
    assert (O[torch.from_numpy(out).cuda()] == 7).all() and (lse[torch.from_numpy(out).cuda()] == 7).all(), "rows outside all slots"
    at = torch.from_numpy(q_slot).cuda()
    within(O[at], wO[q_slot], tO[q_slot], "O")
    seen = np.isfinite(wl[q_slot])
    got = lse[at].cpu().numpy()
    assert np.array_equal(np.isneginf(got), ~seen)
    assert (abs(got[seen] - wl[q_slot][seen]) <= tl[q_slot][seen]).all(), "lse"
    if not gradients:
        return
    dq = torch.full((len(Q), hq * dh + 8), 7.0, dtype=DT[dtype], device="cuda")
    dkv = torch.full((len(K), 2, hk, dh), 7.0, dtype=DT[dtype], device="cuda")  # keys' and values' gradients side by side
    dQ, dK, dV = binding.lime_sequence_attention_backward(g, q, k, v, O, lse, *where, causal=causal, dQ=dq[:, :hq * dh].unflatten(1, (hq, dh)), dK=dkv[:, 0],
                                                          dV=dkv[:, 1], **kw)
    wQ, wK, wV = enc.sequence_attention_backward(G, Q, K, V, wO, inside, scale)
    kt = torch.from_numpy(k_slot).cuda()
    assert (dq[:, hq * dh:] == 7).all() and (dQ[~at] == 7).all() and (dK[~kt] == 7).all() and (dV[~kt] == 7).all()
    within(dQ[at], wQ[q_slot], u * abs(wQ[q_slot]) + tQ[q_slot], "dQ")
    within(dK[kt], wK[k_slot], u * abs(wK[k_slot]) + tK[k_slot], "dK")
    within(dV[kt], wV[k_slot], u * abs(wV[k_slot]) + tV[k_slot], "dV")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,hq,hk,dh", [
    ([1], 1, 1, 32), ([1, 0, 2, 1], 2, 1, 64), ([31, 32, 33], 1, 1, 32), ([63, 64, 65, 0], 4, 2, 64), ([127, 128, 129], 2, 2, 64), ([200, 3, 77], 6, 2, 128),
    ([130], 5, 1, 16), ([70, 257], 3, 3, 80), ([40, 90], 7, 7, 40), ([513], 8, 1, 32), ([19, 45], 2, 1, 1), ([66, 5], 2, 1, 30), ([300], 1, 1, 100),
])
def test_histories(dtype, lens, hq, hk, dh):
    attention_case(dtype, lens, lens, hq, hk, dh)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("q_lens,k_lens,slots,hq,hk,dh,causal", [
    ([1, 1, 1], [5, 0, 64], (1, 64), 4, 2, 64, True),            # one new event; a user without a history
    ([1, 0, 1], [300, 9, 1], (1, 301), 8, 1, 128, True),
    ([3, 2, 0, 4], [700, 2, 5, 64], (4, 700), 4, 4, 32, True),   # a few new events
    ([40, 64, 1], [100, 64, 1], (64, 130), 4, 2, 64, True),
    ([50, 9], [20, 0], (60, 30), 2, 1, 64, True),                # more queries than keys: the first see nothing
    ([50, 9, 33], [20, 0, 200], (60, 210), 2, 1, 48, False),     # every key for every query
    ([128, 127], [400, 129], (130, 401), 1, 1, 32, False),
    ([1, 1, 0, 1, 1, 1, 1, 1], [900, 3, 700, 0, 256, 257, 64, 800], (1, 900), 4, 2, 64, True),  # chunks of sixteen pairs, which change places
    ([1, 1, 1, 1], [3000, 40, 1, 2222], (1, 3000), 16, 2, 100, True),
])
def test_slots_and_lengths(dtype, q_lens, k_lens, slots, hq, hk, dh, causal):
    attention_case(dtype, q_lens, k_lens, hq, hk, dh, causal, slots)


def test_many_heads_on_one_key_head():
    attention_case("bf16", [1], [21000], 200, 1, 32)  # both sides of the backward pass are cut into chunks


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("before", [1, 8, 64])
@pytest.mark.parametrize("dh", [64, 33])
def test_strided_rows(dtype, before, dh):
    attention_case(dtype, [65, 0, 30], [65, 0, 30], 4, 2, dh, before=before)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0, 1e-3])
def test_scales(dtype, scale):
    attention_case(dtype, [150, 20], [150, 20], 2, 1, 64, scale=scale)
    attention_case(dtype, [1, 1], [900, 3], 2, 1, 64, scale=scale, slots=(1, 900), gradients=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_logits_that_keep_growing(dtype):
    """The running maximum is raised at every step, and starts far below zero."""
    dh, n = 32, 400
    q = torch.ones(1, 1, dh, dtype=DT[dtype], device="cuda")
    k = (torch.arange(n, device="cuda").float()[:, None, None] * 0.25 - 60.0).expand(n, 1, dh).to(DT[dtype]).contiguous()
    v, V = make((n, 1, dh), dtype, 3)
    K = k.double().cpu().numpy()
    for order in (1, -1):
        kk = k.flip(0).contiguous() if order < 0 else k
        KK = K[::order]
        O, lse = binding.lime_sequence_attention(q, kk, v, ints([0, 1]), ints([0, n]), 1, n, 1.0)
        wO, wl, inside = enc.sequence_attention(np.ones((1, 1, dh)), KK, V, [(0, 1, 1)], [(0, n, n)], 1.0, True)
        tO, tl, *_ = enc.sequence_attention_bounds(np.ones((1, 1, dh)), KK, V, None, wO, inside, 1.0, U[dtype], True)
        within(O, wO, tO, "O")
        within(lse, wl, tl, "lse")


def test_entries_that_are_not_finite_stay_with_their_user():
    lens = [70, 90, 50]
    at = packed(lens)
    (q, _), (k, _), (v, _), (g, _) = (make((at[-1], h, 64), "bf16", i) for i, h in enumerate((4, 2, 2, 4)))
    where = (ints(at), ints(at), 90, 90, 0.125)

    def both(q, k, v, g):
        O, lse = binding.lime_sequence_attention(q, k, v, *where)
        return (O, lse) + binding.lime_sequence_attention_backward(g, q, k, v, O, lse, *where)

    want = both(q, k, v, g)
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(torch.bfloat16).min):
        for which in range(4):
            x = [q.clone(), k.clone(), v.clone(), g.clone()]
            x[which][at[1] + 30] = bad
            for a, b in zip(both(*x), want):
                assert torch.equal(a[:at[1]], b[:at[1]]) and torch.equal(a[at[2]:], b[at[2]:])


def test_offsets_and_lengths_are_cut_to_the_tensors():
    (q, _), (k, _), (v, _) = (make((40, 2, 32), "bf16", i) for i in range(3))
    a = binding.lime_sequence_attention(q, k, v, ints([0, 40]), ints([0, 40]), 40, 40, 0.2)
    b = binding.lime_sequence_attention(q, k, v, ints([-5, 4000]), ints([-7, 2**31 - 1]), 4000, 10**6, 0.2, q_lens=ints([10**6]), k_lens=ints([2**31 - 1]))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    O, lse = binding.lime_sequence_attention(q, k, v, ints([0, 40]), ints([30, 10]), 40, 40, 0.2, k_lens=ints([-3]))  # descending offsets: no keys
    assert (O == 0).all() and lse.isneginf().all()
    # a longest slot that is too short cuts the slot
    O = torch.full_like(q, 7.0)
    binding.lime_sequence_attention(q, k, v, ints([0, 40]), ints([0, 40]), 16, 40, 0.2, O=O, causal=False)
    assert (O[16:] == 7).all() and not (O[:16] == 7).all()


def test_no_rows():
    (q, _), (k, _) = make((5, 2, 32), "bf16", 0), make((0, 2, 32), "bf16", 1)
    O, lse = binding.lime_sequence_attention(q, k, k, ints([0, 5]), ints([0, 0]), 5, 0, 1.0)
    assert (O == 0).all() and lse.isneginf().all()
    dq, dk, dv = binding.lime_sequence_attention_backward(q, q, k, k, O, lse, ints([0, 5]), ints([0, 0]), 5, 0, 1.0)
    assert (dq == 0).all() and dk.shape == dv.shape == (0, 2, 32)
    O, lse = binding.lime_sequence_attention(k, q, q, ints([0, 0]), ints([0, 5]), 0, 5, 1.0)
    assert O.shape == (0, 2, 32) and lse.shape == (0, 2)
    dq, dk, dv = binding.lime_sequence_attention_backward(k, k, q, q, O, lse, ints([0, 0]), ints([0, 5]), 0, 5, 1.0)
    assert dq.shape == (0, 2, 32) and (dk == 0).all() and (dv == 0).all()


def test_a_cache_whose_offsets_pass_32_bits():
    """One new event of the last user of a cache of 4.4 GB a tensor."""
    hk, dh, slot, users = 8, 128, 68000, 32
    rows = slot * users
    assert rows * hk * dh > 2**31 and rows * hk * dh * 2 > 2**32
    K, V = (torch.empty(rows, hk, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    n = 500
    (q, Q), (k, Kn), (v, Vn) = make((users, hk, dh), "bf16", 0), make((n, hk, dh), "bf16", 1), make((n, hk, dh), "bf16", 2)
    K[rows - slot:rows - slot + n], V[rows - slot:rows - slot + n] = k, v
    lens = [0] * (users - 1) + [n]
    O, _ = binding.lime_sequence_attention(q, K, V, ints(range(users + 1)), ints(np.arange(users + 1) * slot), 1, slot, dh**-0.5, k_lens=ints(lens))
    wO, _, inside = enc.sequence_attention(Q[-1:], Kn, Vn, [(0, 1, 1)], [(0, n, n)], dh**-0.5, True)
    tO = enc.sequence_attention_bounds(Q[-1:], Kn, Vn, None, wO, inside, dh**-0.5, U["bf16"], True)[0]
    within(O[-1:], wO, tO, "O")
    assert (O[:-1] == 0).all()


# ------------------------------------------------------------------------------------------------- the loss
def loss_case(dtype, rows, items, d, unlabelled, scale=None, std=1.0, shift=0.0, seed=0, below=None):
    u, scale = U[dtype], d**-0.5 if scale is None else scale
    (x, X), (w, W) = make((rows, d), dtype, seed, std, shift), make((items, d), dtype, seed + 1, 1.0, -shift)
    r = np.random.default_rng(seed + 2)
    t = r.integers(0, below or items, rows)
    none = r.random(rows) < unlabelled
    t[none] = r.choice([-1, -100, items, 2**31 - 1, -(2**31)], none.sum())
    x[torch.from_numpy(none).cuda()] = float("nan")  # a row without a target may hold anything
    dl = r.standard_normal(rows).astype(np.float32)
    g = torch.from_numpy(np.where(none, np.nan, dl).astype(np.float32)).cuda()
    loss, lse = binding.lime_catalogue_loss(x, w, ints(t), scale)
    wl, wlse, e = enc.catalogue_loss(X, W, t, scale)
    L = abs(scale) * (abs(X) @ abs(W).T).max(1)
    e32 = F * ((d + 8) * L + items + 16)  # of a row's p, and of its lse
    off = e32 + F * 8 * (1 + L + np.log(items))
    within(lse, wlse, np.where(none, 0, off), "lse")
    within(loss, wl, np.where(none, 0, 2 * off), "loss")
    dX, dW = binding.lime_catalogue_loss_backward(g, x, w, ints(t), lse, scale)
    wX, wW = enc.catalogue_loss_backward(dl, X, W, t, scale)
    weight = np.where(none, 0, abs(dl) * abs(scale))[:, None]
    p = e.copy()
    p[~none, t[~none]] += 1.0
    each = weight * p * (u + 4 * off[:, None] + F * max(rows, items)) + F * 8 * weight * abs(e - p)  # of e; the target's own term is exact to fp32
    within(dX, wX, u * abs(wX) + (each + F * 8 * weight * (p + abs(e - p))) @ abs(W), "dX")
    rest = np.zeros_like(p)  # a target's e as an operand: rounded, and the rest rounded
    rest[~none, t[~none]] = u * u
    within(dW, wW, u * abs(wW) + (each + weight * (rest + F * rows * (p + abs(e - p)))).T @ abs(X), "dW")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,items,d,unlabelled", [
    (1, 1, 1, 0.0), (1, 5000, 64, 0.0), (2, 3, 32, 0.5), (127, 129, 64, 0.0), (128, 64, 128, 0.3), (300, 1000, 256, 0.1), (65, 2050, 96, 0.9), (70, 33, 200, 0.0),
    (40, 40, 33, 0.2), (16, 700, 250, 1.0), (1100, 500, 48, 0.5), (20000, 40, 16, 0.4),
])
def test_loss(dtype, rows, items, d, unlabelled):
    loss_case(dtype, rows, items, d, unlabelled)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale,std,shift", [(0.0, 1.0, 0.0), (-0.2, 1.0, 0.0), (1.0, 2.0, 0.0), (1.0, 1.0, 2.0)])
def test_loss_scales(dtype, scale, std, shift):
    """Equal logits; negative scales; sharp softmaxes; logits all near -250, whose exponentials alone would not be numbers."""
    loss_case(dtype, 90, 777, 64, 0.1, scale, std, shift)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,items,d,below", [(500, 1000, 64, 1), (700, 2000, 256, 8), (6000, 300, 32, 2)])
def test_loss_of_popular_items(dtype, rows, items, d, below):
    loss_case(dtype, rows, items, d, 0.1, below=below)


@pytest.mark.parametrize("rows", [1, 300, 5003])
def test_targets_that_are_not_aligned(rows):
    (x, _), (w, _) = make((rows, 64), "bf16", 0), make((400, 64), "bf16", 1)
    t = ints(np.random.default_rng(2).integers(-50, 400, rows + 1))
    g = torch.ones(rows, device="cuda")
    at = [t[1:], t[1:].clone()]
    assert at[0].data_ptr() % 16 == 4 and at[1].data_ptr() % 16 == 0
    loss = [binding.lime_catalogue_loss(x, w, t) for t in at]
    assert same(*loss)
    assert same(*(binding.lime_catalogue_loss_backward(g, x, w, t, loss[0][1]) for t in at))


@pytest.mark.parametrize("rows,items,d", [(130, 700, 64), (600, 260, 256)])
def test_one_gradient_of_the_loss(rows, items, d):
    (x, _), (w, _) = make((rows, d), "bf16", 0), make((items, d), "bf16", 1)
    t = ints(np.random.default_rng(2).integers(-9, items, rows))
    g = torch.ones(rows, device="cuda")
    _, lse = binding.lime_catalogue_loss(x, w, t)
    want = binding.lime_catalogue_loss_backward(g, x, w, t, lse)
    lib = binding.lib()
    need = lib.lime_catalogue_loss_workspace_bytes(rows, items, d, 1, 1)
    room = torch.empty(need, dtype=torch.uint8, device="cuda")
    for which in (0, 1):
        got = torch.full_like(want[which], 7.0)
        out = [None, None]
        out[which] = got.data_ptr()
        status = lib.lime_catalogue_loss_backward(g.data_ptr(), x.data_ptr(), w.data_ptr(), t.data_ptr(), lse.data_ptr(), *out, rows, items, d, 1.0, 1,
                                                  room.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
        assert status == 0, binding.last_error()
        assert torch.equal(got, want[which])


def test_rows_of_the_loss_that_are_not_finite_stay_alone():
    (x, _), (w, _) = make((50, 64), "bf16", 0), make((300, 64), "bf16", 1)
    t, g = ints(np.arange(50)), torch.ones(50, device="cuda")

    def both(x):
        loss, lse = binding.lime_catalogue_loss(x, w, t, 0.1)
        return loss, lse, binding.lime_catalogue_loss_backward(g, x, w, t, lse, 0.1)[0]

    want = both(x)
    bad = x.clone()
    bad[7], bad[33, 5] = float("nan"), float("inf")
    keep = torch.ones(50, dtype=torch.bool, device="cuda")
    keep[7] = keep[33] = False
    for a, b in zip(both(bad), want):
        assert torch.equal(a[keep], b[keep])
    assert both(bad)[0][7].isnan()


# ------------------------------------------------------------------------------------------------- how they are called
def calls():
    """Each operator, both directions, as a function of nothing on fixed inputs."""
    lens = [100, 37, 0, 5]
    at = packed(lens)
    (q, _), (k, _), (v, _), (g, _) = (make((at[-1], h, 64), "bf16", i) for i, h in enumerate((4, 2, 2, 4)))
    (one, _), (x, _), (w, _) = make((3, 4, 64), "bf16", 5), make((150, 64), "bf16", 6), make((900, 64), "bf16", 7)
    pos, off, t = ints(np.arange(at[-1])), ints(at), ints(np.arange(150) * 7 % 1000)
    dl = torch.rand(150, device="cuda")
    K = torch.randn(3 * 1500, 2, 64, device="cuda").bfloat16()
    cache = (ints([0, 1, 2, 3]), ints([0, 1500, 3000, 4500]), 1, 1500, 0.125)
    lens3 = ints([1500, 2, 700])

    def run(**kw):
        qn, kn = binding.lime_norm_rotary(q, k, None, None, pos, **kw)
        O, lse = binding.lime_sequence_attention(qn, kn, v, off, off, 100, 100, 0.125, **kw)
        d = binding.lime_sequence_attention_backward(g, qn, kn, v, O, lse, off, off, 100, 100, 0.125, **kw)
        dq = binding.lime_norm_rotary_backward(d[0], d[1], q, k, None, None, pos, **kw)
        served = binding.lime_sequence_attention(one, K, K, *cache, k_lens=lens3, **kw)
        loss, lse2 = binding.lime_catalogue_loss(x, w, t, 0.1, **kw)
        return (qn, kn, O, lse, *d, *dq[:2], *served, loss, lse2, *binding.lime_catalogue_loss_backward(dl, x, w, t, lse2, 0.1, **kw))

    return run


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_the_same_call_gives_the_same_bits():
    run = calls()
    first = run()
    assert all(same(run(), first) for _ in range(3))


def test_on_another_stream():
    run = calls()
    want = run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    given = run(stream=s)
    with torch.cuda.stream(s):
        current = run()
    torch.cuda.synchronize()
    assert same(given, want) and same(current, want)


def test_captured_and_replayed_between_eager_calls():
    run = calls()
    want = run()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):  # two graphs, replayed on two streams at once
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graphs.append((graph, out, torch.cuda.Stream()))
    for turn in range(4):
        for graph, out, s in graphs:
            for x in out:
                x.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph, _, s in graphs:
            with torch.cuda.stream(s):
                graph.replay()
        eager = run()
        torch.cuda.synchronize()
        assert same(eager, want), turn
        for _, out, _ in graphs:
            assert same(out, want), turn


def test_workspaces():
    (q, _), (k, _), (x, _), (w, _) = make((4, 8, 64), "bf16", 0), make((4 * 2000, 1, 64), "bf16", 1), make((64, 64), "bf16", 2), make((500, 64), "bf16", 3)
    where = (ints(range(5)), ints(np.arange(5) * 2000), 1, 2000, 0.125)
    want = binding.lime_sequence_attention(q, k, k, *where)
    need = 32 << 20
    room = torch.full((need,), 255, dtype=torch.uint8, device="cuda")  # what a workspace holds before does not matter
    assert same(binding.lime_sequence_attention(q, k, k, *where, workspace=room), want)
    t = ints(np.arange(64) - 5)
    loss = binding.lime_catalogue_loss(x, w, t)
    grads = binding.lime_catalogue_loss_backward(loss[0], x, w, t, loss[1])
    room.fill_(255)
    assert same(binding.lime_catalogue_loss(x, w, t, workspace=room), loss)
    room.fill_(255)
    assert same(binding.lime_catalogue_loss_backward(loss[0], x, w, t, loss[1], workspace=room), grads)
    with pytest.raises(binding.LimeError, match="workspace"):
        binding.lime_sequence_attention(q, k, k, *where, workspace=room[:256])
    with pytest.raises(binding.LimeError, match="aligned"):
        binding.lime_sequence_attention(q, k, k, *where, workspace=room[16:])
    with pytest.raises(ValueError, match="uint8"):
        binding.lime_sequence_attention(q, k, k, *where, workspace=room.view(torch.float32))


def test_refusals_of_tensors():
    (q, _), (k, _) = make((10, 4, 64), "bf16", 0), make((10, 2, 64), "bf16", 1)
    off = ints([0, 10])
    call = lambda q=q, k=k, v=k, qo=off, ko=off, **kw: binding.lime_sequence_attention(q, k, v, qo, ko, 10, 10, 1.0, **kw)  # noqa: E731
    for bad in (dict(q=q.float()), dict(k=k[:, :, :32]), dict(v=k[:5]), dict(q=q.transpose(1, 2)), dict(q=q.transpose(0, 1)), dict(qo=off.long()), dict(qo=off[:1]),
                dict(ko=ints([0, 5, 10])), dict(q_lens=ints([1, 2])), dict(k_lens=ints([1]).cpu()), dict(O=q[:5]), dict(O=q.float()),
                dict(lse=torch.zeros(10, 4, device="cuda", dtype=torch.float64))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(binding.LimeError, match="multiple"):
        call(q=q[:, :3])
    with pytest.raises(binding.LimeError, match="overlap"):
        call(q=q[:1].expand(10, 4, 64))
    with pytest.raises(TypeError):
        call(q=q.half(), k=k.half(), v=k.half())
    wide = torch.zeros(10, 4, 256, device="cuda")
    with pytest.raises(binding.LimeError, match="exceeds 128"):
        call(q=wide, k=wide, v=wide)
    with pytest.raises(ValueError, match="gamma"):
        binding.lime_norm_rotary(q, k, torch.ones(32, device="cuda").bfloat16())
    with pytest.raises(ValueError, match="positions"):
        binding.lime_norm_rotary(q, k, positions=ints([1]))
    with pytest.raises(ValueError, match="same rows"):
        binding.lime_norm_rotary(q, k[:5])
    with pytest.raises(ValueError, match="sizes"):
        binding.lime_norm_rotary(q, k, QO=k)
    with pytest.raises(ValueError, match="go together"):
        binding.lime_norm_rotary_backward(q, None, q, k)
    x = torch.zeros(4, 64, device="cuda")
    with pytest.raises(ValueError, match="targets"):
        binding.lime_catalogue_loss(x, x, torch.zeros(4, device="cuda", dtype=torch.int64))
    with pytest.raises(ValueError, match="width"):
        binding.lime_catalogue_loss(x, torch.zeros(4, 32, device="cuda"), ints([0] * 4))
    with pytest.raises(ValueError, match="contiguous"):
        binding.lime_catalogue_loss(x.t(), x.t(), ints([0] * 64))
    with pytest.raises(binding.LimeError, match="exceeds 256"):
        binding.lime_catalogue_loss(torch.zeros(4, 257, device="cuda"), torch.zeros(4, 257, device="cuda"), ints([0] * 4))


# ------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_training_step_and_serving(dtype):
    """A causal block over packed histories and the next-item loss, its gradients against fp64 ones of the same stored values, and the
    last event of each history served alone from the cache of the others."""
    lens, d, hq, hk, dh, items = [90, 33, 140], 64, 4, 2, 32, 300
    at, dt = packed(lens), DT[dtype]
    n, wide = int(at[-1]), (hq + 2 * hk) * dh
    gen = torch.Generator().manual_seed(3)
    rand = lambda *s, std=1.0: (torch.randn(s, generator=gen, dtype=torch.float64) * std).to(dt)  # noqa: E731
    E, Wqkv, Wo, W = rand(n, d), rand(d, wide, std=d**-0.5), rand(hq * dh, d, std=d**-0.5), rand(items, d)
    gq, gk = (1 + rand(dh, std=0.2).float()).to(dt), (1 + rand(dh, std=0.2).float()).to(dt)
    pos = np.concatenate([np.arange(x) for x in lens])
    targets = torch.randint(0, items, (n,), generator=gen)
    targets[at[1:] - 1] = -1  # a history's last event has no next one
    live = targets >= 0

    # fp64, rounding nothing
    leaves = [x.double().requires_grad_() for x in (E, Wqkv, Wo, W, gq, gk)]
    e, wqkv, wo, w, g1, g2 = leaves
    q, k, v = (e @ wqkv).unflatten(1, (hq + 2 * hk, dh)).split((hq, hk, hk), 1)

    def turned(x, g):
        z = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * g
        a = torch.from_numpy(pos)[:, None, None] * 10000.0 ** (-2.0 * torch.arange(dh // 2, dtype=torch.float64) / dh)
        lo, hi = z[..., : dh // 2], z[..., dh // 2:]
        return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)

    q, k = turned(q, g1), turned(k, g2)
    out = []
    for b in range(len(lens)):
        s = slice(at[b], at[b + 1])
        kk, vv = (x[s].repeat_interleave(hq // hk, 1).transpose(0, 1) for x in (k, v))
        z = (q[s].transpose(0, 1) @ kk.transpose(1, 2) * dh**-0.5).masked_fill(torch.ones(lens[b], lens[b], dtype=torch.bool).triu(1), -np.inf)
        out.append((z.softmax(-1) @ vv).transpose(0, 1))
    h = e + torch.cat(out).flatten(1) @ wo
    want = torch.nn.functional.cross_entropy((h @ w.t() * d**-0.5)[live], targets[live])
    want_grads = torch.autograd.grad(want, leaves)

    # the framework's calls, with plain products between them
    E, Wqkv, Wo, W, gq, gk = (x.cuda() for x in (E, Wqkv, Wo, W, gq, gk))
    positions, off, t = ints(pos), ints(at), targets.int().cuda()
    qkv = (E @ Wqkv).unflatten(1, (hq + 2 * hk, dh))
    q0, k0, v0 = qkv.split((hq, hk, hk), 1)
    where = (off, off, max(lens), max(lens), dh**-0.5)
    qn, kn = binding.lime_norm_rotary(q0, k0, gq, gk, positions)
    O, lse = binding.lime_sequence_attention(qn, kn, v0, *where)
    H = E + O.flatten(1) @ Wo
    loss, loss_lse = binding.lime_catalogue_loss(H, W, t, d**-0.5)
    count = int(live.sum())
    dH, dW = binding.lime_catalogue_loss_backward(torch.full((n,), 1.0 / count, device="cuda"), H, W, t, loss_lse, d**-0.5)
    dqkv = torch.empty_like(qkv)
    dq, dk, dv = dqkv.split((hq, hk, hk), 1)
    binding.lime_sequence_attention_backward((dH @ Wo.t()).unflatten(1, (hq, dh)), qn, kn, v0, O, lse, *where, dQ=dq, dK=dk, dV=dv)
    _, _, dgq, dgk = binding.lime_norm_rotary_backward(dq, dk, q0, k0, gq, gk, positions, dQ=dq, dK=dk)
    got = (dH + dqkv.flatten(1) @ Wqkv.t(), E.t() @ dqkv.flatten(1), O.flatten(1).t() @ dH, dW, dgq, dgk)
    # up to eight tensors in a row are rounded on the way to a gradient: eight half steps of the storage type of its norm
    bar = 8 * U[dtype] if dtype == "bf16" else 2.0**-24 * 8 * n
    assert abs(float(loss.sum()) / count - float(want.detach())) <= bar * float(want.detach())
    for a, b in zip(got, want_grads):
        off_by = (a.double().cpu() - b).norm() / b.norm()
        assert off_by <= bar, off_by

    # serving: the last event of every history alone
    slot = max(lens) + 5
    cache = torch.full((2, len(lens) * slot, hk, dh), float("nan"), dtype=dt, device="cuda")
    for b, x in enumerate(lens):
        cache[0, b * slot:b * slot + x], cache[1, b * slot:b * slot + x] = kn[at[b]:at[b + 1]], v0[at[b]:at[b + 1]]
    last = torch.from_numpy(at[1:] - 1).cuda()
    q1, _ = binding.lime_norm_rotary(q0[last], None, gq, None, positions[last])
    assert torch.equal(q1, qn[last])
    O1, lse1 = binding.lime_sequence_attention(q1, cache[0], cache[1], ints(range(len(lens) + 1)), ints(np.arange(len(lens) + 1) * slot), 1, slot, dh**-0.5,
                                               k_lens=ints(lens))
    # the same sums over the same keys, in other chunks: two roundings of p and one of the result
    assert ((O1.float() - O[last].float()).norm() / O[last].float().norm()) <= 3 * U[dtype] + 2.0**-20
    assert (lse1 - lse[last]).abs().max() <= 2.0**-18 * (1 + lse[last].abs().max())
