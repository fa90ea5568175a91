"""CPU oracle of the history encoder's operators (numpy fp64): the formulas written out, user by user and head by head, and for each
result the sums of magnitudes that bound what rounding can do to it."""

from __future__ import annotations

import numpy as np


# ----------------------------------------------------------------------------- norms and rotation of heads
def _turn(positions, rows, dh, base):
    i = np.arange(dh // 2)
    p = np.zeros(rows) if positions is None else np.asarray(positions, dtype=np.float64)
    angle = p[:, None] * np.float64(base) ** (-2.0 * i / dh)
    return np.exp(1j * angle)[:, None, :] if positions is not None else np.ones((rows, 1, dh // 2), dtype=complex)


def norm_rotary(x, gamma, positions, base, eps):
    """y [rows, heads, dh] and a bound of the terms it is summed from."""
    rows, _, dh = x.shape
    h = dh // 2
    g = np.ones(dh) if gamma is None else gamma
    z = x / np.sqrt((x**2).mean(-1, keepdims=True) + eps) * g
    y = (z[..., :h] + 1j * z[..., h:]) * _turn(positions, rows, dh, base)
    size = np.abs(z[..., :h]) + np.abs(z[..., h:])
    return np.concatenate([y.real, y.imag], -1), np.concatenate([size, size], -1)


def norm_rotary_backward(dy, x, gamma, positions, base, eps):
    """(dx, dgamma) and the magnitudes of their terms."""
    rows, _, dh = x.shape
    h = dh // 2
    g = np.ones(dh) if gamma is None else gamma
    s = np.sqrt((x**2).mean(-1, keepdims=True) + eps)
    n = x / s
    b = (dy[..., :h] + 1j * dy[..., h:]) * _turn(positions, rows, dh, base).conj()
    dz = np.concatenate([b.real, b.imag], -1)
    dn = dz * g
    dx = (dn - n * (dn * n).mean(-1, keepdims=True)) / s
    size = np.abs(dy[..., :h]) + np.abs(dy[..., h:])
    dz_size = np.concatenate([size, size], -1)
    dn_size = dz_size * np.abs(g)
    dx_size = (dn_size + np.abs(n) * (dn_size * np.abs(n)).mean(-1, keepdims=True)) / s
    return (dx, (dz * n).sum((0, 1))), (dx_size, (dz_size * np.abs(n)).sum((0, 1)))


# ----------------------------------------------------------------------------- attention over packed sequences
def spans(offsets, lens, rows):
    out = []
    for b in range(len(offsets) - 1):
        used = offsets[b + 1] - offsets[b] if lens is None else lens[b]
        out.append((int(offsets[b]), int(offsets[b + 1]), int(used)))
    return out


def visible(n_q, n_k, causal):
    return np.tril(np.ones((n_q, n_k), dtype=bool), n_k - n_q) if causal else np.ones((n_q, n_k), dtype=bool)


def sequence_attention(Q, K, V, q_spans, k_spans, scale, causal):
    """O, lse, and per user and head the pieces the gradients need: {(b, head): (rows, keys, p, mask)}."""
    hq, hk = Q.shape[1], K.shape[1]
    O, lse, inside = np.zeros(Q.shape), np.full(Q.shape[:2], -np.inf), {}
    for b, ((q0, _, nq), (k0, _, nk)) in enumerate(zip(q_spans, k_spans)):
        mask = visible(nq, nk, causal)
        for a in range(hq):
            q, k, v = Q[q0:q0 + nq, a], K[k0:k0 + nk, a // (hq // hk)], V[k0:k0 + nk, a // (hq // hk)]
            z = np.where(mask, scale * (q @ k.T), -np.inf)
            top = z.max(1, initial=-np.inf)
            seen = np.isfinite(top)
            p = np.where(mask, np.exp(z - np.where(seen, top, 0.0)[:, None]), 0.0)
            total = p.sum(1)
            p = p / np.where(seen, total, 1.0)[:, None]
            lse[q0:q0 + nq, a] = np.where(seen, np.where(seen, top, 0.0) + np.log(np.where(seen, total, 1.0)), -np.inf)
            O[q0:q0 + nq, a] = p @ v
            inside[b, a] = (slice(q0, q0 + nq), slice(k0, k0 + nk), p, mask)
    return O, lse, inside


def sequence_attention_backward(dO, Q, K, V, O, inside, scale):
    hq, hk = Q.shape[1], K.shape[1]
    dQ, dK, dV = np.zeros(Q.shape), np.zeros(K.shape), np.zeros(V.shape)
    for (_, a), (rq, rk, p, _) in inside.items():
        c = a // (hq // hk)
        e = p * (dO[rq, a] @ V[rk, c].T - (dO[rq, a] * O[rq, a]).sum(1)[:, None])
        dQ[rq, a] = scale * (e @ K[rk, c])
        dK[rk, c] += scale * (e.T @ Q[rq, a])
        dV[rk, c] += p.T @ dO[rq, a]
    return dQ, dK, dV


def sequence_attention_bounds(Q, K, V, dO, O, inside, scale, u, causal):
    """How far O, lse, dQ, dK, dV may be from the formulas: a row's p is off by e32 (fp32 logits, exponential and sum) and, as an
    operand, by u (half a step of the storage type); so is e; D carries the error of the O it is taken from; each result is rounded once."""
    f = 2.0**-24
    hq, hk, dh = Q.shape[1], K.shape[1], Q.shape[2]
    tO, tl, tQ, tK, tV = np.zeros(Q.shape), np.zeros(Q.shape[:2]), np.zeros(Q.shape), np.zeros(K.shape), np.zeros(V.shape)
    aQ, aK, aV = abs(Q), abs(K), abs(V)
    for (_, a), (rq, rk, p, mask) in inside.items():
        c = a // (hq // hk)
        if p.size == 0:
            continue
        L = np.where(mask, abs(scale) * (aQ[rq, a] @ aK[rk, c].T), 0.0).max(1)[:, None]
        e32 = f * ((dh + 8) * L + p.shape[1] + 16)
        tO[rq, a] = u * abs(O[rq, a]) + (u + 2 * e32) * (p @ aV[rk, c])
        tl[rq, a] = e32[:, 0] + f * 8 * (1 + L[:, 0] + np.log(p.shape[1]))
        if dO is None:
            continue
        g = abs(dO[rq, a])
        d_off = (g * tO[rq, a]).sum(1)[:, None] + f * dh * ((g * abs(O[rq, a])).sum(1)[:, None] + g @ aV[rk, c].T)
        e = p * abs(dO[rq, a] @ V[rk, c].T - (dO[rq, a] * O[rq, a]).sum(1)[:, None])
        e_off = p * d_off * (1 + 2 * e32) + e * (u + 2 * e32) + f * p.shape[0] * e
        tQ[rq, a] = abs(scale) * (e_off @ aK[rk, c])
        tK[rk, c] += abs(scale) * (e_off.T @ aQ[rq, a])
        tV[rk, c] += ((u + 2 * e32 + f * p.shape[0]) * p).T @ g
    return tO, tl, tQ, tK, tV


# ----------------------------------------------------------------------------- softmax cross entropy over a catalogue
def catalogue_loss(X, W, targets, scale):
    """(loss, lse, e) with e the gradient of each row's loss in its logits."""
    live = (targets >= 0) & (targets < W.shape[0])
    z = scale * (np.where(live[:, None], X, 0.0) @ W.T)
    top = z.max(1, keepdims=True)
    lse = (top + np.log(np.exp(z - top).sum(1, keepdims=True)))[:, 0]
    rows = np.nonzero(live)[0]
    loss, e = np.zeros(len(X)), np.exp(z - lse[:, None])
    loss[rows] = lse[rows] - z[rows, targets[rows]]
    e[rows, targets[rows]] -= 1.0
    e[~live] = 0.0
    return loss, np.where(live, lse, 0.0), e


def catalogue_loss_backward(dloss, X, W, targets, scale):
    live = (targets >= 0) & (targets < W.shape[0])
    _, _, e = catalogue_loss(X, W, targets, scale)
    e = e * (np.where(live, dloss, 0.0) * scale)[:, None]
    return e @ W, e.T @ np.where(live[:, None], X, 0.0)
