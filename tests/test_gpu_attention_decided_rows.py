"""Gradients of the attention where D = sum_j p_j <G, V_j> is close to a row's <G, V_j> itself: rows whose softmax is nearly decided, rows
that see few keys, values with a common part.  There e_j = p_j (<G, V_j> - D) is small beside its two terms, and a D that comes from an O
rounded to the storage type is off by as much as e.

Bounds: e is off by u of itself as an operand, by the fp32 errors of p, and by p times the error of D; D by fp32 errors alone.  A first D
from the rounded O, off by u <|G|, |O|>, may enter dQ where it is taken back with p as an operand: u of itself, twice."""

import numpy as np
import pytest
import torch

from oracle import encoder_oracle as enc
from paper_2510_18239_amd import binding
from test_gpu_encoder import F, U, DT, ints, packed, within

pytestmark = pytest.mark.gpu


def bounds(Q, K, V, G, O, inside, scale, u):
    hq, hk, dh = Q.shape[1], K.shape[1], Q.shape[2]
    tQ, tK, tV = np.zeros(Q.shape), np.zeros(K.shape), np.zeros(V.shape)
    for (_, a), (rq, rk, p, mask) in inside.items():
        c = a // (hq // hk)
        if p.size == 0:
            continue
        q, k, v, g = abs(Q[rq, a]), abs(K[rk, c]), abs(V[rk, c]), abs(G[rq, a])
        L = np.where(mask, abs(scale) * (q @ k.T), 0.0).max(1)[:, None]
        e32 = F * ((dh + 8) * L + p.shape[1] + 16)  # relative, of p; its part common to a row is in D as well
        lse = F * 8 * (1 + L + np.log(p.shape[1]))
        dP, D = G[rq, a] @ V[rk, c].T, (G[rq, a] * O[rq, a]).sum(1)[:, None]
        dP_off = F * (dh + 8) * (g @ v.T)
        first = 2 * u * (g * abs(O[rq, a])).sum(1)[:, None]  # of the D from the rounded O (and the sums up to it)
        if u > F:
            D_off = (p * (2 * e32 * (abs(dP - D) + first) + dP_off)).sum(1)[:, None] + F * (dh + p.shape[1] + 16) * ((p * abs(dP)).sum(1)[:, None] + first) + 2 * lse * first
        else:  # fp32: <G, O>, O with the errors of p and of its own rounding
            D_off = (g * ((2 * u + 2 * e32) * (p @ v))).sum(1)[:, None] + F * dh * ((g * abs(O[rq, a])).sum(1)[:, None])
        e = p * abs(dP - D)
        fp32 = p * (D_off + dP_off) + e * 2 * (e32 + lse) + F * p.shape[1] * (e + p * first)
        tQ[rq, a] = abs(scale) * ((fp32 + u * e + 2 * u * p * first * (u > F)) @ k)
        tK[rk, c] += abs(scale) * ((p * (D_off + dP_off) + e * (u + 2 * (e32 + lse) + F * p.shape[0])).T @ q)
        tV[rk, c] += ((u + 2 * (e32 + lse) + F * p.shape[0]) * p).T @ g
    return tQ, tK, tV


def check(Q, K, V, G, q_lens, k_lens, dtype, scale=None, causal=True, least_p=None):
    dt, u = DT[dtype], U[dtype]
    scale = Q.shape[2] ** -0.5 if scale is None else scale
    q, k, v, g = (torch.from_numpy(x).to(dt) for x in (Q, K, V, G))
    Q, K, V, G = (x.double().numpy() for x in (q, k, v, g))
    q, k, v, g = (x.cuda() for x in (q, k, v, g))
    qo, ko = packed(q_lens), packed(k_lens)
    where = (ints(qo), ints(ko), int(max(q_lens)), int(max(k_lens)), scale)
    O, lse = binding.lime_sequence_attention(q, k, v, *where, causal=causal)
    got = binding.lime_sequence_attention_backward(g, q, k, v, O, lse, *where, causal=causal)
    wO, _, inside = enc.sequence_attention(Q, K, V, enc.spans(qo, q_lens, None), enc.spans(ko, k_lens, None), scale, causal)
    if least_p is not None:  # what this test is about is there
        assert max(p.max() for _, _, p, _ in inside.values()) >= least_p
    want = enc.sequence_attention_backward(G, Q, K, V, wO, inside, scale)
    for x, y, t, what in zip(got, want, bounds(Q, K, V, G, wO, inside, scale, u), ("dQ", "dK", "dV")):
        within(x, y, u * abs(y) + t, what)


def rand(seed, *shapes):
    r = np.random.default_rng(seed)
    return [r.standard_normal(s) for s in shapes]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n_q,n_k,hq,hk,dh", [(40, 1000, 1, 1, 64), (1000, 1000, 2, 1, 64), (600, 600, 4, 4, 32), (300, 300, 2, 1, 128), (260, 700, 3, 1, 40), (7, 513, 1, 1, 80),
                                              (200, 2000, 2, 2, 96), (130, 300, 1, 1, 20)])
def test_one_key_among_many_takes_nearly_all(dtype, n_q, n_k, hq, hk, dh):
    """Every query points at one of the keys that it sees, with p from one half to 0.9999."""
    Q, K, V, G = rand(n_q + dh, (n_q, hq, dh), (n_k, hk, dh), (n_k, hk, dh), (n_q, hq, dh))
    r = np.random.default_rng(1)
    for i in range(n_q):
        for a in range(hq):
            j, c = r.integers(0, n_k - n_q + i + 1), a // (hq // hk)
            gap = r.uniform(0, 9.2) + np.log(n_k)
            Q[i, a] = 0.2 * Q[i, a] + K[j, c] * gap * dh**0.5 / (K[j, c] ** 2).sum()
    check(Q, K, V, G, [n_q], [n_k], dtype, least_p=0.99)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("q_lens,k_lens,hq,hk,dh", [([256], [130], 1, 1, 64), ([256, 3], [131, 3], 2, 1, 32), ([400, 200, 100], [1, 2, 3], 1, 1, 128), ([700], [520], 4, 2, 64)])
def test_rows_of_few_keys_behind_rows_of_none(dtype, q_lens, k_lens, hq, hk, dh):
    """More queries than keys: the rows that see one, two, three keys stand in a later tile, beside rows that see many."""
    check(*rand(3, (sum(q_lens), hq, dh), (sum(k_lens), hk, dh), (sum(k_lens), hk, dh), (sum(q_lens), hq, dh)), q_lens, k_lens, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,hq,hk,dh", [(300, 2, 1, 64), (700, 1, 1, 32), (129, 4, 2, 128)])
def test_keys_and_values_with_a_common_part(dtype, causal, n, hq, hk, dh):
    """The common part of the values cancels in e, that of the keys in dQ, wherever e sums to zero."""
    Q, K, V, G = rand(5, (n, hq, dh), (n, hk, dh), (n, hk, dh), (n, hq, dh))
    check(Q * 0.5, K + 4.0, V + 8.0, G, [n], [n], dtype, causal=causal)
