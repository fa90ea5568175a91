"""Gradients of the last user of a padded batch of 6.8 GB a tensor: rows past 2^31 elements and 2^32 bytes.  (54 GB.)"""

import numpy as np
import pytest
import torch

from oracle import encoder_oracle as enc
from paper_2510_18239_amd import binding
from test_gpu_encoder import U, ints, make, within

pytestmark = pytest.mark.gpu


def test_gradients_past_32_bits():
    heads, dh, slot, users, n = 8, 128, 1_100_000, 3, 300
    rows, first, scale = slot * users, slot * (users - 1), dh**-0.5
    assert first * heads * dh > 2**31 and first * heads * dh * 2 > 2**32
    small = [make((n, heads, dh), "bf16", i) for i in range(4)]
    Q, K, V, G = (torch.empty(rows, heads, dh, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    for big, (x, _) in zip((Q, K, V, G), small):
        big[first:first + n] = x
    lens, off = ints([0, 0, n]), ints(np.arange(users + 1) * slot)
    where = dict(q_lens=lens, k_lens=lens)
    O, lse = binding.lime_sequence_attention(Q, K, V, off, off, slot, slot, scale, **where)
    got = binding.lime_sequence_attention_backward(G, Q, K, V, O, lse, off, off, slot, slot, scale, **where)
    q, k, v, g = (X for _, X in small)
    span = [(0, n, n)]
    wO, _, inside = enc.sequence_attention(q, k, v, span, span, scale, True)
    u = U["bf16"]
    tO, _, *t = enc.sequence_attention_bounds(q, k, v, g, wO, inside, scale, u, True)
    within(O[first:first + n], wO, tO, "O")
    for x, want, allowed, what in zip(got, enc.sequence_attention_backward(g, q, k, v, wO, inside, scale), t, ("dQ", "dK", "dV")):
        within(x[first:first + n], want, u * abs(want) + allowed, what)
        assert not x[:first].any() and not x[first + n:].any(), what  # rows of slots that are not in use
    del Q, K, V, G, O, got, x
    torch.cuda.empty_cache()
