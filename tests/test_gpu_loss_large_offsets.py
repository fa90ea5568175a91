"""The loss of so many rows that their elements pass 2^31: the last of them, and the items' gradient, to which most rows add nothing.  (30 GB.)"""

import numpy as np
import pytest
import torch

from oracle import encoder_oracle as enc
from paper_2510_18239_amd import binding
from test_gpu_encoder import F, U, make, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("others", [True, False])  # rows without a target in front, which are not read; or rows of zeros without a weight
def test_rows_past_32_bits(others):
    d, items, n, rows, scale = 256, 40, 200, 9_000_001, 256**-0.5
    first = rows - n
    assert first * d > 2**31 and first * d * 2 > 2**32
    (x, X), (w, W) = make((n, d), "bf16", 0), make((items, d), "bf16", 1)
    t = np.random.default_rng(2).integers(0, items, n)
    big = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda").fill_(float("nan") if others else 0.0)
    big[first:] = x
    targets = torch.full((rows,), -1 if others else 3, dtype=torch.int32, device="cuda")
    targets[first:] = torch.from_numpy(t).int().cuda()
    weight = torch.zeros(rows, device="cuda")
    weight[first:] = 1.0
    loss, lse = binding.lime_catalogue_loss(big, w, targets, scale)
    dX, dW = binding.lime_catalogue_loss_backward(weight, big, w, targets, lse, scale)
    wl, wlse, e = enc.catalogue_loss(X, W, t, scale)
    wX, wW = enc.catalogue_loss_backward(np.ones(n), X, W, t, scale)
    u, L = U["bf16"], abs(scale) * (abs(X) @ abs(W).T).max(1)
    off = F * ((d + 8) * L + items + 16) + F * 8 * (1 + L + np.log(items))
    within(lse[first:], wlse, off, "lse")
    within(loss[first:], wl, 2 * off, "loss")
    if not others:  # equal logits
        assert (loss[:first] - np.log(items)).abs().max() <= 16 * F * (1 + np.log(items))
    each = scale * (abs(e) * (u + 4 * off[:, None] + F * n) + 4 * off[:, None])
    within(dX[first:], wX, u * abs(wX) + each @ abs(W), "dX")
    # (in chunks of many rows, all but n of which add nothing)
    within(dW, wW, u * abs(wW) + (each + scale * abs(e) * F * 4096).T @ abs(X), "dW")
    assert not dX[:first].any()
    del big, targets, weight, loss, lse, dX, dW
    torch.cuda.empty_cache()
