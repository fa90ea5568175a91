"""The loss's gradients for rows that have learnt their target: p of the target from one half to nearly one, where its e = p - 1 is
small beside p.  The bounds take e as it is, not p less one: half a step of the storage type (u) for e of every other item as an operand,
fp32 errors for the target's own.

fp32 errors: a logit's sum of d products is off by (d + 8) F of the sum of their magnitudes L, the logarithm and the sum over the items by
items + 16 steps, and lse once more by its own size; exp turns them into relative errors of p."""

import numpy as np
import pytest
import torch

from oracle import encoder_oracle as enc
from paper_2510_18239_amd import binding
from test_gpu_encoder import F, U, DT, ints, within

pytestmark = pytest.mark.gpu


def learnt(rows, items, d, dtype, seed, low, high):
    """Rows along their target's direction: logits of the targets near `low` .. `high` above the logarithm of the others' sum."""
    r = np.random.default_rng(seed)
    W = torch.from_numpy(r.standard_normal((items, d))).to(DT[dtype])
    w, t, scale = W.double().numpy(), r.integers(0, items, rows), d**-0.5
    gap = np.linspace(low, high, rows)
    square = (w[t] ** 2).sum(1) * scale  # the target's logit of a row that is the target itself
    along = (gap + np.log(items)) / square
    X = torch.from_numpy(w[t] * along[:, None] + 0.05 * r.standard_normal((rows, d))).to(DT[dtype])
    return X, W, t, scale


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,items,d,unlabelled", [(200, 1000, 64, 0.0), (131, 200, 32, 0.2), (300, 77, 256, 0.1), (97, 3000, 96, 0.0), (40, 130, 33, 0.3),
                                                     (5000, 64, 128, 0.05), (1, 500, 64, 0.0)])
def test_gradients_of_rows_that_have_learnt_their_target(dtype, rows, items, d, unlabelled):
    u = U[dtype]
    x, w, t, scale = learnt(rows, items, d, dtype, rows + d, 0.5, 10.0)
    X, W = x.double().numpy(), w.double().numpy()
    r = np.random.default_rng(1)
    none = r.random(rows) < unlabelled
    t = np.where(none, -1, t)
    dl = r.standard_normal(rows).astype(np.float32)
    x, w = x.cuda(), w.cuda()
    loss, lse = binding.lime_catalogue_loss(x, w, ints(t), scale)
    dX, dW = binding.lime_catalogue_loss_backward(torch.from_numpy(dl).cuda(), x, w, ints(t), lse, scale)
    wl, _, e = enc.catalogue_loss(X, W, t, scale)
    wX, wW = enc.catalogue_loss_backward(dl, X, W, t, scale)
    if rows > 100:  # what this test is about is there
        p = 1 + e[~none, t[~none]]
        assert p.min() < 0.8 and p.max() > 0.999
    L = abs(scale) * (abs(X) @ abs(W).T).max(1)
    z_off = F * (d + 8) * L
    lse_off = z_off + F * (items + 16) + F * 8 * (1 + L + np.log(items))
    off = (z_off + lse_off)[:, None] + 4 * F  # relative, of p
    weight = np.where(none, 0, abs(dl) * abs(scale))[:, None]
    others, own = abs(e), np.zeros_like(e)
    at = (np.nonzero(~none)[0], t[~none])
    own[at], others[at] = 1.0, 0.0
    own = own * (off + 8 * F * abs(e))  # of e = p - 1, with p at most 1
    each = others * (u + off)
    within(loss, wl, np.where(none, 0, 2 * lse_off + z_off), "loss")
    within(dX, wX, u * abs(wX) + weight * ((each + own + F * items * abs(e)) @ abs(W)), "dX")
    rest = np.where(own > 0, u * u * abs(e), 0)  # an item's sum has its targets' e in two parts
    within(dW, wW, u * abs(wW) + (weight * (each + own + rest + F * rows * abs(e))).T @ abs(X), "dW")


def test_a_decided_row_is_still_pulled_to_its_target():
    """Two items, p = 0.998 .. 0.9999 of the target: dX = (p - 1) (W_target - W_other), so its sign and size show the target's own e."""
    d = 32
    w = torch.zeros(2, d, dtype=torch.bfloat16)
    w[0], w[1] = 1.0, -1.0
    for gap in (6.25, 7.5, 9.0):
        x = torch.full((1, d), gap / (2 * d), dtype=torch.bfloat16)
        z = float((x.double() @ w.double().t())[0, 0])
        _, lse = binding.lime_catalogue_loss(x.cuda(), w.cuda(), ints([0]), 1.0)
        dX, _ = binding.lime_catalogue_loss_backward(torch.ones(1, device="cuda"), x.cuda(), w.cuda(), ints([0]), lse, 1.0)
        q = 1 / (1 + np.exp(2 * z))  # p of the other item
        # half a step for p of the other as an operand and for the result; fp32: the logits' 40 F of |z| and the logarithm's steps, over q
        allowed = 2 * q * (2 * U["bf16"]) + 2 * (F * 40 * 3 * z + 16 * F)
        assert abs(dX.double().cpu().numpy() + 2 * q).max() <= allowed


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,d,scale", [(400, 256, 0.0625), (5000, 64, 0.125), (37, 100, -0.1)])
def test_loss_of_learnt_rows_among_large_logits(dtype, rows, d, scale):
    """Eight items whose logits all lie near 100 in size, so that lse and a target's logit agree in most of their bits: what is left is the loss.
    The target's logit is the one that went into lse, so that of its error only 1 - p is left, and of lse's sum the rounding of its few terms."""
    items, r = 8, np.random.default_rng(rows)
    W = torch.from_numpy(r.standard_normal((items, d))).to(DT[dtype])
    common = torch.from_numpy(np.sign(scale) * 100.0 / (abs(scale) * d) * np.ones(d))
    W = (W.double() + 1.0).to(DT[dtype])
    w, t = W.double().numpy(), r.integers(0, items, rows)
    gap = np.linspace(0.0, 12.0, rows)
    apart = w[t] - w.mean(0)
    X = torch.from_numpy(common.numpy() + apart * (gap / ((apart * w[t]).sum(1) * scale))[:, None]).to(DT[dtype])
    x = X.double().numpy()
    loss, lse = binding.lime_catalogue_loss(X.cuda(), W.cuda(), ints(t), scale)
    want, wlse, e = enc.catalogue_loss(x, w, t, scale)
    L = abs(scale) * (abs(x) @ abs(w).T).max(1)
    rest = -e[np.arange(rows), t]
    assert rest.min() < 1e-3 and rest.max() > 0.3 and abs(wlse).min() > 60
    # logits: d + 8 steps of L, of the target and of the others, as far as they matter; the maximum's product and the sum of eight terms of at most
    # one, its logarithm and the products that follow: 32 steps of one, and of the loss
    within(loss, want, F * (rest * 2 * (d + 8) * L + 32 * (1 + want)), "loss")
    # what is handed to the gradients: one rounding of lse besides
    within(lse, wlse, F * ((d + 8) * L + 32 * (1 + want) + abs(wlse)), "lse")
