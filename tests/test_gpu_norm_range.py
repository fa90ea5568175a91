"""Norms of heads whose squares leave fp32's range while they themselves do not: the norm is what it is at any size."""

import numpy as np
import pytest
import torch

from oracle import encoder_oracle as enc
from paper_2510_18239_amd import binding
from test_gpu_encoder import F, U, ints, make, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("power,eps", [(120, 1e-6), (80, 0.0), (60, 1e-6), (-80, 0.0), (-60, 0.0), (-33, 1e-30), (0, 0.0)])
@pytest.mark.parametrize("dh", [64, 20, 256])
def test_heads_of_any_size(dtype, power, eps, dh):
    """Every other row is of the size 2^power, those between them ordinary."""
    u, rows, base = U[dtype], 33, 10000.0
    size = np.where(np.arange(rows) % 2, 2.0**power, 1.0)[:, None, None]
    (q, Q), (g, G), (dy, DY) = make((rows, 3, dh), dtype, 1), make((dh,), dtype, 2, 0.3, 1.0), make((rows, 3, dh), dtype, 3)
    q, Q = (q.double() * torch.from_numpy(size).cuda()).to(q.dtype), Q * size  # (a power of two: no rounding)
    assert np.array_equal(q.double().cpu().numpy(), Q)
    pos = np.arange(rows) * 7
    eps = float(np.float32(eps))
    y, _ = binding.lime_norm_rotary(q, None, g, None, ints(pos), base, eps)
    want, s = enc.norm_rotary(Q, G, pos, base, eps)
    within(y, want, u * abs(want) + F * (dh + 24) * s, "y")
    dx, _, dg, _ = binding.lime_norm_rotary_backward(dy, None, q, None, g, None, ints(pos), base, eps)
    (wx, wg), (sx, sg) = enc.norm_rotary_backward(DY, Q, G, pos, base, eps)
    # a gradient below the least normal number loses bits: half a step there is 2^-150 (fp32), 2^-134 (bf16), and twice that for its factor
    least = 2.0**-149 * (2 + np.abs(sx * 2.0**power)) if dtype == "fp32" else 2.0**-133 + 2.0**-149 * np.abs(sx * 2.0**power)
    within(dx, wx, u * abs(wx) + F * (3 * dh + 40) * sx + least, "dx")
    within(dg, wg, u * abs(wg) + F * (dh + 40 + rows * 3) * sg, "dgamma")


def test_a_head_of_nothing_but_zeros():
    q = torch.zeros(5, 2, 64, device="cuda")
    q[1] = 1.0
    y, _ = binding.lime_norm_rotary(q, None, positions=ints(range(5)))
    assert (y[[0, 2, 3, 4]] == 0).all() and y[1].abs().max() > 0
