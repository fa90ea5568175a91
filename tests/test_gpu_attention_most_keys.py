"""A user with 2^31 - 256 keys, the most that a call takes: the last chunk would end past 32 bits.  (34 GB of keys.)"""

import numpy as np
import pytest
import torch

from paper_2510_18239_amd import binding
from test_gpu_encoder import F, U, ints

pytestmark = pytest.mark.gpu


def test_the_last_of_2_31_keys():
    n, dh = 2**31 - 256, 8
    keys = torch.zeros(n, 1, dh, dtype=torch.bfloat16, device="cuda")
    keys[-1] = 2.5  # the only key with a logit, 40: exp(40) is 10^8 times the others' sum
    for hq in (1, 64):  # one wave a workgroup, and four
        q = torch.full((1, hq, dh), 2.0, dtype=torch.bfloat16, device="cuda")
        O, lse = binding.lime_sequence_attention(q, keys, keys, ints([0, 1]), ints([0, n]), 1, n, 1.0)
        others = n * np.exp(-40.0)
        # p of the last key and the result are rounded once each
        assert (O.float() - 2.5).abs().max() <= 2.5 * (2 * U["bf16"] + others)
        # fp32: 16 products and 40 steps of the largest logit, the logarithm's of lse, and the others
        assert (lse - 40.0).abs().max() <= F * 64 * 40 + others
    del keys, O
    torch.cuda.empty_cache()
