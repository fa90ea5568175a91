"""Workspace sizes of the attention for shapes that the calls refuse: a caller may ask for the size first (CPU)."""

import ctypes
import itertools

import pytest

from paper_2510_18239_amd import binding

FAKE = 0x1000  # never dereferenced


@pytest.mark.parametrize("backward", [0, 1])
def test_sizes_of_shapes_whose_tiles_pass_32_bits(backward):
    """max_q times the heads of a group beyond 2^31 and 2^32: no division by a count that was cut to 32 bits and became zero."""
    size = binding.lib().lime_sequence_attention_workspace_bytes
    most = (1 << 31) - 1
    for B, hq, hk, max_q, max_k, lens in itertools.product((1, 65535), (1, 32768, 65535), (1, 32768, 65535), (0, 1, 1 << 24, (1 << 24) + 1, most), (0, 1, 1 << 24, most), (None, FAKE)):
        if hq % hk:
            continue
        w = binding.Sequences(FAKE, FAKE, lens, lens, max(max_q, 1), max(max_k, 1), B, max_q, max_k)
        for dh, dtype in ((1, 0), (128, 1)):
            need = size(ctypes.byref(w), hq, hk, dh, dtype, backward)
            assert need % 256 == 0
            if backward:
                assert need >= 2 * w.q_rows * hq * 4  # two words a query and head
            else:  # fewer than 2^17 rows' states in all chunks together
                assert 256 <= need <= (1 << 17) * (128 + 2) * 4 + 512


@pytest.mark.parametrize("k_rows,max_k,status", [((1 << 31) - 1, (1 << 31) - 1, 2), ((1 << 31) - 255, (1 << 31) - 1, 2), ((1 << 31) - 1, (1 << 31) - 256, 3), (1 << 30, (1 << 31) - 1, 3)])
def test_most_keys(k_rows, max_k, status):
    """Slots that may end within a step of 2^31 are refused; a longest slot past the tensor counts as the tensor's rows."""
    w = binding.Sequences(FAKE, FAKE, None, None, 1, k_rows, 1, 1, max_k)
    assert binding.lib().lime_sequence_attention(ctypes.byref(w), FAKE, 8, FAKE, 8, FAKE, 8, FAKE, FAKE, 1, 1, 8, 1.0, 1, 1, FAKE, 0, None) == status
