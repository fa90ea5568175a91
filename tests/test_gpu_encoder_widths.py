"""Head widths with kernels of their own, in every form of the attention: histories, single events over cut caches, few new events, rows
that are not whole 16-byte pieces."""

import pytest

from test_gpu_encoder import attention_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh", [18, 48, 81, 88, 96])
@pytest.mark.parametrize("lens,hq,hk", [([65, 200, 0, 31], 2, 2), ([300], 6, 2)])
def test_histories(dtype, dh, lens, hq, hk):
    attention_case(dtype, lens, lens, hq, hk, dh)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh", [20, 40, 48, 72, 80, 84, 90, 96])
def test_single_events(dtype, dh):
    attention_case(dtype, [1, 1, 0, 1], [1500, 3, 700, 0], 8, 2, dh, slots=(1, 1500))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh", [48, 80, 96, 112])
@pytest.mark.parametrize("q_lens,slot", [([9, 16, 1], 16), ([50, 64, 7], 64)])  # a wave's rows, and more
def test_few_new_events(dtype, dh, q_lens, slot):
    attention_case(dtype, q_lens, [1000, 64, 300], 2, 1, dh, slots=(slot, 1000))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh,before", [(96, 1), (88, 3), (48, 8), (82, 0)])
def test_strided_rows(dtype, dh, before):
    attention_case(dtype, [65, 0, 30, 300], [65, 0, 30, 300], 4, 2, dh, before=before)
