"""Two threads that call on one stream: a call's launches stay together, so that neither reads the other's scratch memory."""

import threading

import pytest
import torch

from paper_2510_18239_amd import binding
from test_gpu_encoder import ints, make, same

pytestmark = pytest.mark.gpu


def step(seed):
    """Calls of several launches each, of the same sizes for every seed."""
    rows, items, d = 300, 900, 64
    (x, _), (w, _), (g, _) = make((rows, d), "bf16", seed), make((items, d), "bf16", seed + 1), make((rows,), "fp32", seed + 2)
    (q, _), (k, _), (v, _), (o, _) = (make((n, h, 64), "bf16", seed + 3 + i) for i, (n, h) in enumerate(((8, 4), (4000, 2), (4000, 2), (8, 4))))
    t = (torch.arange(rows, device="cuda") * (seed + 7) % items).int()
    where = (ints([0, 4, 8]), ints([0, 2000, 4000]), 4, 2000, 0.125)

    def run():
        loss, lse = binding.lime_catalogue_loss(x, w, t, 0.1)
        out = (loss, lse) + binding.lime_catalogue_loss_backward(g, x, w, t, lse, 0.1)
        O, l = binding.lime_sequence_attention(q, k, v, *where)
        return out + (O, l) + binding.lime_sequence_attention_backward(o, q, k, v, O, l, *where)

    return run


def test_two_threads_on_one_stream():
    runs = [step(seed) for seed in (0, 100)]
    want = [run() for run in runs]
    torch.cuda.synchronize()
    got, start = [[], []], threading.Barrier(2)

    def work(i):
        start.wait()
        for _ in range(40):
            got[i].append(runs[i]())

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(len(g) == 40 for g in got)
    assert all(same(x, want[i]) for i in range(2) for x in got[i])
