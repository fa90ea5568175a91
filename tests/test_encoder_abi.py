"""Refusals of the history encoder's entry points, made on the host before anything is launched (no GPU needed)."""

import ctypes

import pytest
import torch

from paper_2510_18239_amd import binding

FAKE = 0x1000  # never dereferenced: every call below fails its host-side checks
ROOM = 1 << 62


def rotary(Q=FAKE, qs=128, K=FAKE, ks=64, gq=None, gk=None, pos=FAKE, base=1e4, eps=1e-6, QO=FAKE, qos=128, KO=FAKE, kos=64, rows=0, hq=2, hk=1, dh=64,
           dtype=1):
    return binding.lib().lime_norm_rotary(Q, qs, K, ks, gq, gk, pos, base, eps, QO, qos, KO, kos, rows, hq, hk, dh, dtype, None)


def test_rotary():
    assert rotary() == 1 and "positive" in binding.last_error()
    assert rotary(rows=4, Q=None) == 1 and rotary(rows=4, QO=None) == 1 and rotary(rows=4, K=None) == 1 and rotary(rows=4, KO=None) == 1
    assert rotary(rows=4, hq=0) == 1 and rotary(rows=4, hk=-1) == 1 and rotary(rows=4, dtype=2) == 1
    assert rotary(rows=4, dh=63) == 1 and "odd" in binding.last_error()
    assert rotary(rows=4, dh=258, qs=1000, qos=1000) == 2
    assert rotary(rows=4, base=0.0) == 1 and rotary(rows=4, base=float("nan")) == 1 and rotary(rows=4, eps=-1.0) == 1
    assert rotary(rows=4, qs=127) == 1 and "overlap" in binding.last_error()
    assert rotary(rows=4, qos=127) == 1 and rotary(rows=4, ks=0) == 1 and rotary(rows=4, kos=63) == 1
    assert rotary(rows=4, qs=1 << 23) == 2
    assert rotary(rows=1 << 31) == 2
    assert rotary(rows=(1 << 31) - 1) == 2  # more than one launch takes


def rotary_backward(dQO=FAKE, Q=FAKE, dQ=FAKE, hk=0, rows=4, ws=FAKE, ws_bytes=0, dh=64, K=None):
    return binding.lib().lime_norm_rotary_backward(dQO, 128, None, 0, Q, 128, K, 0, None, None, None, 1e4, 1e-6, dQ, 128, None, 0, None, None, rows, 2, hk, dh, 1,
                                                   ws, ws_bytes, None)


def test_rotary_backward():
    need = binding.lib().lime_norm_rotary_backward_workspace_bytes(4, 64)
    assert need > 0 and need % 256 == 0
    assert rotary_backward() == 3 and rotary_backward(ws=None, ws_bytes=ROOM) == 3 and rotary_backward(ws_bytes=need - 1) == 3
    assert rotary_backward(ws=FAKE + 16, ws_bytes=ROOM) == 1 and "aligned" in binding.last_error()
    assert rotary_backward(dQO=None) == 1 and rotary_backward(Q=None) == 1 and rotary_backward(dQ=None) == 1 and rotary_backward(hk=1) == 1
    assert rotary_backward(rows=0) == 1 and rotary_backward(dh=7) == 1
    size = binding.lib().lime_norm_rotary_backward_workspace_bytes
    assert size(0, 64) == 0 and size(4, 63) == 0 and size(4, 300) == 0 and size(1 << 40, 64) == size(1 << 20, 64)


def where(q_offsets=FAKE, k_offsets=FAKE, q_lens=None, k_lens=None, q_rows=100, k_rows=100, B=2, max_q=50, max_k=50):
    return binding.Sequences(q_offsets, k_offsets, q_lens, k_lens, q_rows, k_rows, B, max_q, max_k)


def attention(w=None, Q=FAKE, qs=256, K=FAKE, ks=128, V=FAKE, vs=128, O=FAKE, lse=FAKE, hq=4, hk=2, dh=64, dtype=1, ws=FAKE, ws_bytes=0, null=False):
    w = None if null else ctypes.byref(w or where())
    return binding.lib().lime_sequence_attention(w, Q, qs, K, ks, V, vs, O, lse, hq, hk, dh, 1.0, 1, dtype, ws, ws_bytes, None)


def attention_backward(w=None, dO=FAKE, Q=FAKE, K=FAKE, V=FAKE, O=FAKE, lse=FAKE, dQ=FAKE, dqs=256, dK=FAKE, dks=128, dV=FAKE, dvs=128, hq=4, hk=2, dh=64,
                       ws=FAKE, ws_bytes=0):
    return binding.lib().lime_sequence_attention_backward(ctypes.byref(w or where()), dO, Q, 256, K, 128, V, 128, O, lse, dQ, dqs, dK, dks, dV, dvs, hq, hk, dh, 1.0,
                                                          1, 1, ws, ws_bytes, None)


def test_attention():
    assert attention() == 3 and attention(ws=None, ws_bytes=ROOM) == 3
    assert attention(ws=FAKE + 8, ws_bytes=ROOM) == 1
    assert attention(null=True) == 1 and attention(where(q_offsets=None)) == 1 and attention(where(k_offsets=None)) == 1
    assert attention(Q=None) == 1 and attention(K=None) == 1 and attention(V=None) == 1 and attention(O=None) == 1
    assert attention(where(B=0)) == 1 and attention(where(q_rows=-1)) == 1 and attention(where(max_k=-1)) == 1
    assert attention(where(B=70000)) == 2 and attention(where(q_rows=1 << 31)) == 2
    assert attention(hq=3) == 1 and "multiple" in binding.last_error()
    assert attention(hk=0) == 1 and attention(dh=0) == 1 and attention(dtype=9) == 1
    assert attention(dh=130, qs=1000, ks=1000, vs=1000) == 2
    assert attention(qs=255) == 1 and attention(ks=127) == 1 and attention(vs=0) == 1 and attention(qs=1 << 23) == 2
    big = where(q_rows=(1 << 31) - 1, k_rows=(1 << 31) - 1, max_q=(1 << 31) - 1, max_k=(1 << 31) - 1, B=60000)
    assert attention(big, ws_bytes=ROOM) == 2 and "launch" in binding.last_error()
    # nothing to do is not an error
    assert attention(where(q_rows=0), Q=None, O=None, lse=None, ws_bytes=ROOM) == 0
    assert attention(where(max_q=0), ws_bytes=ROOM) == 0


def test_attention_backward():
    assert attention_backward() == 3
    for name in ("dO", "Q", "K", "V", "O", "lse", "dQ", "dK", "dV"):
        assert attention_backward(**{name: None}) == 1, name
    assert attention_backward(dqs=255) == 1 and attention_backward(dks=1) == 1 and attention_backward(dvs=-128) == 1
    assert attention_backward(hq=5) == 1 and attention_backward(where(B=-1)) == 1
    assert attention_backward(where(q_rows=0, k_rows=0), Q=None, K=None, V=None, O=None, dO=None, lse=None, dQ=None, dK=None, dV=None, ws_bytes=ROOM) == 0


def test_attention_workspace():
    size = binding.lib().lime_sequence_attention_workspace_bytes
    ask = lambda backward=0, hq=4, hk=2, dh=64, **kw: size(ctypes.byref(where(**kw)), hq, hk, dh, 1, backward)  # noqa: E731
    assert ask() >= 256 and ask() % 256 == 0 and ask(1) >= 2 * 100 * 4 * 4
    assert ask(hk=3) == 0 and ask(dh=129) == 0 and ask(B=0) == 0 and size(None, 4, 2, 64, 1, 0) == 0
    few = dict(B=4, max_q=1, q_rows=4, max_k=100000, k_rows=400000)
    assert ask(**few) > 4 * 64 * 4 * 4  # the chunks' states
    assert ask(q_rows=0, k_rows=0) >= 256
    most = dict(B=1 << 30, q_rows=1 << 40, k_rows=1 << 40, max_q=(1 << 31) - 1, max_k=(1 << 31) - 1)
    assert ask(0, 1 << 30, 1 << 30, **most) == 0 and ask(1, 1 << 30, 1 << 30, **most) == 0  # past the limits: their products pass 64 bits
    largest = dict(B=65535, q_rows=(1 << 31) - 1, k_rows=(1 << 31) - 1, max_q=(1 << 31) - 1, max_k=(1 << 31) - 1)
    assert ask(0, 65535, 65535, **largest) >= 256 and ask(1, 65535, 65535, **largest) > 0
    assert binding.lib().lime_catalogue_loss_workspace_bytes((1 << 63) - 1, 10, 64, 1, 1) == 0


def loss(X=FAKE, W=FAKE, t=FAKE, out=FAKE, lse=FAKE, rows=10, items=20, d=64, dtype=1, ws=FAKE, ws_bytes=0):
    return binding.lib().lime_catalogue_loss(X, W, t, out, lse, rows, items, d, 1.0, dtype, ws, ws_bytes, None)


def loss_backward(g=FAKE, X=FAKE, W=FAKE, t=FAKE, lse=FAKE, dX=FAKE, dW=FAKE, rows=10, items=20, d=64, ws=FAKE, ws_bytes=0):
    return binding.lib().lime_catalogue_loss_backward(g, X, W, t, lse, dX, dW, rows, items, d, 1.0, 0, ws, ws_bytes, None)


def test_loss():
    assert loss() == 3 and loss(ws=FAKE + 128, ws_bytes=ROOM) == 1
    assert loss(X=None) == 1 and loss(W=None) == 1 and loss(t=None) == 1 and loss(out=None) == 1 and loss(lse=None) == 1
    assert loss(rows=0) == 1 and loss(items=0) == 1 and loss(d=-1) == 1 and loss(dtype=3) == 1
    assert loss(d=257) == 2 and loss(rows=1 << 26) == 2
    assert loss_backward() == 3
    for name in ("g", "X", "W", "t", "lse"):
        assert loss_backward(**{name: None}) == 1, name
    assert loss_backward(dX=None, dW=None) == 1 and loss_backward(dX=None) == 3 and loss_backward(d=300) == 2
    size = binding.lib().lime_catalogue_loss_workspace_bytes
    assert size(10, 20, 64, 1, 0) % 256 == 0 and size(10, 20, 64, 1, 1) > size(10, 20, 64, 1, 0) > 0
    assert size(0, 20, 64, 1, 0) == 0 and size(10, 20, 257, 1, 0) == 0 and size(10, 20, 64, 5, 0) == 0


def test_binding_refuses_what_it_cannot_hand_on():
    x = torch.zeros(4, 2, 8)
    off = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        binding.lime_norm_rotary(x, None)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        binding.lime_norm_rotary(x.double(), None)
    with pytest.raises(ValueError, match="CUDA"):
        binding.lime_sequence_attention(x, x, x, off, off, 2, 2, 1.0)
    with pytest.raises(ValueError, match="required"):
        binding.lime_sequence_attention(x, None, x, off, off, 2, 2, 1.0)
    with pytest.raises(ValueError, match="CUDA"):
        binding.lime_catalogue_loss(torch.zeros(4, 8), torch.zeros(5, 8), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match=r"\[rows, hq, dh\]"):
        binding.lime_norm_rotary(torch.zeros(4, 8), None)
