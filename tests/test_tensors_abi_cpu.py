"""Refusals and limits of AdamW over many tensors, without a GPU: every argument is
checked before anything is enqueued, the state's address last."""
import ctypes
import math

import numpy as np
import pytest

import paper_2609_20359_amd as P
import state8 as S8
from paper_2609_20359_amd import flround as F

INVALID, ALIGN = F.FL_ERR_INVALID, F.FL_ERR_ALIGN
A = 1 << 20   # an address that is aligned to anything; never dereferenced
H = F.AdamwHparams(1e-3, 0.9, 0.95, 1e-8, 0.1)
PASSED = ALIGN   # of a state at an odd address


def step(tensors=((100, A, 2 * A, 1),), grads=(3 * A,), dtype=1, scale=1.0, h=H, number=1, bits=8,
         state=A + 1, seed=0, count=None):
    arr = (F.FlTensor * max(len(tensors), 1))(*[F.FlTensor(*t) for t in tensors])
    g = (ctypes.c_void_p * max(len(grads), 1))(*grads)
    return P.lib().fl_adamw_tensors(len(tensors) if count is None else count, arr, g, dtype, scale,
                                    ctypes.byref(h), number, bits, state, seed, None)


def test_what_passes():
    assert step() == PASSED
    assert step(tensors=((100, A, None, 0),)) == PASSED            # no working copy
    assert step(bits=32) == step(seed=7) == step(dtype=0, grads=(3 * A + 2,)) == PASSED
    assert step(tensors=((100, A + 4, A + 2, 0),), grads=(3 * A + 4,)) == PASSED
    assert step(tensors=((0, None, None, 0), (5, A, None, 0)), grads=(None, 3 * A)) == PASSED
    assert step(tensors=((1 << 41, A, None, 0),)) == PASSED
    assert step(tensors=((5, A, None, 0),), grads=(None,)) == PASSED
    assert step(tensors=(), grads=(), state=None) == F.FL_OK
    assert step(tensors=((0, None, None, 0),), state=None) == F.FL_OK


def test_refusals():
    assert step(count=-1) == INVALID
    for t in ((-1, A, None, 0), ((1 << 41) + 1, A, None, 0), (5, None, None, 0)):
        assert step(tensors=(t,)) == INVALID, t
    assert step(tensors=((1 << 41, A, None, 0), (1, A, None, 0)), grads=(A, A)) == INVALID
    assert step(state=None) == INVALID
    assert step(tensors=((5, A + 2, None, 0),)) == step(tensors=((5, A, A + 1, 0),)) == ALIGN
    assert step(grads=(A + 2,)) == ALIGN
    assert step(grads=(A,)) == step(grads=(2 * A,)) == INVALID      # the gradient is an output
    for kw in (dict(dtype=2), dict(scale=math.inf), dict(scale=math.nan), dict(number=0),
               dict(bits=16), dict(bits=0), dict(bits=32, seed=1)):
        assert step(**kw) == INVALID, kw
    for bad in ((math.nan, .9, .9, 1e-8, 0), (1e-3, 1.0, .9, 1e-8, 0), (1e-3, .9, -.1, 1e-8, 0),
                (1e-3, .9, .9, 0, 0), (1e-3, .9, .9, 1e-8, -1)):
        assert step(h=F.AdamwHparams(*bad)) == INVALID, bad
    L = P.lib()
    arr = (F.FlTensor * 1)(F.FlTensor(5, A, None, 0))
    assert L.fl_adamw_tensors(1, None, arr, 1, 1.0, ctypes.byref(H), 1, 8, A + 1, 0, None) == INVALID
    assert L.fl_adamw_tensors(1, arr, None, 1, 1.0, ctypes.byref(H), 1, 8, A + 1, 0, None) == INVALID
    assert L.fl_adamw_tensors(1, arr, arr, 1, 1.0, None, 1, 8, A + 1, 0, None) == INVALID


def test_sizes():
    L = P.lib()

    def numel(*sizes):
        arr = (F.FlTensor * max(len(sizes), 1))(*[F.FlTensor(n, None, None, 0) for n in sizes])
        return L.fl_tensors_state_numel(len(sizes), arr)

    assert numel() == 0 and numel(0) == 0 and numel(1) == 512 and numel(512) == 512
    assert numel(513, 0, 1) == 1536 and numel((1 << 40) + 1, 1) == (1 << 40) + 1024
    assert numel(-1) == numel((1 << 41) + 1) == numel(1 << 41, 1) == -1
    assert L.fl_tensors_state_numel(1, None) == L.fl_tensors_state_numel(-1, None) == -1
    assert L.fl_tensors_state_bytes(1024, 32) == 8192
    assert L.fl_tensors_state_bytes(1024, 8) == 2048 + 32
    for n, bits in ((-512, 8), (100, 8), (512, 16), ((1 << 41) + 512, 8)):
        assert L.fl_tensors_state_bytes(n, bits) == 0


def test_convert():
    c = P.lib().fl_state_convert
    assert c(0, 8, None, None, None) == F.FL_OK
    assert c(512, 8, A + 1, 2 * A, None) == c(512, 32, A, 2 * A + 8, None) == ALIGN
    assert c(512, 8, A, A, None) == c(512, 8, None, A, None) == c(512, 8, A, None, None) == INVALID
    assert c(-512, 8, A, 2 * A, None) == c(100, 8, A, 2 * A, None) == c(512, 16, A, 2 * A, None) == INVALID
    assert c((1 << 41) + 512, 8, A, 2 * A, None) == INVALID


def test_binding_refuses_cpu_tensors():
    import torch

    with pytest.raises(ValueError):
        P.Tensors([torch.zeros(10)])
    with pytest.raises(ValueError):
        P.fl_state_convert(torch.zeros(2, dtype=torch.uint8), torch.zeros(4))


def test_codes_hold_what_they_stand_for():
    """The definition itself: every code's value is held by that code, whatever its block's
    exponent; a value between two codes goes to the nearer one."""
    for top in (S8.TOP_M, S8.TOP_V):
        t = S8.table(top)
        assert (np.diff(t) > 0).all() and t[-1] == 1.75
        for b in (12, 13, 60, 127, 200, 254):
            x = np.resize(t, (len(t) + 63) // 64 * 64) * 2.0 ** (b - 127)
            x = x[:len(t)].astype(np.float32)
            x = x[x > 0]
            for k in range(0, len(x), 63):
                block = np.zeros(64, np.float32)
                block[:len(x[k:k + 63])] = x[k:k + 63]
                block[63] = t[-1] * 2.0 ** (b - 127)
                code, e = S8.encode(block, top)
                assert e[0] == b and np.array_equal(S8.decode(code, e, top), block)
                # less than half a code's step more (no more than the block's largest)
                other = np.minimum(block * np.float32(1 + 2.0 ** -6), block[63])
                normal = block >= t[8] * 2.0 ** (b - 127)
                assert np.array_equal(S8.encode(other, top)[0][normal], code[normal])
