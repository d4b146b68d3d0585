"""Refusals of the output head's entry points, without a GPU: every argument is
checked before anything is enqueued, so an invalid call returns its status and
a call that passes the checks is the only one to reach the device."""
import ctypes
import math

import pytest

import paper_2609_20359_amd as P
from paper_2609_20359_amd import flround as F

INVALID, ALIGN, SCRATCH = F.FL_ERR_INVALID, F.FL_ERR_ALIGN, F.FL_ERR_SCRATCH
A = 1 << 20   # an address that is aligned to anything; never dereferenced on the host
BIG = 1 << 40


def shape(T=8, V=100, D=64, lh=0, lw=0):
    return F.HeadShape(T, V, D, lh, lw)


def loss(s, hidden=A, weight=A, labels=A, out=A, lse=A, target=A, ws=A, nbytes=BIG):
    return P.lib().fl_head_loss(ctypes.byref(s), hidden, weight, labels, out, lse, target, ws, nbytes,
                                None)


def loss_grad(s, hidden=A, weight=2 * A, labels=A, lse=A, target=A, dloss=A, dh=3 * A, dw=4 * A,
              ws=A, nbytes=BIG):
    return P.lib().fl_head_loss_grad(ctypes.byref(s), hidden, weight, labels, lse, target, dloss, dh,
                                     dw, ws, nbytes, None)


def distill(s, k=4, ids=A, teacher=A, teacher_lse=A, tau=1.0, out=A, ws=A, nbytes=BIG):
    return P.lib().fl_head_distill(ctypes.byref(s), A, A, k, ids, teacher, teacher_lse, tau, out, A, A,
                                   ws, nbytes, None)


def distill_grad(s, k=4, tau=1.0, ids=A, dw=4 * A, ws=A, nbytes=BIG):
    return P.lib().fl_head_distill_grad(ctypes.byref(s), A, 2 * A, k, ids, A, None, tau, A, A, A, 3 * A,
                                        dw, ws, nbytes, None)


def top(rows=4, vocab=100, stride=0, dtype=0, logits=A, k=5, tau=1.0, values=A, ids=A, lse=A, ws=A,
        nbytes=BIG):
    return P.lib().fl_top_logits(rows, vocab, stride, dtype, logits, k, tau, values, ids, lse, ws,
                                 nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(V=0), dict(V=-5), dict(D=0), dict(T=(1 << 20) + 1), dict(V=(1 << 24) + 1),
    dict(D=(1 << 16) + 1), dict(lh=63), dict(lw=63), dict(lh=-8), dict(lw=(1 << 22) + 8),
    dict(T=1 << 20, V=1 << 24)])
def test_shapes(bad):
    s = shape(**bad)
    assert loss(s) == loss_grad(s) == distill(s) == distill_grad(s) == INVALID
    assert P.lib().fl_head_workspace_bytes(ctypes.byref(s), 0, 0) == 0
    assert P.lib().fl_head_workspace_bytes(None, 0, 0) == 0


def test_null_and_misaligned_pointers():
    s = shape()
    for name in ("hidden", "weight", "labels", "out", "lse", "target", "ws"):
        assert loss(s, **{name: None}) == INVALID, name
    for name in ("hidden", "weight", "labels", "lse", "target", "dloss", "dh", "dw", "ws"):
        assert loss_grad(s, **{name: None}) == INVALID, name
    for name in ("ids", "teacher", "out", "ws"):
        assert distill(s, **{name: None}) == INVALID, name
    assert loss(s, hidden=A + 1) == loss(s, weight=A + 2) == loss(s, labels=A + 4) == ALIGN
    assert loss(s, out=A + 2) == loss(s, lse=A + 1) == loss(s, target=A + 2) == ALIGN
    assert loss_grad(s, dh=A + 1) == loss_grad(s, dw=A + 1) == loss_grad(s, dloss=A + 2) == ALIGN
    assert distill(s, ids=A + 2) == distill(s, teacher=A + 2) == distill(s, teacher_lse=A + 1) == ALIGN
    for name in ("logits", "values", "ids"):
        assert top(**{name: None}) == INVALID, name
    assert top(logits=A + 1) == top(dtype=1, logits=A + 2) == top(values=A + 1) == ALIGN
    assert top(ids=A + 2) == top(lse=A + 3) == ALIGN


def test_outputs_that_are_inputs():
    s = shape()
    assert loss_grad(s, dw=2 * A) == loss_grad(s, dw=A) == INVALID
    assert loss_grad(s, dh=A) == loss_grad(s, dh=2 * A) == loss_grad(s, dh=4 * A) == INVALID


def test_targets():
    s = shape()
    for k in (0, -1, F.FL_MAX_TARGETS + 1):
        assert distill(s, k=k) == distill_grad(s, k=k) == INVALID
    for tau in (0.0, -1.0, math.inf, math.nan):
        assert distill(s, tau=tau) == distill_grad(s, tau=tau) == INVALID
        assert top(tau=tau) == INVALID
    for k in (0, -3, 101, 129):
        assert top(k=k) == INVALID
    assert top(vocab=1000, k=129) == INVALID


def test_top_shapes():
    assert top(rows=-1) == top(vocab=0) == top(stride=99) == top(dtype=2) == INVALID
    assert top(rows=(1 << 20) + 1) == top(vocab=(1 << 20) + 1) == INVALID
    assert top(rows=0, logits=None, values=None, ids=None) == F.FL_OK


def test_workspace_too_small():
    for T, V, D, k in ((8, 100, 64, 0), (300, 5003, 321, 7), (4096, 128256, 4096, 0)):
        s = shape(T, V, D)
        L = P.lib()
        need = [L.fl_head_workspace_bytes(ctypes.byref(s), k, g) for g in (0, 1)]
        assert need[0] > 0 and need[1] > 0
        assert need == [P.head_workspace_bytes(T, V, D, k, g) for g in (False, True)]
        if k == 0:
            assert loss(s, nbytes=need[0] - 1) == loss_grad(s, nbytes=need[1] - 1) == SCRATCH
        else:
            assert distill(s, k=k, nbytes=need[0] - 1) == SCRATCH
            assert distill_grad(s, k=k, nbytes=need[1] - 1) == SCRATCH
    need = P.top_workspace_bytes(4, 100000, 5)
    assert need > 0
    assert top(vocab=100000, nbytes=need - 1) == SCRATCH
    assert top(vocab=100000, ws=None) == INVALID


def test_the_gradient_holds_one_piece_not_the_logits():
    T, V = 4096, 128256
    got = P.head_workspace_bytes(T, V, 4096, grad=True)
    assert got < 2 * T * V, got                        # less than the logits in bf16
    # and does not grow with the vocabulary
    assert P.head_workspace_bytes(T, 4 * V, 4096, grad=True) - got < 16 << 20


def test_rows_that_have_to_be_copied_need_room():
    aligned = P.head_workspace_bytes(8, 1000, 64)
    assert P.head_workspace_bytes(8, 1000, 64, weight_stride=65) >= aligned + 2 * 1000 * 64
    assert P.head_workspace_bytes(8, 1000, 63) >= aligned + 2 * 1000 * 64


def test_binding_refuses_host_tensors_and_wrong_shapes():
    import torch

    b = torch.zeros(4, 8, dtype=torch.bfloat16)
    f, y = torch.zeros(4), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        P.fl_head_loss(b, b, y, f, f, f)
    with pytest.raises(ValueError, match="CUDA"):
        P.fl_head_loss_grad(b, b, y, f, f, f, b, b)
    with pytest.raises(ValueError, match="CUDA"):
        P.fl_head_distill(b, b, y[:, None].int(), f[:, None], None, 1.0, f, f, f[:, None])
    with pytest.raises(ValueError, match="CUDA"):
        P.fl_top_logits(b, 2, 1.0, f, f)
