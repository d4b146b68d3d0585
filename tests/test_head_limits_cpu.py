"""Limits of the output head's entry points and what lies just inside them,
without a GPU: a call that passes the checks of its arguments goes on to its
workspace, so a workspace of no bytes shows which check comes first."""
import ctypes

import pytest

import paper_2609_20359_amd as P
from paper_2609_20359_amd import flround as F

INVALID, ALIGN, SCRATCH = F.FL_ERR_INVALID, F.FL_ERR_ALIGN, F.FL_ERR_SCRATCH
A = 1 << 20   # an address that is aligned to anything; never dereferenced


def calls(s, weight=2 * A, k=4, nbytes=0, tau=1.0):
    """The status of each of the head's four calls with a workspace of nbytes."""
    L, s = P.lib(), ctypes.byref(s)
    return [L.fl_head_loss(s, A, weight, A, A, A, A, A, nbytes, None),
            L.fl_head_loss_grad(s, A, weight, A, A, A, A, 3 * A, 4 * A, A, nbytes, None),
            L.fl_head_distill(s, A, weight, k, A, A, None, tau, A, A, A, A, nbytes, None),
            L.fl_head_distill_grad(s, A, weight, k, A, A, None, tau, A, A, A, 3 * A, 4 * A, A, nbytes,
                                   None)]


def test_weight_rows_that_are_copied_may_start_anywhere():
    for T, V, D, ldw in ((8, 100, 63, 0), (8, 100, 64, 65), (8, 100, 65, 72)):
        s = F.HeadShape(T, V, D, 0, ldw)
        assert calls(s, weight=2 * A + 2) == [SCRATCH] * 4
        assert calls(s, weight=2 * A + 1) == [ALIGN] * 4
    for D, ldw in ((64, 0), (64, 72)):    # these are read as they are
        assert calls(F.HeadShape(8, 100, D, 0, ldw), weight=2 * A + 2) == [ALIGN] * 4


def test_hidden_rows_may_be_far_apart():
    """One row of each of many long sequences: only the weight's rows are held to
    32 bits of bytes a tile."""
    for ld in ((1 << 22) + 8, 131072 * 4096, 1 << 40):
        assert calls(F.HeadShape(8, 100, 64, ld, 0)) == [SCRATCH] * 4
    assert calls(F.HeadShape(8, 100, 64, (1 << 40) + 1, 0)) == [INVALID] * 4
    assert calls(F.HeadShape(8, 100, 64, 0, 1 << 22)) == [SCRATCH] * 4
    assert calls(F.HeadShape(8, 100, 64, 0, (1 << 22) + 8)) == [INVALID] * 4


def test_temperatures_whose_reciprocal_overflows():
    """The kernels scale by log2(e) / tau: where that is not finite in 32 bits no
    result would be."""
    top = P.lib().fl_top_logits
    s = F.HeadShape(8, 100, 64, 0, 0)
    for tau in (2.0 ** -149, 2.0 ** -128):
        assert calls(s, tau=tau)[2:] == [INVALID] * 2
        assert top(4, 100000, 0, F.FL_BF16, A, 5, tau, A, A, A, A, 0, None) == INVALID
    for tau in (2.0 ** -127, 2.0 ** -126, 1e-30, 3e38):
        assert calls(s, tau=tau)[2:] == [SCRATCH] * 2
        assert top(4, 100000, 0, F.FL_BF16, A, 5, tau, A, A, A, A, 0, None) == SCRATCH


def test_both_sides_of_the_limits():
    L = P.lib()
    K, V, D = F.FL_MAX_TARGETS, 1 << 21, 1 << 15
    T = 1 << 20
    inside = [(T, 100, 64), (T - 1, 65536, 64), (T, 65536, 64), (T, 65536, D), (256, V, 64), (256, V - 1, D),
              (8, 100, D), (8, 100, D - 1), (8, V, D), (0, V, D), (32, V, D), (33, V, 65), (1, 1, 1)]
    outside = [(T + 1, 100, 64), (8, V + 1, 64), (8, 100, D + 1), (T, 65537, 64), (T - 127, 65537, 64),
               (262145, V, 64)]
    for t, v, d in inside:
        s = F.HeadShape(t, v, d, 0, 0)
        assert calls(s, k=K) == [SCRATCH] * 4, (t, v, d)
        for k in (0, 1, K):
            forward = L.fl_head_workspace_bytes(ctypes.byref(s), k, 0)
            grad = L.fl_head_workspace_bytes(ctypes.byref(s), k, 1)
            copied = 2 * v * d if d % 8 else 0      # the weight's rows
            listed = 4 * t * k                      # the teacher's probabilities
            # statistics of each word tile; G of 8192 words, or all, and a row of sums per token
            assert forward >= 2 * t * d + copied + listed + 8 * t * (v // 256), (t, v, d, k)
            assert grad >= 2 * t * d + copied + listed + 2 * t * min(v, 8192) + 4 * t * d, (t, v, d, k)
            assert max(forward, grad) < 1 << 42, (t, v, d, k)
    for t, v, d in outside:
        s = F.HeadShape(t, v, d, 0, 0)
        assert calls(s, k=K) == [INVALID] * 4, (t, v, d)
        assert L.fl_head_workspace_bytes(ctypes.byref(s), 0, 0) == 0
        assert L.fl_head_workspace_bytes(ctypes.byref(s), K, 1) == 0
    s = F.HeadShape(8, 200, 64, 0, 0)
    assert calls(s, k=K)[2:] == [SCRATCH] * 2 and calls(s, k=K + 1)[2:] == [INVALID] * 2
    assert L.fl_head_workspace_bytes(ctypes.byref(s), K + 1, 0) == 0
    assert L.fl_head_workspace_bytes(ctypes.byref(s), -1, 0) == 0


def test_both_sides_of_the_limits_of_top_logits():
    L = P.lib()

    def top(rows, vocab, k, dtype):
        return L.fl_top_logits(rows, vocab, 0, dtype, A, k, 1.0, A, A, A, A, 0, None)

    for dtype in (F.FL_BF16, F.FL_F32):
        for rows, vocab, k in ((1 << 20, 1 << 20, 128), (1, 1 << 20, 128), (1 << 20, 50000, 1),
                               (4, 100000, 128)):
            need = L.fl_top_workspace_bytes(rows, vocab, dtype, k)
            # where a row is cut, an entry for each of k of each segment, two at least
            assert need == 0 or need >= 2 * rows * 8 * k, (rows, vocab, k)
            if need:
                assert top(rows, vocab, k, dtype) == SCRATCH
        for rows, vocab, k in (((1 << 20) + 1, 100, 1), (4, (1 << 20) + 1, 1), (4, 1000, 129), (4, 127, 128),
                               (4, 128, 0)):
            assert L.fl_top_workspace_bytes(rows, vocab, dtype, k) == 0
            assert top(rows, vocab, k, dtype) == INVALID
        assert L.fl_top_workspace_bytes(1, 1 << 20, dtype, 128) > 0


def test_binding_refuses_listed_words_that_are_no_matrix():
    import torch

    b, f = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4)
    for ids in (torch.tensor(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32),
                torch.zeros(4, 2, 1, dtype=torch.int32)):
        with pytest.raises(ValueError, match="2-D"):
            P.fl_head_distill(b, b, ids, f, None, 1.0, f, f, f)
        with pytest.raises(ValueError, match="2-D"):
            P.fl_head_distill_grad(b, b, ids, f, None, 1.0, f, f, f, b, b)
