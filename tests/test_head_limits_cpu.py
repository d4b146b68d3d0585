"""Limits of the output head's entry points and what lies just inside them,
without a GPU: a call that passes the checks of its arguments goes on to its
workspace, so a workspace of no bytes shows which check comes first."""
import ctypes

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
