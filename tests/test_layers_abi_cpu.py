"""Refusals and limits of the embedding's and the layer norm's entry points, without a
GPU: every argument is checked before anything is enqueued.  The gradients check their
workspace last, so one of no bytes shows that the other checks were passed."""
import ctypes
import math

import pytest

import paper_2609_20359_amd as P
from paper_2609_20359_amd import flround as F

INVALID, ALIGN, SCRATCH = F.FL_ERR_INVALID, F.FL_ERR_ALIGN, F.FL_ERR_SCRATCH
A = 1 << 20   # an address that is aligned to anything; never dereferenced


def embed(s, ids=A, weight=2 * A, scale=1.0, out=3 * A):
    return P.lib().fl_embed(ctypes.byref(s), ids, weight, scale, out, None)


def embed_grad(s, ids=A, dout=2 * A, scale=1.0, add=0, dw=3 * A, ws=4 * A, nbytes=0):
    return P.lib().fl_embed_grad(ctypes.byref(s), ids, dout, scale, add, dw, ws, nbytes, None)


def norm(s, x=A, w=2 * A, b=3 * A, eps=1e-5, y=4 * A, mean=5 * A, rstd=6 * A):
    return P.lib().fl_layer_norm(ctypes.byref(s), x, w, b, eps, y, mean, rstd, None)


def norm_grad(s, x=A, w=2 * A, mean=3 * A, rstd=4 * A, dy=5 * A, dx=6 * A, dw=7 * A, db=8 * A,
              ws=9 * A, nbytes=0):
    return P.lib().fl_layer_norm_grad(ctypes.byref(s), x, w, mean, rstd, dy, dx, dw, db, ws, nbytes,
                                      None)


def eshape(T=8, V=100, D=64, ld=0, dtype=0):
    return F.EmbedShape(T, V, D, ld, dtype)


def nshape(R=8, D=64, ldx=0, ldy=0, dtype=0, rms=0):
    return F.NormShape(R, D, ldx, ldy, dtype, rms)


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(T=(1 << 20) + 1), dict(V=0), dict(V=-3), dict(V=(1 << 21) + 1), dict(D=0),
    dict(D=(1 << 15) + 1), dict(ld=63), dict(ld=-64), dict(ld=(1 << 40) + 1), dict(dtype=2),
    dict(dtype=-1)])
def test_embedding_shapes(bad):
    s = eshape(**bad)
    assert embed(s) == embed_grad(s) == INVALID
    assert P.lib().fl_embed_workspace_bytes(ctypes.byref(s)) == 0


@pytest.mark.parametrize("bad", [
    dict(R=-1), dict(R=(1 << 20) + 1), dict(D=0), dict(D=(1 << 15) + 1), dict(ldx=63), dict(ldy=63),
    dict(ldx=-64), dict(ldy=(1 << 40) + 1), dict(dtype=2)])
def test_norm_shapes(bad):
    s = nshape(**bad)
    assert norm(s) == norm_grad(s) == INVALID
    assert P.lib().fl_layer_norm_workspace_bytes(ctypes.byref(s)) == 0


def test_no_shape():
    L = P.lib()
    assert L.fl_embed(None, A, A, 1.0, A, None) == INVALID
    assert L.fl_embed_grad(None, A, A, 1.0, 0, A, A, 1 << 40, None) == INVALID
    assert L.fl_layer_norm(None, A, A, A, 1e-5, A, A, A, None) == INVALID
    assert L.fl_layer_norm_grad(None, A, A, A, A, A, A, A, A, A, 1 << 40, None) == INVALID
    assert L.fl_embed_workspace_bytes(None) == L.fl_layer_norm_workspace_bytes(None) == 0


def test_largest_shapes_pass():
    for s in (eshape(T=1 << 20, V=1 << 21, D=1 << 15, ld=1 << 40), eshape(dtype=1), eshape(T=0),
              eshape(T=1, V=1, D=1)):
        assert embed_grad(s) == SCRATCH
        assert P.lib().fl_embed_workspace_bytes(ctypes.byref(s)) > 0
    for s in (nshape(R=1 << 20, D=1 << 15, ldx=1 << 40, ldy=1 << 40), nshape(dtype=1, rms=1),
              nshape(R=0), nshape(R=1, D=1)):
        assert norm_grad(s) == SCRATCH
        assert P.lib().fl_layer_norm_workspace_bytes(ctypes.byref(s)) > 0
    # one byte less than what is asked for
    s = eshape()
    assert embed_grad(s, nbytes=P.lib().fl_embed_workspace_bytes(ctypes.byref(s)) - 1) == SCRATCH
    s = nshape()
    assert norm_grad(s, nbytes=P.lib().fl_layer_norm_workspace_bytes(ctypes.byref(s)) - 1) == SCRATCH


def test_pointers():
    s = eshape()
    for name in ("ids", "weight", "out"):
        assert embed(s, **{name: None}) == INVALID, name
    for name in ("ids", "dout", "dw", "ws"):
        assert embed_grad(s, **{name: None}) == INVALID, name
    assert embed(s, ids=A + 4) == embed(s, weight=A + 1) == embed(s, out=A + 1) == ALIGN
    assert embed_grad(s, ids=A + 4) == embed_grad(s, dout=A + 1) == embed_grad(s, dw=A + 1) == ALIGN
    assert embed_grad(s, dout=A + 2, dw=3 * A + 2, ws=4 * A + 1) == SCRATCH
    f = eshape(dtype=1)
    assert embed(f, weight=A + 2) == embed_grad(f, dw=A + 2) == ALIGN
    s = nshape()
    for name in ("x", "y", "rstd"):
        assert norm(s, **{name: None}) == INVALID, name
    for name in ("x", "mean", "rstd", "dy", "dx", "ws"):
        assert norm_grad(s, **{name: None}) == INVALID, name
    for name in ("w", "dw", "db"):
        assert norm_grad(s, **{name: None}) == SCRATCH, name
    assert norm_grad(nshape(rms=1), mean=None) == SCRATCH
    for name in ("x", "w", "b", "y"):
        assert norm(s, **{name: 7 * A + 1}) == ALIGN, name
    for name in ("mean", "rstd"):
        assert norm(s, **{name: 7 * A + 2}) == norm_grad(s, **{name: 7 * A + 2}) == ALIGN, name
    assert norm(nshape(dtype=1), w=7 * A + 2) == norm_grad(nshape(dtype=1), dx=10 * A + 2) == ALIGN


def test_values():
    s = eshape()
    for x in (math.nan, math.inf, -math.inf):
        assert embed(s, scale=x) == embed_grad(s, scale=x) == INVALID
    for x in (math.nan, math.inf, -1e-9):
        assert norm(nshape(), eps=x) == INVALID


def test_outputs_that_are_inputs():
    assert embed(eshape(), out=2 * A) == embed_grad(eshape(), dw=2 * A) == INVALID
    s = nshape()
    assert norm(s, y=A) == norm(s, y=2 * A) == norm(s, y=3 * A) == INVALID
    for name in ("dx", "dw", "db"):
        for at in (1, 2, 5):
            assert norm_grad(s, **{name: at * A}) == INVALID, (name, at)
    assert norm_grad(s, dw=6 * A) == norm_grad(s, db=6 * A) == norm_grad(s, db=7 * A) == INVALID


def test_nothing_to_do():
    """No tokens, no rows: the arrays that are empty may be absent, and a forward call
    reaches no device."""
    assert embed(eshape(T=0), ids=None, out=None) == F.FL_OK
    assert norm(nshape(R=0), x=None, y=None, mean=None, rstd=None) == F.FL_OK


def test_binding_refuses_cpu_tensors():
    import torch

    ids, w = torch.zeros(4, dtype=torch.int64), torch.zeros(10, 8)
    with pytest.raises(ValueError):
        P.fl_embed(ids, w, torch.zeros(4, 8))
    with pytest.raises(ValueError):
        P.fl_embed_grad(ids, torch.zeros(4, 8), w)
    with pytest.raises(ValueError):
        P.fl_layer_norm(w, None, None, 1e-5, w.clone(), None, torch.zeros(10))
    with pytest.raises(ValueError):
        P.fl_layer_norm_grad(w, None, None, torch.zeros(10), w.clone(), w.clone(), None, None,
                             rms=True)


def test_calls_of_one_launch_need_no_workspace():
    """Up to 512 tokens, or rows of up to 8192 bf16 or 4096 fp32 elements; more need theirs."""
    L = P.lib()
    for T, V, D in ((0, 100, 64), (1, 1 << 21, 1 << 15), (512, 5003, 1 << 15)):
        for dtype in (F.FL_BF16, F.FL_F32):
            assert L.fl_embed_workspace_bytes(ctypes.byref(eshape(T, V, D, 0, dtype))) == 256
    assert L.fl_embed_workspace_bytes(ctypes.byref(eshape(513, 5003, 64))) > 4 * 5004 + 8 * 513
    for R, D, dtype, few in ((0, 64, 0, True), (1, 64, 0, True), (512, 8192, 0, True), (512, 8193, 0, False),
                             (513, 64, 0, False), (512, 4096, 1, True), (512, 4097, 1, False)):
        n = L.fl_layer_norm_workspace_bytes(ctypes.byref(nshape(R, D, dtype=dtype)))
        assert n == 256 if few else n > 8 * D, (R, D, dtype)
