"""A whole local step as examples/local_step.py makes it: embedding, norm, head, their
gradients and AdamW, against the model in 64 bits; the round, and the step captured into a
graph.

The bounds follow each rounding through the step, element by element (half a step of bf16
is H = 2^-8 of a value; what fp32 adds is far below and covered by the factor at the end):
  y    = norm(x):    e_y = H |y|                    (x, scaled, is rounded too: it is taken
                                                     as the call made it)
  z    = y W^T:      e_z = e_y |W|^T;  p = softmax(z) is off by p (exp(2 max e_z) - 1)
  G    = (p - 1)/T:  e_G = that / T + H |G|         (G is rounded to bf16)
  dy   = G W:        e_dy = e_G |W| + H |dy|;   dW = G^T y: e_G^T |y| + (|G| + e_G)^T e_y + H |dW|
  dx   = the norm's: rstd (w e_dy + |xh| mean(w e_dy |xh|)) + H |dx|
  dw   = sum dy xh:  sum e_dy |xh| + H |dw|;   dE = scale * sum dx: scale * sum e_dx + H |dE|
"""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

H = 2.0 ** -8
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "local_step.py")


@pytest.fixture(scope="module")
def ex():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("local_step", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_gradients(ex):
    import torch

    m, (ids, labels) = ex.Model(3, 0), ex.Data(5).batch()
    ids = ids.clone()
    m.gradients(ids, labels)
    V, D, T = ex.V, ex.D, ex.T
    E, w, W = (m.w[k].double() for k in ("embed", "norm", "head"))
    E, W = E.view(V, D), W.view(V, D)
    x = (m.w["embed"].view(V, D)[ids].float() * ex.SCALE).bfloat16()
    assert torch.equal(x, m.x)
    x = x.double()
    rstd = 1 / (x.square().mean(1, keepdim=True) + ex.EPS).sqrt()
    xh = x * rstd
    y = xh * w
    e_y = H * y.abs()
    z = y @ W.t()
    e_z = (e_y @ W.abs().t()).amax(1, keepdim=True)
    p = torch.softmax(z, 1)
    G = (p - torch.nn.functional.one_hot(labels, V)) / T
    e_G = p * torch.expm1(2 * e_z) / T + H * G.abs()
    dy = G @ W
    e_dy = e_G @ W.abs() + H * dy.abs()
    c = dy * w
    dx = rstd * (c - xh * (c * xh).mean(1, keepdim=True))
    e_c = e_dy * w.abs()
    e_dx = rstd * (e_c + xh.abs() * (e_c * xh.abs()).mean(1, keepdim=True)) + H * dx.abs()
    zero = torch.zeros(V, D, dtype=torch.float64, device="cuda")
    want = dict(head=G.t() @ y, norm=(dy * xh).sum(0),
                embed=zero.index_add(0, ids, dx) * ex.SCALE)
    off = dict(head=e_G.t() @ y.abs() + (G.abs() + e_G).t() @ e_y, norm=(e_dy * xh.abs()).sum(0),
               embed=zero.index_add(0, ids, e_dx) * ex.SCALE)
    loss = torch.logsumexp(z, 1) - z.gather(1, labels[:, None])[:, 0]
    assert bool(((m.loss.double() - loss).abs() <= 2.1 * e_z[:, 0] + 1e-5).all())
    for k in want:
        got = m.g[k].double().view(want[k].shape)
        bound = (off[k] + H * (want[k].abs() + off[k])) * 1.02 + 1e-9
        assert bool(((got - want[k]).abs() <= bound).all()), k
        # and the bound says something
        assert float(bound.norm()) < 0.5 * float(want[k].norm()), k


def test_gradients_are_differences_of_the_loss(ex):
    """Along random directions of each parameter: the model's loss in 64 bits, whose
    gradient the step's is off from by no more than the bound above, here by 1/2 in norm."""
    import torch

    m, (ids, labels) = ex.Model(3, 0), ex.Data(6).batch()
    m.gradients(ids, labels)
    w = {k: m.w[k].double() for k in ex.SIZES}

    def loss(w):
        x = w["embed"].view(ex.V, ex.D)[ids] * ex.SCALE
        y = x / (x.square().mean(1, keepdim=True) + ex.EPS).sqrt() * w["norm"]
        z = y @ w["head"].view(ex.V, ex.D).t()
        return (torch.logsumexp(z, 1) - z.gather(1, labels[:, None])[:, 0]).mean()

    for k in ex.SIZES:
        g = m.g[k].double()
        v = g / g.norm()           # along the gradient itself: its norm
        h = 1e-3 / float(v.abs().max()) * 1e-2
        up, down = dict(w, **{k: w[k] + h * v}), dict(w, **{k: w[k] - h * v})
        slope = float((loss(up) - loss(down)) / (2 * h))
        assert abs(slope - float(g.norm())) <= 0.5 * float(g.norm()), k


def test_the_step_is_the_flat_one(ex):
    """Moments in 8 bits of a first step: the masters are fl_adamw_step's of the same
    gradients, as all moments are 0 before it."""
    import torch

    P = ex.P
    m, (ids, labels) = ex.Model(3, 7), ex.Data(5).batch()
    master = m.master.clone()
    m.step(ids, labels, 1)
    mm, v = torch.zeros_like(master), torch.zeros_like(master)
    working = torch.empty_like(m.working)
    P.fl_adamw_step(m.layout, ex.HP, 1, m.grad.float(), master, mm, v, working)
    assert torch.equal(master, m.master) and torch.equal(working, m.working)


def test_round(ex):
    """The example runs, its groups end alike, and again with the same bits."""
    import torch

    a, b = ex.run(), ex.run()
    assert torch.equal(a["models"][0], a["models"][1])
    for k in ("models", "masters", "states"):
        assert all(torch.equal(x, y) for x, y in zip(a[k], b[k])), k
    assert a["first"] == b["first"] and a["last"] == b["last"]
    assert all(x == x and abs(x) < 1e3 for x in a["first"] + a["last"])


def test_step_in_a_graph(ex):
    """The gradients and the step captured, replayed with new tokens in the same places,
    against a model that runs eagerly between the replays."""
    import torch

    m, e, data = ex.Model(3, 7), ex.Model(3, 7), ex.Data(9)
    ids, labels = data.batch()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.gradients(ids, labels)
        ex.P.fl_adamw_tensors(m.tensors, ex.HP, 2, m.g.values(), m.state, seed=m.seed)
    for _ in range(5):
        new = data.batch()
        ids.copy_(new[0])
        labels.copy_(new[1])
        graph.replay()
        e.gradients(*new)
        ex.P.fl_adamw_tensors(e.tensors, ex.HP, 2, e.g.values(), e.state, seed=e.seed)
        torch.cuda.synchronize()
        assert torch.equal(m.grad, e.grad) and torch.equal(m.state, e.state)
        assert torch.equal(m.master, e.master) and torch.equal(m.working, e.working)


def bounds(ex, m, ids, labels):
    """What each element of the gradients may be off by: the errors at the top of this file
    (x is exact here, as the scale is a power of two)."""
    import torch

    V, D, T = ex.V, ex.D, ex.T
    w, W = m.w["norm"].double(), m.w["head"].double().view(V, D)
    x = m.x.double()
    rstd = 1 / (x.square().mean(1, keepdim=True) + ex.EPS).sqrt()
    xh = x * rstd
    y = xh * w
    e_y = H * y.abs()
    z = y @ W.t()
    e_z = (e_y @ W.abs().t()).amax(1, keepdim=True)
    p = torch.softmax(z, 1)
    G = (p - torch.nn.functional.one_hot(labels, V)) / T
    e_G = p * torch.expm1(2 * e_z) / T + H * G.abs()
    dy = G @ W
    e_dy = e_G @ W.abs() + H * dy.abs()
    e_c = e_dy * w.abs()
    c = dy * w
    dx = rstd * (c - xh * (c * xh).mean(1, keepdim=True))
    e_dx = rstd * (e_c + xh.abs() * (e_c * xh.abs()).mean(1, keepdim=True)) + H * dx.abs()
    zero = torch.zeros(V, D, dtype=torch.float64, device="cuda")
    off = dict(head=e_G.t() @ y.abs() + (G.abs() + e_G).t() @ e_y, norm=(e_dy * xh.abs()).sum(0),
               embed=zero.index_add(0, ids, e_dx) * ex.SCALE)
    return {k: (off[k].flatten() + H * (m.g[k].double().abs() + off[k].flatten())) * 1.02 for k in off}


def test_slopes_within_the_roundings(ex):
    """Differences of the model's loss in 64 bits along each parameter's gradient and along
    its signs: off from the step's gradient by no more than its elements may be, and by
    1e-4 of it for the differences themselves (h moves a parameter by 1e-5 at most, so that
    h^2 times a third derivative is far below).  Along the gradient that is about 1, 19 and
    6 % for the head, the norm and the embedding."""
    import torch

    m, (ids, labels) = ex.Model(3, 0), ex.Data(6).batch()
    m.gradients(ids, labels)
    w, off = {k: m.w[k].double() for k in ex.SIZES}, bounds(ex, m, ids, labels)
    most = dict(head=0.03, norm=0.25, embed=0.1)

    def loss(w):
        x = w["embed"].view(ex.V, ex.D)[ids] * ex.SCALE
        y = x / (x.square().mean(1, keepdim=True) + ex.EPS).sqrt() * w["norm"]
        z = y @ w["head"].view(ex.V, ex.D).t()
        return (torch.logsumexp(z, 1) - z.gather(1, labels[:, None])[:, 0]).mean()

    for k in ex.SIZES:
        g = m.g[k].double()
        for v in (g / g.norm(), torch.sign(g) / g.numel() ** 0.5):
            h = 1e-5 / float(v.abs().max())
            up, down = dict(w, **{k: w[k] + h * v}), dict(w, **{k: w[k] - h * v})
            slope, want = float((loss(up) - loss(down)) / (2 * h)), float((g * v).sum())
            may = float((off[k] * v.abs()).sum())
            assert abs(slope - want) <= may + 1e-4 * want, k
        v = g / g.norm()
        assert float((off[k] * v.abs()).sum()) <= most[k] * float(g.norm()), k   # it says something
