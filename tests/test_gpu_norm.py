"""The layer norm and its gradient on the GPU against their definition in 64 bits.

Tolerances (u = 2^-24).  A row's sums have at most 64 terms one after the other in a
lane, 7 steps of a wave and 16 waves: off by at most S = 96 u of the sum of magnitudes.
  mean:  S E|x| + 2 u |mean|  (call it m)
  rstd:  q = E(d^2) is off by 2 m E|d| + m^2 + (S + 6 u) q, so 1 / sqrt(q + eps) is off
         by half of that over q + eps, and 4 u of its own roundings, relative (call it r)
  y:     |w| rstd (m + 2 u |d|) + |d rstd w| (r + 4 u) + 2 u |y|, and half a step of its type
  dx:    xh is off by 3 u, c by u, relative; the means by S + 6 u of those of magnitudes;
         the sum's terms by 3 u more each; half a step
  dw:    a sum over R rows in fp32 of terms off by 4 u, relative, (R + 40) u of the sum of
         magnitudes; half a step
"""
import math

import pytest

from test_gpu_embed import HALF_STEP, U, dtype_of, env, framed  # noqa: F401

pytestmark = pytest.mark.gpu

S = 96 * U
EPS = 1e-5


class Case:
    def __init__(self, torch, R, D, dtype, rms=False, weight=True, bias=True, pad=0, off=0, seed=0,
                 at=0.3):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 1000 * R + D)
        dt = dtype_of(torch, dtype)
        self.torch, self.R, self.D, self.rms, self.dt = torch, R, D, rms, dt
        self.half = HALF_STEP[dtype]

        def rows(scale, shift):
            n = R * (D + pad) + off
            flat = (torch.randn(n, generator=g, device="cuda") * scale + shift).to(dt)
            return flat[off:].view(R, D + pad)[:, :D]

        self.x, self.dy = rows(1.5, at), rows(0.1, 0.01)
        self.w = (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dt) if weight else None
        self.b = torch.randn(D, generator=g, device="cuda").to(dt) if bias else None

    def forward(self, P, eps=EPS, **kw):
        torch, R, D = self.torch, self.R, self.D
        y, self.untouched = framed(torch, (R, D), self.dt, off=1)
        mean = torch.full((R,), -7.0, device="cuda")
        rstd = torch.full((R,), -7.0, device="cuda")
        P.fl_layer_norm(self.x, self.w, self.b, eps, y, mean, rstd, rms=self.rms, **kw)
        return y, mean, rstd

    def check_forward(self, P, eps=EPS):
        y, mean, rstd = self.forward(P, eps)
        x = self.x.double()
        w = self.w.double() if self.w is not None else 1.0
        b = self.b.double() if self.b is not None else 0.0
        mu = x.mean(1, keepdim=True) * (0.0 if self.rms else 1.0)
        m = (S * x.abs().mean(1, keepdim=True) + 2 * U * mu.abs()) * (0.0 if self.rms else 1.0)
        d = x - mu
        q = d.square().mean(1, keepdim=True)
        qo = 2 * m * d.abs().mean(1, keepdim=True) + m * m + (S + 6 * U) * q
        r = 0.5 * qo / (q + eps) * 1.01 + 4 * U
        rs = 1.0 / (q + eps).sqrt()
        yy = d * rs * w
        off = (m + 2 * U * d.abs()) * rs * abs(w) + yy.abs() * (r + 4 * U) + 2 * U * (yy + b).abs()
        want = yy + b
        off = off * 1.01 + self.half * (want.abs() + off) + 1e-37
        assert not bool(y.isnan().any())
        assert bool(((mean.double()[:, None] - mu).abs() <= m + 1e-37).all())
        assert bool(((rstd.double()[:, None] - rs).abs() <= rs * r * 1.01).all())
        bad = (y.double() - want).abs() > off
        assert not bool(bad.any()), int(bad.sum())
        self.untouched()

    def grads(self, P, mean, rstd, dweight=True, dbias=True, **kw):
        torch, R, D = self.torch, self.R, self.D
        dx, c0 = framed(torch, (R, D), self.dt, off=1)
        dw, c1 = framed(torch, (D,), self.dt)
        db, c2 = framed(torch, (D,), self.dt)
        P.fl_layer_norm_grad(self.x, self.w, None if self.rms else mean, rstd, self.dy, dx,
                             dw if dweight else None, db if dbias else None, rms=self.rms, **kw)
        c0(), c1(), c2()
        return dx, dw, db

    def check_backward(self, P, dweight=True, dbias=True):
        R, D = self.R, self.D
        _, mean, rstd = self.forward(P)
        dx, dw, db = self.grads(P, mean, rstd, dweight, dbias)
        x, dy = self.x.double(), self.dy.double()
        w = self.w.double() if self.w is not None else 1.0
        mu = 0.0 if self.rms else mean.double()[:, None]
        rs = rstd.double()[:, None]
        xh, c = (x - mu) * rs, dy * w
        E = lambda t: t.mean(1, keepdim=True)  # noqa: E731
        m0, m1 = E(c * xh), 0.0 if self.rms else E(c)
        want = rs * (c - m1 - xh * m0)
        o0, o1 = (S + 12 * U) * E((c * xh).abs()), 0.0 if self.rms else (S + 6 * U) * E(c.abs())
        off = rs * (8 * U * (c.abs() + abs(m1) + (xh * m0).abs()) + o1 + xh.abs() * o0) * 1.01
        off = off + self.half * (want.abs() + off) + 1e-37
        bad = (dx.double() - want).abs() > off
        assert not bool(bad.any()) and not bool(dx.isnan().any()), int(bad.sum())
        for ok, got, term in ((dweight, dw, dy * xh), (dbias, db, dy)):
            if not ok:
                assert bool((got == -7.0).all())
                continue
            want, size = term.sum(0), term.abs().sum(0)
            off = (R + 40) * U * size
            off = off + self.half * (want.abs() + off) + 1e-37
            bad = (got.double() - want).abs() > off
            assert not bool(bad.any()) and not bool(got.isnan().any()), int(bad.sum())


WIDTHS = [1, 2, 7, 8, 9, 63, 64, 255, 321, 512, 513, 1024, 1601, 2048, 2049, 4096, 4100, 8192, 8193,
          16384, 20001, 32768]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("D", WIDTHS)
def test_widths(env, D, rms, dtype):  # noqa: F811
    for R, pad, off in ((1, 0, 0), (5, 3, 1), (130, 8, 0), (530, 0, 2)):
        c = Case(env["torch"], R, D, dtype, rms, pad=pad, off=off)
        c.check_forward(env["P"])
        c.check_backward(env["P"])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("R,D", [(2, 100), (700, 64), (1029, 768), (3000, 1000), (5000, 24),
                                 (2050, 2560), (512, 500), (513, 500), (512, 4096),
                                 (1500, 40), (1300, 9000), (1100, 1), (16, 63), (17, 65)])
def test_rows(env, R, D, dtype):  # noqa: F811
    c = Case(env["torch"], R, D, dtype)
    c.check_forward(env["P"])
    c.check_backward(env["P"])


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
def test_without_weight_or_bias(env, weight, bias, rms):  # noqa: F811
    for D in (300, 4500):
        c = Case(env["torch"], 40, D, "fp32", rms, weight, bias)
        c.check_forward(env["P"])
        c.check_backward(env["P"], dweight=weight, dbias=bias)


def test_far_from_zero(env):  # noqa: F811
    """A mean a thousand times the spread: the variance is taken about the mean."""
    for D in (768, 5000):
        c = Case(env["torch"], 33, D, "fp32", at=1500.0)
        c.check_forward(env["P"])
        c.check_backward(env["P"])


def test_constant_rows_and_special_values(env):  # noqa: F811
    torch, P = env["torch"], env["P"]
    c = Case(torch, 6, 200, "fp32")
    c.x[1] = 2.5                               # no variance: y is the bias
    c.x[2, 7] = math.nan
    c.x[3, 9] = math.inf
    c.x[4] = 0.0
    y, mean, rstd = c.forward(P)
    assert torch.equal(y[1], c.b) and torch.equal(y[4], c.b)
    assert abs(float(rstd[1]) * math.sqrt(EPS) - 1) < 1e-6
    assert bool(y[2].isnan().all()) and bool(y[3].isnan().all())
    clean = Case(torch, 6, 200, "fp32")
    y0, _, _ = clean.forward(P)
    assert torch.equal(y[0], y0[0]) and torch.equal(y[5], y0[5])
    dx, dw, _ = c.grads(P, mean, rstd)
    assert bool(dx[2].isnan().all()) and not bool(dx[[0, 1, 4, 5]].isnan().any())
    assert bool(dw[7].isnan())


def test_no_rows(env):  # noqa: F811
    torch, P = env["torch"], env["P"]
    c = Case(torch, 0, 100, "bf16")
    c.forward(P)
    _, dw, db = c.grads(P, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"))
    assert not bool(dw.any()) and not bool(db.any())


@pytest.mark.parametrize("rms", [False, True])
def test_difference_of_the_loss(env, rms):  # noqa: F811
    """Gradients against central differences of the definition in 64 bits."""
    torch, P = env["torch"], env["P"]
    c = Case(torch, 12, 90, "fp32", rms)
    _, mean, rstd = c.forward(P)
    dx, dw, db = c.grads(P, mean, rstd)
    x, w, b, dy = (t.double() for t in (c.x, c.w, c.b, c.dy))

    def value(x, w, b):
        mu = 0.0 if rms else x.mean(1, keepdim=True)
        d = x - mu
        return (dy * (d / (d.square().mean(1, keepdim=True) + EPS).sqrt() * w + b)).sum()

    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    h = 1e-4
    for k, grad in enumerate((dx, dw, db)):
        args = [x, w, b]
        for _ in range(5):
            v = torch.randn(args[k].shape, generator=g, device="cuda", dtype=torch.float64)
            up, down = list(args), list(args)
            up[k], down[k] = args[k] + h * v, args[k] - h * v
            diff = float((value(*up) - value(*down)) / (2 * h))
            want = float((grad.double() * v).sum())
            size = float((grad.double() * v).abs().sum())
            # h^2 times a third derivative of order one over six, and fp32's roundings
            assert abs(diff - want) <= 1e-6 * size + 1e-6


def test_same_bits_whatever_the_workspace(env):  # noqa: F811
    torch, P = env["torch"], env["P"]
    c = Case(torch, 2000, 640, "bf16")
    _, mean, rstd = c.forward(P)
    first = None
    for off in (0, 1, 17):
        ws = torch.randint(0, 255, (P.layer_norm_workspace_bytes(2000, 640) + off,),
                           dtype=torch.uint8, device="cuda")[off:]
        got = [t.clone() for t in c.grads(P, mean, rstd, workspace=ws)]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_rows_past_32_bits(env):  # noqa: F811
    """Rows 2^22 elements apart: the last one lies past 2^32 elements."""
    torch, P = env["torch"], env["P"]
    R, ld, D = 1030, 1 << 22, 128
    c = Case(torch, R, D, "bf16")
    far = torch.empty(R, ld, dtype=torch.bfloat16, device="cuda")
    far[:, :D] = c.x
    near, c.x = c.x, far[:, :D]
    got = c.forward(P)
    c.x = near
    for a, b in zip(got, c.forward(P)):
        assert torch.equal(a, b)


def test_streams_and_graphs(env):  # noqa: F811
    torch, P = env["torch"], env["P"]
    c = Case(torch, 900, 1200, "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y1, mean, rstd = c.forward(P, stream=side)
    dx1, dw1, db1 = c.grads(P, mean, rstd, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    y0, mean0, rstd0 = c.forward(P)
    assert torch.equal(y0, y1) and torch.equal(mean, mean0) and torch.equal(rstd, rstd0)
    assert all(torch.equal(a, b) for a, b in zip(c.grads(P, mean, rstd), (dx1, dw1, db1)))
    graphs = []
    for _ in range(2):
        ws = torch.empty(P.layer_norm_workspace_bytes(900, 1200), dtype=torch.uint8, device="cuda")
        o = [torch.empty_like(c.x), torch.empty(900, device="cuda"), torch.empty(900, device="cuda"),
             torch.empty_like(c.x), torch.empty_like(c.w), torch.empty_like(c.w)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            P.fl_layer_norm(c.x, c.w, c.b, EPS, o[0], o[1], o[2])
            P.fl_layer_norm_grad(c.x, c.w, o[1], o[2], c.dy, o[3], o[4], o[5], workspace=ws)
        graphs.append((graph, o, ws))
    for turn in range(4):
        c.x.copy_(torch.randn(900, 1200, device="cuda") + turn)
        for graph, o, _ in graphs:
            for t in o:
                t.fill_(-3.0)
            graph.replay()
        y, mean, rstd = c.forward(P)
        want = [y, mean, rstd, *c.grads(P, mean, rstd)]
        torch.cuda.synchronize()
        for _, o, _ in graphs:
            assert all(torch.equal(a, b) for a, b in zip(o, want))


def test_refusals(env):  # noqa: F811
    torch, P = env["torch"], env["P"]
    c = Case(torch, 4, 32, "bf16")
    y, mean, rstd = c.forward(P)
    for args in ((c.x, c.w.float(), c.b, EPS, y, mean, rstd), (c.x, c.w, c.b[:31], EPS, y, mean, rstd),
                 (c.x, c.w, c.b, EPS, y[:3], mean, rstd), (c.x, c.w, c.b, EPS, y, mean.half(), rstd),
                 (c.x.half(), c.w, c.b, EPS, y, mean, rstd), (c.x[0], c.w, c.b, EPS, y, mean, rstd),
                 (c.x.cpu(), c.w, c.b, EPS, y, mean, rstd), (c.x.t(), c.w, c.b, EPS, y, mean, rstd)):
        with pytest.raises(ValueError):
            P.fl_layer_norm(*args)
    dx, dw = torch.empty_like(c.x), torch.empty_like(c.w)
    for kw in (dict(dy=c.dy[:3]), dict(dy=c.dy.float()), dict(dx=dx[:3]), dict(dw=dw.float()),
               dict(rstd=rstd[:3])):
        a = dict(dict(rstd=rstd, dy=c.dy, dx=dx, dw=dw), **kw)
        with pytest.raises(ValueError):
            P.fl_layer_norm_grad(c.x, c.w, mean, a["rstd"], a["dy"], a["dx"], a["dw"], None)
    for call in (lambda: P.fl_layer_norm(c.x, c.w, c.b, -1.0, y, mean, rstd),
                 lambda: P.fl_layer_norm(c.x, c.w, c.b, math.nan, y, mean, rstd),
                 lambda: P.fl_layer_norm(c.x, c.w, c.b, EPS, c.x, mean, rstd),
                 lambda: P.fl_layer_norm_grad(c.x, c.w, None, rstd, c.dy, dx, dw, None),
                 lambda: P.fl_layer_norm_grad(c.x, c.w, mean, rstd, c.dy, c.dy, dw, None),
                 lambda: P.fl_layer_norm_grad(c.x, c.w, mean, rstd, c.dy, dx, dw, dw)):
        with pytest.raises(P.FlError):
            call()
