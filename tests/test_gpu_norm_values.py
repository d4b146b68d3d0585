"""The layer norm and its gradient on rows at the ends of fp32, against the definition in
64 bits, with the tolerances that test_gpu_norm.py derives (they are relative, so they hold
at any scale)."""
import math

import pytest

from test_gpu_embed import U, env  # noqa: F401
from test_gpu_norm import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("R", [5, 530])
@pytest.mark.parametrize("D", [100, 500, 512, 1601, 4100, 8200])
def test_gradient_of_large_rows_without_variance(env, D, R, dtype):  # noqa: F811
    """Rows of one value, 2^100, and eps 2^-60: rstd is 2^30 and y the bias, but mean * rstd
    is no fp32 number, and times 0 no number, where a lane behind the row's end takes its 0
    for a value.  xh is 0, so dx = rstd (c - E(c)), and only the first row adds to dweight."""
    torch, P = env["torch"], env["P"]
    c = Case(torch, R, D, dtype)
    c.x[1:] = 2.0 ** 100
    y, mean, rstd = c.forward(P, 2.0 ** -60)
    assert bool((mean[1:] == 2.0 ** 100).all()) and bool((rstd[1:] == 2.0 ** 30).all())
    assert torch.equal(y[1:], c.b.expand(R - 1, D))
    dx, dw, db = c.grads(P, mean, rstd)
    cc = c.dy.double() * c.w.double()
    m1 = cc.mean(1, keepdim=True)
    want = 2.0 ** 30 * (cc - m1)
    # c rounded once, the mean's sum (102 u of the magnitudes), the subtraction, the
    # product and the rounding to the type
    off = 2.0 ** 30 * (2 * U * cc.abs() + 104 * U * cc.abs().mean(1, keepdim=True) + 2 * U * m1.abs())
    off = off + c.half * (want.abs() + off)
    assert bool(((dx.double() - want).abs() <= off)[1:].all())
    # the other row's part alone
    xh = (c.x[0].double() - mean[0].double()) * rstd[0].double()
    part = c.dy[0].double() * xh
    bound = 4 * U * part.abs()
    assert bool(((dw.double() - part).abs() <= bound + c.half * (part.abs() + bound)).all())
    assert not bool(db.isnan().any())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("D", [7, 500, 1601, 4096, 9000, 20001])
@pytest.mark.parametrize("power,eps", [(62, 1e-5), (100, 1e-5), (122, 1e-5), (-64, 0.0), (-64, 2.0 ** -130),
                                       (-100, 0.0), (-100, 2.0 ** -149), (-100, 2.0 ** -122)])
def test_rows_whose_squares_are_no_numbers(env, power, eps, D, rms, dtype):  # noqa: F811
    """Values whose squares, or whose sum, pass fp32's range or lose bits below it."""
    torch, P = env["torch"], env["P"]
    c = Case(torch, 5, D, dtype, rms, pad=3)
    c.x[1:] *= 2.0 ** power                   # (the first row is an ordinary one)
    c.check_forward(P, eps)
    c.forward = lambda P, e=eps, **kw: Case.forward(c, P, e, **kw)
    c.check_backward(P)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rms", [False, True])
def test_rows_at_the_ends_of_the_range(env, rms, dtype):  # noqa: F811
    """Rows of zeros, of one value, with infinities and with the largest numbers."""
    torch, P = env["torch"], env["P"]
    c = Case(torch, 7, 300, dtype, rms)
    top = torch.finfo(c.dt).max
    c.x[0] = 0.0
    c.x[1, ::2], c.x[1, 1::2] = top, -top     # their mean is 0, and y +-w + b
    c.x[2] = top / 2                          # its sum is no number
    c.x[3] = 0.0
    c.x[3, 5] = top
    c.x[4, 7] = math.inf
    c.x[5, 9] = math.nan
    for eps in (0.0, 1e-5):
        y, mean, rstd = c.forward(P, eps)
        w, b = c.w.double(), c.b.double()
        sign = torch.ones(300, device="cuda", dtype=torch.float64)
        sign[1::2] = -1.0
        for r, want in ((1, sign * w + b),) + (((2, w + b),) if rms else ()):
            off = 200 * U * w.abs() + 2 * U * want.abs()
            assert bool(((y[r].double() - want).abs() <= off + c.half * (want.abs() + off)).all()), r
        assert math.isclose(float(rstd[1]) * float(top), 1.0, rel_tol=2.0 ** -17)   # (subnormal)
        # one value of 300: (1 - 1/300) over the root of (1/300 - 1/300^2), and -1/300
        n = 300.0
        for at, z in ((5, math.sqrt(n) if rms else math.sqrt(n - 1)), (6, 0.0 if rms else -1 / math.sqrt(n - 1))):
            want = z * float(w[at]) + float(b[at])
            off = 200 * U * abs(z * float(w[at])) + 1e-6
            assert abs(float(y[3, at]) - want) <= off + c.half * (abs(want) + off)
        if eps == 0.0:
            assert bool(y[0].isnan().all()) and math.isinf(float(rstd[0]))   # 0 / 0
        else:
            assert torch.equal(y[0], c.b) and abs(float(rstd[0]) * math.sqrt(1e-5) - 1) < 1e-6
        assert bool(y[5].isnan().all()) and bool(y[4, 7].isnan())
        assert bool(y[4].isnan().all()) or rms and torch.equal(y[4, :7], c.b[:7])
        assert not bool(y[6].isnan().any())
