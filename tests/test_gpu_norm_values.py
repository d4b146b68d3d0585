"""The layer norm and its gradient on rows at the ends of fp32, against the definition in
64 bits, with the tolerances that test_gpu_norm.py derives (they are relative, so they hold
at any scale)."""
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
