"""The output head and the top logits at values where arithmetic in 32 bits
could go wrong: logits past 2^30, masks of the types' lowest values, infinities,
teachers at the ends of the range; and calls that follow another call's error.

Tolerances (u = 2^-24), with logits that are exact in fp32 (one product, or a
power of two times a bf16 number):
  lse:  its own rounding and that of m / tau and of the sum's logarithm, 4 u |lse|,
        and 2^-16 for the exponentials' and the additions' errors.
  loss: the difference in 64 bits of what lse is before its rounding and the
        target, so 2^-16 and its own rounding, 2^-22 |loss|.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_20359_amd as P

    P.lib()
    return dict(torch=torch, P=P)


def same(torch, what, got, want, off):
    """got against want in 64 bits: within off where want is finite in fp32,
    and the same infinity or NaN where it is not."""
    rounded = want.float().double()
    got = got.double()
    bad = torch.where(torch.isfinite(rounded), ~((got - want).abs() <= off),
                      ~((got == rounded) | (got.isnan() & rounded.isnan())))
    i = [tuple(x) for x in bad.nonzero().tolist()[:4]]
    assert not i, (what, int(bad.sum()), [(k, float(got[k]), float(want[k])) for k in i])


# ---- top logits ----------------------------------------------------------------


def top(P, torch, x, k, tau):
    n = x.shape[0]
    v, s = torch.full((n, k), -7.0, device="cuda"), torch.full((n,), -7.0, device="cuda")
    i = torch.full((n, k), -7, dtype=torch.int32, device="cuda")
    P.fl_top_logits(x, k, tau, v, i, s)
    return v, i, s


def check_top(P, torch, x, k, tau):
    v, i, s = top(P, torch, x, k, tau)
    want, at = torch.sort(x.double() + 0.0, dim=1, descending=True, stable=True)
    assert torch.equal(i.long(), at[:, :k])
    assert torch.equal(v.double().nan_to_num(nan=1e300), want[:, :k].nan_to_num(nan=1e300))
    lse = torch.logsumexp(x.double() / tau, 1)
    same(torch, "lse", s, lse, 2.0 ** -16 + 4 * U * lse.abs())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0, 3.7])
def test_top_lse_of_rows_far_from_zero(env, tau, dtype):
    """Rows masked whole by a large negative number, the type's lowest among
    them, and rows of large positive ones: their lse is their maximum over tau,
    and the logarithm of how many there are."""
    torch, P = env["torch"], env["P"]
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    fills = [torch.finfo(dt).min, -1e38, -1e30, -1e12, -1e9, -1e4, 1e9, 1e12, 1e30, 1e38,
             torch.finfo(dt).max]
    for vocab in (5, 700, 40001):     # a segment that is not full, a full one, several
        x = torch.tensor(fills, device="cuda", dtype=dt)[:, None].repeat(1, vocab)
        check_top(P, torch, x, 3, tau)
        x[:, vocab // 2:] *= 0.5
        check_top(P, torch, x, 3, tau)
        x[:, 1] = -math.inf
        x[:, 2] = torch.finfo(dt).min
        check_top(P, torch, x, 3, tau)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [6, 700, 40001])
def test_top_lse_of_rows_with_infinities(env, vocab, dtype):
    """+inf among the logits gives +inf, NaN gives NaN beside anything, and a
    row of -inf alone gives -inf."""
    torch, P = env["torch"], env["P"]
    g = torch.Generator(device="cuda")
    g.manual_seed(vocab)
    x = torch.randn(8, vocab, generator=g, device="cuda").to(
        torch.bfloat16 if dtype == "bf16" else torch.float32)
    x[0, vocab - 1] = math.inf
    x[1, 0] = x[1, vocab // 2] = x[1, vocab - 2] = math.inf
    x[2] = math.inf
    x[3] = -math.inf
    x[3, 4] = math.inf
    x[4, 1], x[4, vocab - 1] = math.inf, math.nan
    x[5, 3] = math.nan
    x[6] = -math.inf
    x[7, ::2] = -math.inf
    for tau in (1.0, 2.0):
        check_top(P, torch, x, 4, tau)
