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
import ctypes
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


# ---- the head's statistics -----------------------------------------------------

# (tokens, words): each of the four tiles of the statistics
TILES = [(5, 300), (40, 300), (100, 500), (256, 66000)]


def forward(P, torch, h, w, labels):
    T = h.shape[0]
    out = [torch.full((T,), -7.0, device="cuda") for _ in range(3)]
    P.fl_head_loss(h, w, labels, *out)
    return out


@pytest.mark.parametrize("T,V", TILES)
def test_logits_far_from_zero(env, T, V):
    """A token's logits are a power of two, up to 2^110 and of both signs, times
    small whole numbers: every one is exact, and so is what is expected."""
    torch, P = env["torch"], env["P"]
    D = 16
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    power = torch.randint(-4, 111, (T,), generator=g, device="cuda").double()
    h = torch.zeros(T, D, device="cuda", dtype=torch.bfloat16)
    sign = torch.randint(0, 2, (T,), generator=g, device="cuda").double() * 2 - 1
    h[:, 0] = (2.0 ** power * sign).bfloat16()
    w = torch.zeros(V, D, device="cuda", dtype=torch.bfloat16)
    w[:, 0] = torch.randint(-100, 101, (V,), generator=g, device="cuda").bfloat16()
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    labels[::2] = torch.where(sign[::2] > 0, w[:, 0].float().argmax(), w[:, 0].float().argmin())
    z = h[:, :1].double() @ w[:, :1].double().t()
    lse = torch.logsumexp(z, 1)
    at = z.gather(1, labels[:, None])[:, 0]
    # (as a difference from the maximum: lse in 64 bits has lost the sum's logarithm)
    m = z.amax(1)
    want = torch.log(torch.exp(z - m[:, None]).sum(1)) + (m - at)
    loss, got, target = forward(P, torch, h, w, labels)
    same(torch, "lse", got, lse, 2.0 ** -16 + 4 * U * lse.abs())
    same(torch, "target", target, at, 0.0 * at)
    # what the kernel's sum in 64 bits holds beside so large a maximum
    same(torch, "loss", loss, want, 2.0 ** -16 + 2.0 ** -22 * want.abs() + 2.0 ** -50 * m.abs())


@pytest.mark.parametrize("T,V", TILES)
def test_infinite_logits(env, T, V):
    """A logit of +inf gives an lse and a loss of +inf, one of -inf is a word of
    no probability, NaN gives NaN."""
    torch, P = env["torch"], env["P"]
    D = 16
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    h = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    h[h == 0] = 1.0
    w = torch.randn(V, D, generator=g, device="cuda").bfloat16()
    w[V - 3, 0] = math.inf
    w[1, 0] = math.inf
    h[3, 1] = math.nan
    labels = torch.randint(2, V - 3, (T,), generator=g, device="cuda")
    # each product by itself, in 64 bits, with the infinite ones put in by sign
    clean = torch.where(torch.isfinite(w), w, 0.0).double()
    z = h.double() @ clean.t()
    for v in (V - 3, 1):
        z[:, v] = torch.where(z[:, v].isnan(), math.nan, h[:, 0].double().sign() * math.inf)
    lse = torch.logsumexp(z, 1)
    at = z.gather(1, labels[:, None])[:, 0]
    z_off = (D + 8) * U * (h.double().abs().nan_to_num(nan=0.0) @ clean.abs().t()).amax(1)
    loss, got, target = forward(P, torch, h, w, labels)
    assert bool(torch.isinf(lse).any()) and bool(torch.isfinite(lse).any())
    off = z_off + 2.0 ** -16
    same(torch, "lse", got, lse, off + 4 * U * lse.abs().nan_to_num(posinf=0.0))
    same(torch, "loss", loss, lse - at, off + z_off + 2.0 ** -22 * (lse - at).abs().nan_to_num(posinf=0.0))


@pytest.mark.parametrize("T,V", [(5, 300), (40, 300), (100, 500), (1030, 16500)])
def test_gradient_of_logits_far_from_zero(env, T, V):
    """Where one logit is far above the others, the softmax is 1 there and 0
    elsewhere, however large the logits are; G and its products are whole
    numbers times the tokens' weight."""
    torch, P = env["torch"], env["P"]
    D = 16
    g = torch.Generator(device="cuda")
    g.manual_seed(T + V)
    h = torch.zeros(T, D, device="cuda", dtype=torch.bfloat16)
    power = torch.randint(0, 100, (T,), generator=g, device="cuda").double()
    h[:, 0] = (2.0 ** power).bfloat16()
    h[:, 1:] = torch.randint(-3, 4, (T, D - 1), generator=g, device="cuda").bfloat16()
    w = torch.zeros(V, D, device="cuda", dtype=torch.bfloat16)
    w[:, 0] = torch.randint(-100, 1, (V,), generator=g, device="cuda").bfloat16() * 4
    best = V // 2
    w[best, 0] = 101.0
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    labels[::3] = best
    loss, lse, target = forward(P, torch, h, w, labels)
    dl = torch.full((T,), 0.25, device="cuda")
    dh = torch.full((T, D), -7.0, device="cuda", dtype=torch.bfloat16)
    dw = torch.full((V, D), -7.0, device="cuda", dtype=torch.bfloat16)
    P.fl_head_loss_grad(h, w, labels, lse, target, dl, dh, dw)
    G = torch.zeros(T, V, device="cuda", dtype=torch.float64)
    G[:, best] = 0.25
    G[torch.arange(T, device="cuda"), labels] -= 0.25
    for what, got, want, size in (("dhidden", dh, G @ w.double(), G.abs() @ w.double().abs()),
                                  ("dweight", dw, G.t() @ h.double(), G.abs().t() @ h.double().abs())):
        # sums in fp32, the results' rounding, and what is left of the other words
        off = 2.0 ** -7.9 * want.abs() + (T + V) * U * size + math.exp(-500.0)
        same(torch, what, got, want, off)


@pytest.mark.parametrize("tau", [2.0 ** -127, 2.0 ** -100, 1e-20, 1e20, 2.0 ** 100])
def test_temperatures_at_both_ends(env, tau):
    """Close to 0 all probability is at the largest logit, far from it all words have
    the same; the results are those, as far as fp32 holds them."""
    torch, P = env["torch"], env["P"]
    T, V, D, K = 40, 300, 16, 3
    tau = float(torch.tensor(tau, dtype=torch.float32))
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    h = torch.zeros(T, D, device="cuda", dtype=torch.bfloat16)
    h[:, 0] = torch.randint(1, 9, (T,), generator=g, device="cuda").bfloat16()
    w = torch.zeros(V, D, device="cuda", dtype=torch.bfloat16)
    w[:, 0] = torch.randint(-60, 60, (V,), generator=g, device="cuda").bfloat16()
    w[17, 0] = 64.0
    z = h.double() @ w.double().t()
    x = z.float()
    values, ids, alse = top(P, torch, x, K, tau)
    want = torch.logsumexp(z / tau, 1)
    same(torch, "teacher's lse", alse, want, 2.0 ** -16 + 4 * U * want.abs())
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    target = torch.empty(T, K, device="cuda")
    dh = torch.empty(T, D, device="cuda", dtype=torch.bfloat16)
    dw = torch.empty(V, D, device="cuda", dtype=torch.bfloat16)
    P.fl_head_distill(h, w, ids, values, None, tau, loss, lse, target)
    same(torch, "lse", lse, want, 2.0 ** -16 + 4 * U * want.abs())
    if not bool(torch.isfinite(lse).all()):
        return                       # 2^-127: the quotient itself overflows
    dl = torch.ones(T, device="cuda")
    P.fl_head_distill_grad(h, w, ids, values, None, tau, lse, target, dl, dh, dw)
    p = torch.zeros(T, V, device="cuda", dtype=torch.float64)
    p.scatter_(1, ids.long(), torch.softmax(values.double() / tau, 1))
    # the softmax of z / tau, from lse as fp32 holds it where that is exact
    soft = torch.softmax(z / tau, 1)
    G = tau * (soft - p)
    # both sides 1 at the same word, or 1 / V and 1 / K; each is off by 2^-8 at most
    off = tau * 2.0 ** -7 * ((soft + p) @ w.double().abs())
    same(torch, "dhidden", dh, G @ w.double(), off)


# ---- the teacher ---------------------------------------------------------------


def teacher_case(torch, P, a, alse, tau):
    """Loss and gradients of len(a) tokens that list the first words."""
    T, K = a.shape
    V, D = 200, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(31)
    h = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    w = (torch.randn(V, D, generator=g, device="cuda") * 0.3).bfloat16()
    ids = torch.arange(K, device="cuda", dtype=torch.int32).repeat(T, 1)
    loss, lse = torch.full((T,), -7.0, device="cuda"), torch.full((T,), -7.0, device="cuda")
    target = torch.full((T, K), -7.0, device="cuda")
    dh = torch.full((T, D), -7.0, device="cuda", dtype=torch.bfloat16)
    dw = torch.full((V, D), -7.0, device="cuda", dtype=torch.bfloat16)
    P.fl_head_distill(h, w, ids, a, alse, tau, loss, lse, target)
    dl = torch.full((T,), 0.25, device="cuda")
    P.fl_head_distill_grad(h, w, ids, a, alse, tau, lse, target, dl, dh, dw)
    z = h.double() @ w.double().t()
    z_off = (D + 8) * U * (h.double().abs() @ w.double().abs().t()).amax(1)
    return dict(h=h, w=w, z=z, z_off=z_off, dl=dl, loss=loss, lse=lse, dh=dh, dw=dw)


@pytest.mark.parametrize("tau", [0.25, 0.5, 1.0, 2.0])
def test_teachers_at_the_ends_of_the_range(env, tau):
    """Teacher logits at fp32's lowest and largest value are finite: a token that
    lists nothing else takes part, with the probabilities of the formula."""
    torch, P = env["torch"], env["P"]
    lo, hi = torch.finfo(torch.float32).min, torch.finfo(torch.float32).max
    a = torch.tensor([[lo, lo, lo, lo], [hi, lo, 0.0, hi], [lo, lo, -math.inf, lo], [hi, hi, hi, hi],
                      [-math.inf, -math.inf, lo, -math.inf], [1.0, 2.0, 3.0, lo]], device="cuda")
    c = teacher_case(torch, P, a, None, tau)
    x = (a.double() - a.double().amax(1, keepdim=True)) / tau
    logp = x - torch.logsumexp(x, 1, keepdim=True)
    p = logp.exp()
    full = torch.logsumexp(c["z"] / tau, 1)
    terms = torch.where(p > 0, p * (logp - c["z"][:, :4] / tau + full[:, None]), 0.0)
    off = tau * tau * (2 * c["z_off"] / tau + 2.0 ** -16 + 4 * U * full.abs() + 64 * U * 16)
    same(torch, "loss", c["loss"], tau * tau * terms.sum(1), off)
    same(torch, "lse", c["lse"], full, c["z_off"] / tau + 2.0 ** -16 + 4 * U * full.abs())
    G = torch.exp(c["z"] / tau - full[:, None])
    G[:, :4] -= p
    G *= (c["dl"].double() * tau)[:, None]
    want = G @ c["w"].double()
    # 2^-8 of each entry of G for its rounding, as much again for the softmax's error
    allowed = 2.0 ** -7 * (G.abs() @ c["w"].double().abs()) + 2.0 ** -7.9 * want.abs()
    same(torch, "dhidden", c["dh"], want, allowed)


def test_teachers_lse_of_minus_infinity(env):
    """A teacher_lse of -inf beside a logit above it has no finite result, and
    none is made up: loss and gradient say so.  Beside logits of -inf alone the
    token takes no part."""
    torch, P = env["torch"], env["P"]
    a = torch.tensor([[1.0, 2.0, 3.0], [-math.inf] * 3, [-math.inf, 0.5, -math.inf], [3.0, 2.0, 1.0]],
                     device="cuda")
    alse = torch.tensor([-math.inf, -math.inf, -math.inf, 4.0], device="cuda")
    c = teacher_case(torch, P, a, alse, 2.0)
    assert torch.isfinite(c["loss"]).tolist() == [False, True, False, True]
    assert torch.isfinite(c["lse"]).all()
    assert torch.isfinite(c["dh"]).any(1).tolist() == [False, True, False, True]
    assert float(c["loss"][1]) == 0.0 and float(c["lse"][1]) == 0.0 and not c["dh"][1].any()
    assert not torch.isfinite(c["dw"]).any()


# ---- after another call's error -------------------------------------------------


def test_an_earlier_error_is_not_this_calls(env):
    """An error that an earlier call of the runtime left behind neither stops a
    call that has nothing to do with it nor makes it fail."""
    torch, P = env["torch"], env["P"]
    from paper_2609_20359_amd import flround as F

    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    T, V, D, K = 40, 500, 64, 4
    h = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    w = torch.randn(V, D, generator=g, device="cuda").bfloat16()
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    x = torch.randn(T, 60000, generator=g, device="cuda")
    dl = torch.full((T,), 0.25, device="cuda")
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    hip = F.hip_runtime()

    def leave_error():
        assert hip.hipSetDevice(ctypes.c_int(1 << 20)) != 0    # no such device; nothing is changed

    def calls(before):
        out = dict(f=[torch.zeros(T, device="cuda") for _ in range(3)],
                   b=[torch.zeros(T, D, device="cuda", dtype=torch.bfloat16),
                      torch.zeros(V, D, device="cuda", dtype=torch.bfloat16)],
                   t=[torch.zeros(T, K, device="cuda"),
                      torch.zeros(T, K, device="cuda", dtype=torch.int32),
                      torch.zeros(T, device="cuda")],
                   d=[torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda"),
                      torch.zeros(T, K, device="cuda")],
                   e=[torch.zeros(T, D, device="cuda", dtype=torch.bfloat16),
                      torch.zeros(V, D, device="cuda", dtype=torch.bfloat16)])
        words = torch.randint(0, V, (T, K), device="cuda",
                              generator=torch.Generator(device="cuda").manual_seed(4)).int()
        torch.cuda.synchronize()
        before()
        P.fl_head_loss(h, w, labels, *out["f"], workspace=ws)
        before()
        P.fl_head_loss_grad(h, w, labels, out["f"][1], out["f"][2], dl, *out["b"], workspace=ws)
        before()
        P.fl_top_logits(x, K, 1.0, *out["t"], workspace=ws)
        before()
        P.fl_head_distill(h, w, words, out["t"][0], None, 1.0, *out["d"], workspace=ws)
        before()
        P.fl_head_distill_grad(h, w, words, out["t"][0], None, 1.0, out["d"][1], out["d"][2], dl,
                               *out["e"], workspace=ws)
        hip.hipGetLastError()                 # nothing is left for the calls of others
        torch.cuda.synchronize()
        return [t for k in sorted(out) for t in out[k]]

    want = calls(lambda: None)
    got = calls(leave_error)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
