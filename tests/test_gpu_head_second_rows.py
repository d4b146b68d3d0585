"""The gradient of up to 32 tokens, whose G counts with 16 bits (two bf16 numbers
an entry, the value rounded and what that left): inputs for which a G of 8 bits
would show.

A row of G sums to 0.  A weight whose columns are 1 plus a few steps of 2^-7
therefore takes the large parts of a row's terms out of dhidden, and hidden states
of opposite signs, in columns that the weight does not have, those of a word's
terms out of dweight: what G's rounding leaves stands beside results some 2^-7 of
the terms, whose own rounding is 2^-15 of them.

Bound, per entry of G (u = 2^-24): 2^-16 |G| for its two roundings; twice what lse
is off by, for its exponential's share; 2^-20 of the listed words' share.  lse is
off by (D + 8) u sum |h||w|, 2^-16 and 4 u |lse|.  The products' sums in fp32 add
(n + 64) u of their terms, and the results' rounding 2^-8 of them.
"""
import pytest

U = 2.0 ** -24


def bf16(torch, x):
    return x.bfloat16().double()


class Inputs:
    def __init__(self, torch, T, V, K, dev, seed=0):
        g = torch.Generator()
        g.manual_seed(1000 * T + 10 * V + K + seed)
        self.T, self.V, self.K, self.tau = T, V, K, 1.0
        # columns: 0 to 3 make the logits, 4 to 11 show dhidden, 12 to 19 dweight
        D = self.D = 20
        h = torch.zeros(T, D)
        h[:, :4] = torch.randint(6, 11, (T, 4), generator=g) / 8.0
        h[:, 12:] = (1.0 - 2.0 * (torch.arange(T) % 2).float())[:, None]
        w = torch.zeros(V, D)
        w[:, :4] = torch.randint(-8, 9, (V, 4), generator=g) / 16.0
        w[:, 4:12] = 1.0 + torch.randint(0, 4, (V, 8), generator=g) / 128.0
        self.h, self.w = h.bfloat16().to(dev), w.bfloat16().to(dev)
        dl = (0.75 + 0.25 * torch.rand(T, generator=g)) / T
        self.dloss = dl.to(dev)
        hd, wd = self.h.double(), self.w.double()
        z = hd @ wd.t()
        if K == 0:
            self.labels = torch.randint(0, V, (1,), generator=g).repeat(T).to(dev)
            ids = self.labels[:, None]
            p = torch.ones(T, 1, dtype=torch.float64, device=dev)
        else:
            self.ids = torch.arange(K, dtype=torch.int32).repeat(T, 1).to(dev)
            self.a = (torch.randint(0, 9, (1, K), generator=g) / 4.0).repeat(T, 1).to(dev)
            ids = self.ids.long()
            p = torch.softmax(self.a.double(), 1)
        lse = torch.logsumexp(z, 1)
        c = dl.double().to(dev)[:, None]
        share = torch.exp(z - lse[:, None]) * c
        spot = torch.zeros_like(share).scatter_add_(1, ids, c * p)
        self.G = share - spot
        z_off = ((self.D + 8) * U * (hd.abs() @ wd.abs().t())).amax(1)
        lse_off = z_off + 2.0 ** -16 + 4 * U * lse.abs()
        off = (2.0 ** -16 * self.G.abs() + (2 * lse_off + 2.0 ** -20)[:, None] * share
               + 2.0 ** -20 * spot)
        self.dh, self.dw = self.G @ wd, self.G.t() @ hd
        self.dh_off = (off @ wd.abs() + (V + 64) * U * (self.G.abs() @ wd.abs())
                       + 2.0 ** -8 * self.dh.abs())
        self.dw_off = (off.t() @ hd.abs() + (2 * T + 64) * U * (self.G.abs().t() @ hd.abs())
                       + 2.0 ** -8 * self.dw.abs())

    def beyond(self, dh, dw):
        """The share of results beyond the bound, in the columns that show it."""
        a = ((dh.double() - self.dh).abs() > self.dh_off)
        b = ((dw.double() - self.dw).abs() > self.dw_off)
        return float(a[:, 4:12].double().mean()), float(b[:, 12:].double().mean()), a, b


SIZES = [(2, 5, 0), (2, 5, 3), (6, 9, 0), (8, 12, 4), (32, 40, 0), (32, 40, 9), (17, 300, 0)]


@pytest.mark.parametrize("T,V,K", SIZES)
def test_one_rounding_would_show(T, V, K):
    """The bound says something: a G rounded once to bf16, in units of the largest
    |dloss|, exceeds it, and one of two such numbers does not."""
    import torch

    c = Inputs(torch, T, V, K, "cpu")
    scale = float(c.dloss.max())
    G = c.G / scale
    once = bf16(torch, G)
    twice = once + bf16(torch, G - once)
    h, w = c.h.double(), c.w.double()

    def results(g):
        return bf16(torch, g @ w * scale), bf16(torch, g.t() @ h * scale)

    dh, dw, _, _ = c.beyond(*results(once))
    assert dh > 0.1 and dw > 0.1, (dh, dw)
    *_, a, b = c.beyond(*results(twice))
    assert not a.any() and not b.any()


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,K", SIZES)
def test_gradient_of_few_tokens(T, V, K):
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_20359_amd as P

    c = Inputs(torch, T, V, K, "cuda")
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dh = torch.full((T, c.D), -7.0, device="cuda", dtype=torch.bfloat16)
    dw = torch.full((V, c.D), -7.0, device="cuda", dtype=torch.bfloat16)
    if K == 0:
        target = torch.empty(T, device="cuda")
        P.fl_head_loss(c.h, c.w, c.labels, loss, lse, target)
        P.fl_head_loss_grad(c.h, c.w, c.labels, lse, target, c.dloss, dh, dw)
    else:
        target = torch.empty(T, K, device="cuda")
        P.fl_head_distill(c.h, c.w, c.ids, c.a, None, c.tau, loss, lse, target)
        P.fl_head_distill_grad(c.h, c.w, c.ids, c.a, None, c.tau, lse, target, c.dloss, dh, dw)
    *_, a, b = c.beyond(dh, dw)
    assert not a.any(), ("dhidden", int(a.sum()), a.nonzero()[:3].tolist())
    assert not b.any(), ("dweight", int(b.sum()), b.nonzero()[:3].tolist())
