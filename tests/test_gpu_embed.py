"""The embedding and its gradient on the GPU against their definition in 64 bits.

Tolerances (u = 2^-24): the forward pass is one product in fp32 and one rounding to the
result's type, so it has torch's bits for the same two steps.  The gradient is an fp32
sum of n terms in any order, off by at most n u sum |x|, times the scale (u), with an
addition (u) where it is added, rounded to its type once (half a step: 2^-8 of a bf16
value, 2^-24 of an fp32 one).
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


@pytest.fixture(scope="module")
def env():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_20359_amd as P

    P.lib()
    return dict(torch=torch, P=P)


def dtype_of(torch, name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def framed(torch, shape, dt, off=3, fill=-7.0):
    """A tensor inside a larger one, `off` elements in, and a check that nothing beside it
    was written."""
    n = math.prod(shape)
    flat = torch.full((n + off + 64,), fill, dtype=dt, device="cuda")

    def check():
        assert bool((flat[:off] == fill).all()) and bool((flat[off + n:] == fill).all())

    return flat[off:off + n].view(shape), check


def make_ids(torch, T, V, kind, g):
    if kind == "same":
        return torch.full((T,), V // 2, dtype=torch.int64, device="cuda")
    if kind == "none":
        return torch.full((T,), -1, dtype=torch.int64, device="cuda")
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    if kind == "all":
        return ids
    r = torch.rand(T, generator=g, device="cuda")
    ids = torch.where(r < 0.3, V - 1, ids)                  # one word of many tokens
    ids = torch.where(r > 0.8, -1 - ids, ids)               # no part
    return torch.where((r > 0.77) & (r <= 0.8), V + ids, ids)   # beyond the vocabulary


def make(torch, T, V, D, dtype, kind="mixed", pad=0, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1000 * T + V + D)
    dt = dtype_of(torch, dtype)
    ids = make_ids(torch, T, V, kind, g)
    w = torch.randn(V, D + pad, generator=g, device="cuda").to(dt)[:, :D]
    d = torch.randn(T, D + pad, generator=g, device="cuda").to(dt)[:, :D]
    return ids, w, d


SIZES = [(1, 1, 1), (1, 70000, 4096), (3, 3, 5), (16, 257, 8), (17, 257, 64), (64, 5003, 321),
         (333, 5003, 515), (700, 40, 1000), (5000, 1, 24), (4096, 40000, 129), (20000, 3000, 72)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("scale,pad", [(1.0, 0), (-17.9, 5)])
def test_embed(env, T, V, D, dtype, scale, pad):
    torch, P = env["torch"], env["P"]
    ids, w, _ = make(torch, T, V, D, dtype, pad=pad)
    out, untouched = framed(torch, (T, D), w.dtype)
    P.fl_embed(ids, w, out, scale=scale)
    rows = (w[ids.clamp(0, V - 1)].float() * scale).to(w.dtype)
    want = torch.where(ids[:, None] < 0, torch.zeros_like(rows), rows)
    want = torch.where(ids[:, None] >= V, torch.full_like(rows, math.nan), want)
    torch.testing.assert_close(out, want, rtol=0, atol=0, equal_nan=True)
    untouched()


def check_grad(env, ids, d, V, scale, add=False, off=3, **kw):
    torch, P = env["torch"], env["P"]
    T, D = d.shape
    half = HALF_STEP["bf16" if d.dtype == torch.bfloat16 else "fp32"]
    dw, untouched = framed(torch, (V, D), d.dtype, off)
    live = (ids >= 0) & (ids < V)
    d[~live] = math.nan                      # not looked at
    at, x = ids[live], d[live].double()
    old = torch.zeros(V, D, device="cuda", dtype=torch.float64)
    if add:
        dw.copy_(torch.randn(V, D, device="cuda").to(d.dtype))
        empty = torch.ones(V, dtype=torch.bool, device="cuda")
        empty[at] = False
        dw[empty] = math.nan                 # left as they are
        old = torch.where(empty[:, None], 0.0, dw.double())
    # (summed on the CPU: many additions to one row at once take a GPU minutes)
    at_c, x_c = at.cpu(), x.cpu()

    def by_word(rows):
        return torch.zeros(V, rows.shape[1], dtype=torch.float64).index_add_(0, at_c, rows).cuda()

    total, size = by_word(x_c), by_word(x_c.abs())
    n = by_word(torch.ones(len(at_c), 1, dtype=torch.float64))
    P.fl_embed_grad(ids, d, dw, scale=scale, add=add, **kw)
    want = old + scale * total
    off64 = abs(scale) * (n * U * size + U * total.abs()) * (1 + 1e-6) + U * want.abs()
    off64 = off64 + half * (want.abs() + off64) + 1e-38
    got = dw.double()
    if add:
        assert bool(got[empty].isnan().all())
        got = torch.where(empty[:, None], 0.0, got)
        want = torch.where(empty[:, None], 0.0, want)
    bad = (got - want).abs() > off64
    assert not bool(bad.any()) and not bool(got.isnan().any()), int(bad.sum())
    untouched()
    return dw


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("add", [False, True])
def test_embed_grad(env, T, V, D, dtype, add):
    ids, _, d = make(env["torch"], T, V, D, dtype, pad=7 if T % 2 else 0)
    check_grad(env, ids, d, V, 1.0 if T % 3 else 5.3, add)


@pytest.mark.parametrize("kind", ["same", "none", "all"])
@pytest.mark.parametrize("T", [15, 16, 17, 48, 257, 511, 512, 513, 1024, 1025, 8192, 8193, 8256, 30000])
def test_runs_of_one_word(env, T, kind):
    """A word of many tokens ends inside a wave's tokens, at their end, or beyond."""
    ids, _, d = make(env["torch"], T, 600, 96, "bf16", kind)
    check_grad(env, ids, d, 600, 0.25)


@pytest.mark.parametrize("T,V,kind", [(20000, 150001, "all"), (20000, 1 << 18, "mixed"),
                                      (1 << 20, 3000, "mixed"), (1 << 20, 700, "same")])
def test_many_tokens_and_words(env, T, V, kind):
    """Workgroups of as many words as they take, and words of more tokens than a wave of
    the sort lists."""
    ids, _, d = make(env["torch"], T, V, 8, "fp32", kind)
    check_grad(env, ids, d, V, 1.0)


def test_ids_past_32_bits(env):
    """Ids from V on are no words, whatever their low bits."""
    torch, P = env["torch"], env["P"]
    ids = torch.tensor([3, (1 << 32) + 3, -(1 << 32) + 3, 1 << 31, (1 << 32) - 1, 20, 19, 3,
                        (1 << 63) - 1, -(1 << 63)], device="cuda")
    d = torch.ones(10, 8, device="cuda")
    dw = torch.empty(20, 8, device="cuda")
    P.fl_embed_grad(ids, d, dw)
    want = torch.zeros(20, 8, device="cuda")
    want[3], want[19] = 2.0, 1.0
    assert torch.equal(dw, want)
    out = torch.empty(10, 8, device="cuda")
    P.fl_embed(ids, want, out)
    nan = [False, True, False, True, True, True, False, False, True, False]
    assert out.isnan().all(1).tolist() == nan and not bool(out[[2, 9]].any())


@pytest.mark.parametrize("first", [1, 14, 15, 16, 17, 31, 32, 33, 63, 64, 65])
def test_words_at_the_borders(env, first):
    """Words of a given number of tokens one after the other."""
    torch = env["torch"]
    words = torch.repeat_interleave(torch.arange(7, device="cuda"),
                                    torch.tensor([first, 1, 16, 33, 15, 64, 2], device="cuda"))
    g = torch.Generator(device="cuda")
    g.manual_seed(first)
    ids = words[torch.randperm(words.numel(), generator=g, device="cuda")]
    d = torch.randn(ids.numel(), 40, generator=g, device="cuda")
    check_grad(env, ids, d, 9, 1.0)


def test_no_tokens(env):
    torch, P = env["torch"], env["P"]
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    P.fl_embed(ids, torch.ones(5, 8, device="cuda"), torch.empty(0, 8, device="cuda"))
    dw = torch.full((5, 8), 3.0, device="cuda")
    P.fl_embed_grad(ids, torch.empty(0, 8, device="cuda"), dw, add=True)
    assert bool((dw == 3.0).all())
    P.fl_embed_grad(ids, torch.empty(0, 8, device="cuda"), dw)
    assert bool((dw == 0.0).all())


def test_same_bits_again_and_in_any_place(env):
    torch, P = env["torch"], env["P"]
    ids, _, d = make(torch, 9000, 300, 200, "fp32")
    d[(ids < 0) | (ids >= 300)] = 0.0
    first = None
    for off in (0, 1, 2, 3):
        dw, _ = framed(torch, (300, 200), torch.float32, off)
        ws = torch.randint(0, 255, (P.embed_workspace_bytes(9000, 300, 200, P.FL_F32) + off,),
                           dtype=torch.uint8, device="cuda")[off:]
        P.fl_embed_grad(ids, d, dw, workspace=ws)
        first = dw.clone() if first is None else first
        assert torch.equal(first, dw)


def test_difference_of_the_loss(env):
    """The gradient against differences: out is linear in the weight, so the differences
    are exact but for the roundings of out (fp32: 2^-24 each)."""
    torch, P = env["torch"], env["P"]
    T, V, D = 200, 50, 16
    ids, w, d = make(torch, T, V, D, "fp32")
    ids = ids.clamp(max=V - 1)
    dw = torch.empty(V, D, device="cuda")
    P.fl_embed_grad(ids, torch.where(ids[:, None] < 0, 0.0, d), dw, scale=3.0)

    def value(weight):
        out = torch.empty(T, D, device="cuda")
        P.fl_embed(ids, weight, out, scale=3.0)
        return (out.double() * d.double()).sum()

    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    step = torch.randn(V, D, generator=g, device="cuda")
    a, b = value(w + step), value(w - step)
    moved = ((w + step).double() - (w - step).double())
    want = (dw.double() * moved).sum()
    live = (ids >= 0).sum()
    off = (2 * U * 3 * 8 * d.double().abs().sum()                 # roundings of out (|out| < 24)
           + (T + 2) * U * 3 * 16 * d.double().abs().sum())       # the gradient's sums (|moved| < 16)
    assert int(live) > 0 and abs(float(a - b - want)) <= float(off)


def test_rows_past_32_bits(env):
    """A table of more than 2^32 elements: its last rows."""
    torch, P = env["torch"], env["P"]
    V, D = (1 << 20) + 3, 4100
    w = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    w[V - 1] = torch.arange(D, device="cuda").bfloat16()
    ids = torch.tensor([V - 1, 0, V - 2, V - 1], device="cuda")
    out = torch.empty(4, D, dtype=torch.bfloat16, device="cuda")
    P.fl_embed(ids, w, out)
    assert torch.equal(out[0], w[V - 1]) and torch.equal(out[3], w[V - 1])
    assert not bool(out[1].any()) and not bool(out[2].any())
    w.fill_(5.0)
    P.fl_embed_grad(ids, torch.ones(4, D, dtype=torch.bfloat16, device="cuda"), w)
    assert bool((w[V - 1] == 2.0).all()) and bool((w[V - 2] == 1.0).all())
    assert bool((w[0] == 1.0).all()) and not bool(w[1:V - 2].any())


def test_streams_and_graphs(env):
    """On another stream, and captured: replays with new inputs in the same places, eager
    calls between them, and two graphs with a workspace each."""
    torch, P = env["torch"], env["P"]
    T, V, D = 3000, 1000, 128
    ids, w, d = make(torch, T, V, D, "bf16", "all")
    side = torch.cuda.Stream()
    out, dw = torch.empty_like(d), torch.empty_like(w)
    side.wait_stream(torch.cuda.current_stream())
    P.fl_embed(ids, w, out, stream=side)
    P.fl_embed_grad(ids, d, dw, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    want_out, want = w[ids], dw.clone()
    eager = torch.empty_like(w)
    P.fl_embed_grad(ids, d, eager)
    assert torch.equal(out, want_out) and torch.equal(eager, want)
    graphs = []
    for k in range(2):
        ws = torch.empty(P.embed_workspace_bytes(T, V, D), dtype=torch.uint8, device="cuda")
        o, g = torch.empty_like(d), torch.empty_like(w)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            P.fl_embed(ids, w, o)
            P.fl_embed_grad(ids, d, g, workspace=ws)
        graphs.append((graph, o, g, ws))
    for turn in range(4):
        ids.copy_(make_ids(torch, T, V, "all", torch.Generator(device="cuda")).roll(turn * 7))
        d.copy_(torch.randn(T, D, device="cuda"))
        P.fl_embed_grad(ids, d, eager)
        for graph, o, g, _ in graphs:
            g.fill_(-3.0)
            graph.replay()
        torch.cuda.synchronize()
        for _, o, g, _ in graphs:
            assert torch.equal(g, eager) and torch.equal(o, w[ids])


def test_refusals(env):
    torch, P = env["torch"], env["P"]
    ids, w, d = make(torch, 8, 20, 16, "bf16", "all")
    out, dw = torch.empty_like(d), torch.empty(20, 16, dtype=torch.bfloat16, device="cuda")
    for args in ((ids.int(), w, out), (ids, w.half(), out), (ids, w, out.float()),
                 (ids, w, out[:7]), (ids[:, None], w, out), (ids.cpu(), w, out),
                 (ids, w.t(), out), (ids, w.cpu(), out)):
        with pytest.raises(ValueError):
            P.fl_embed(*args)
    for args in ((ids.int(), d, dw), (ids, d[:7], dw), (ids, d, dw.float()), (ids, d, dw[:, :15]),
                 (ids, d, dw[0])):
        with pytest.raises(ValueError):
            P.fl_embed_grad(*args)
    for call in (lambda: P.fl_embed(ids, w, out, scale=math.inf),
                 lambda: P.fl_embed(ids, w, w[:8]),
                 lambda: P.fl_embed_grad(ids, d, dw, scale=math.nan),
                 lambda: P.fl_embed_grad(ids, d, dw, workspace=torch.empty(
                     64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(P.FlError):
            call()


def test_ids_past_32_bits_among_many(env):
    """As above, by way of the sort: ids whose low or high 32 bits are a word's, or a
    negative number's, or 0."""
    torch, P = env["torch"], env["P"]
    V, top = 700, 1 << 31
    odd = [1 << 32, (1 << 32) + 3, -(1 << 32) + 3, top - 1, top, top + 1, top + V, (1 << 32) - 1, (1 << 32) - V,
           V, V + 1, -1, (1 << 63) - 1, -(1 << 63), 3 << 32, (699 << 32) + 699]
    words = torch.arange(2000, device="cuda") % V
    ids = torch.cat([words, torch.tensor(odd * 40, device="cuda")])
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    ids = ids[torch.randperm(ids.numel(), generator=g, device="cuda")]
    d = torch.ones(ids.numel(), 8, device="cuda")
    d[(ids < 0) | (ids >= V)] = math.nan
    dw = torch.empty(V, 8, device="cuda")
    P.fl_embed_grad(ids, d, dw)
    want = torch.full((V, 8), 2.0, device="cuda")
    want[:600] = 3.0
    assert torch.equal(dw, want)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("T", [1024, 1025, 2048, 2049, 8192, 8193, 16384, 16385])
def test_both_sides_of_the_tiles_sizes(env, T, add):
    """A third of the tokens one word, which goes on over many waves' tokens."""
    ids, _, d = make(env["torch"], T, 900, 136, "bf16")
    check_grad(env, ids, d, 900, 1.0, add)
