"""AdamW over many tensors on the GPU: with states in 32 bits bit for bit what
fl_adamw_step gives for each tensor; with states in 8 bits the same of the values held,
and codes bit for bit those of their definition (state8.py)."""
import math

import numpy as np
import pytest

import state8 as S8

pytestmark = pytest.mark.gpu

HP = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def env():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_20359_amd as P

    P.lib()
    return dict(torch=torch, P=P)


def carve(torch, sizes, dt, skew, fill):
    """Tensors inside one buffer, each `skew` elements behind the one before it."""
    flat = torch.full((sum(sizes) + skew * (len(sizes) + 1) + 64,), fill, dtype=dt, device="cuda")
    at, out = skew, []
    for n in sizes:
        out.append(flat[at:at + n])
        at += n + skew
    return flat, out


class Group:
    """Masters, working copies and gradients of tensors, and what is around them."""

    def __init__(self, torch, sizes, grad="fp32", skew=1, seed=0, spread=1.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + sum(sizes))
        self.torch, self.sizes, self.skew, self.g, self.spread = torch, sizes, skew, g, spread
        self.grad_dtype = torch.bfloat16 if grad == "bf16" else torch.float32
        self.mflat, self.masters = carve(torch, sizes, torch.float32, skew, -7.0)
        self.wflat, self.workings = carve(torch, sizes, torch.bfloat16, skew, -7.0)
        for m, w in zip(self.masters, self.workings):
            m.copy_(torch.randn(m.numel(), generator=g, device="cuda"))
            w.copy_(m)
        self.decays = [i % 3 != 1 for i in range(len(sizes))]
        self.gflat, self.grads = carve(torch, sizes, self.grad_dtype, skew, -7.0)
        self.new_grads()

    def new_grads(self):
        torch = self.torch
        for x in self.grads:
            n = x.numel()
            size = torch.exp(self.spread * torch.randn(n, generator=self.g, device="cuda"))
            x.copy_(size * torch.randn(n, generator=self.g, device="cuda") * 1e-2)

    def starts(self):
        at, out = 0, []
        for n in self.sizes:
            out.append(at)
            at += -(-n // S8.UNIT) * S8.UNIT
        return out, at

    def check_frames(self):
        for flat, parts in ((self.mflat, self.masters), (self.wflat, self.workings)):
            at = 0
            for p in parts:
                first = (p.data_ptr() - flat.data_ptr()) // flat.element_size() if p.numel() else at
                assert bool((flat[at:first] == -7.0).all())
                at = first + p.numel()
            assert bool((flat[at:] == -7.0).all())


def reference(env, grp, m, v, step, hp=HP, scale=1.0):
    """fl_adamw_step of each tensor on copies: lists of master, m, v, working."""
    torch, P = env["torch"], env["P"]
    out = []
    starts, _ = grp.starts()
    for k, n in enumerate(grp.sizes):
        if n == 0:
            out.append(None)
            continue
        lay = P.Layout([0, n], [1 if grp.decays[k] else 0])
        t = [x.clone().contiguous() for x in (grp.masters[k], m[starts[k]:starts[k] + n],
                                              v[starts[k]:starts[k] + n])]
        w = torch.empty(n, dtype=torch.bfloat16, device="cuda")
        P.fl_adamw_step(lay, hp, step, (grp.grads[k].float() * scale).contiguous(), *t, working=w)
        out.append(t + [w])
        torch.cuda.synchronize()
        lay.close()
    return out


SIZES = [[1], [3, 511, 512, 513], [0, 5, 0, 1024, 700, 0], [4097, 64, 63, 65, 100000, 2],
         list(range(1, 301)), [20000] * 5 + [7] * 97]


@pytest.mark.parametrize("grad", ["fp32", "bf16"])
@pytest.mark.parametrize("sizes", SIZES, ids=[str(len(s)) for s in SIZES])
@pytest.mark.parametrize("skew", [0, 1, 8])
def test_32_bits_are_the_flat_step(env, sizes, grad, skew):
    torch, P = env["torch"], env["P"]
    grp = Group(torch, sizes, grad, skew)
    ts = P.Tensors(grp.masters, grp.workings, grp.decays)
    state = ts.state(32)
    starts, n = grp.starts()
    assert ts.n_state == n
    steps = 3 if len(sizes) < 100 else 2
    for step in range(1, steps + 1):
        want = reference(env, grp, state[:n], state[n:], step, scale=0.25)
        P.fl_adamw_tensors(ts, HP, step, grp.grads, state, grad_scale=0.25)
        for k, size in enumerate(sizes):
            if size == 0:
                continue
            a = starts[k]
            got = (grp.masters[k], state[a:a + size], state[n + a:n + a + size], grp.workings[k])
            for x, y in zip(got, want[k]):
                assert torch.equal(x, y), (k, size)
            end = starts[k + 1] if k + 1 < len(sizes) else n
            assert not bool(state[a + size:end].any()) and not bool(state[n + a + size:n + end].any())
        grp.check_frames()
        grp.new_grads()


@pytest.mark.parametrize("grad", ["fp32", "bf16"])
@pytest.mark.parametrize("seed", [0, 12345, (1 << 63) + 7])
@pytest.mark.parametrize("sizes", SIZES[:5], ids=[str(len(s)) for s in SIZES[:5]])
def test_8_bits(env, sizes, grad, seed):
    """From the values held, the step is the flat one's; what is held afterwards is the
    code of its moments."""
    torch, P = env["torch"], env["P"]
    grp = Group(torch, sizes, grad, 1, spread=3.0)
    ts = P.Tensors(grp.masters, grp.workings, grp.decays)
    state = ts.state(8)
    starts, n = grp.starts()
    for step in range(1, 4 if len(sizes) < 100 else 3):
        mc, vc, me, ve = S8.split(state.cpu().numpy(), n)
        m = torch.from_numpy(S8.decode(mc, me, S8.TOP_M)).cuda()
        v = torch.from_numpy(S8.decode(vc, ve, S8.TOP_V)).cuda()
        want = reference(env, grp, m, v, step)
        P.fl_adamw_tensors(ts, HP, step, grp.grads, state, seed=seed)
        mn, vn = np.zeros(n, np.float32), np.zeros(n, np.float32)
        for k, size in enumerate(sizes):
            if size == 0:
                continue
            assert torch.equal(grp.masters[k], want[k][0]) and torch.equal(grp.workings[k], want[k][3])
            mn[starts[k]:starts[k] + size] = want[k][1].cpu().numpy()
            vn[starts[k]:starts[k] + size] = want[k][2].cpu().numpy()
        dm, dv = S8.draws(n, seed, step) if seed else (None, None)
        got = S8.split(state.cpu().numpy(), n)
        for x, y in zip(got[0::2], S8.encode(mn, S8.TOP_M, dm)):
            assert np.array_equal(x, y)
        for x, y in zip(got[1::2], S8.encode(vn, S8.TOP_V, dv)):
            assert np.array_equal(x, y)
        grp.check_frames()
        grp.new_grads()


def specials():
    """Blocks of values at the ends of the codes."""
    f = np.float32
    tiny = np.ldexp(f(1), np.arange(-149, -85).astype(np.int32)).astype(f)
    huge = np.ldexp(f(1.9), np.arange(64, 128).astype(np.int32)).astype(f)
    one = np.ones(64, f)
    near = np.array([1.75, 1.7500001, 1.8125, 1.99999, 1.0, 0.9375] * 11, f)[:64]
    mixed = np.geomspace(1e-30, 1e30, 64).astype(f)
    odd = one.copy()
    odd[[3, 9, 11]] = [np.nan, np.inf, 1e-3]
    rng = np.random.RandomState(3)
    rand = (np.exp(rng.randn(64 * 8) * 6) * rng.choice([-1, 1], 64 * 8)).astype(f)
    ties = np.concatenate([(np.arange(64) + 8.5) / 8 * 2.0 ** -k for k in range(4)]).astype(f)
    sub = np.concatenate([np.array([448.0] + [(k + 0.5) * 2.0 ** -9 for k in range(63)])]).astype(f)
    none = np.zeros(64, f)
    only = np.full(64, np.inf, f)
    zeros = one * np.float32(1e-3)
    zeros[::3] = -0.0
    x = np.concatenate([zeros, tiny, huge, one, near, mixed, odd, rand, ties, sub, none, only, -one, -mixed])
    return np.pad(x, (0, -len(x) % 512))


def test_convert_special_values(env):
    torch, P = env["torch"], env["P"]
    x = specials()
    n = len(x)
    v = np.abs(x)
    v[0] = -0.0                                # (held as 0)
    wide = torch.from_numpy(np.concatenate([x, v])).cuda()
    narrow = torch.full((2 * n + n // 32,), 99, dtype=torch.uint8, device="cuda")
    P.fl_state_convert(wide, narrow)
    mc, vc, me, ve = S8.split(narrow.cpu().numpy(), n)
    for got, want in ((mc, S8.encode(x, 15)[0]), (me, S8.encode(x, 15)[1]),
                      (vc, S8.encode(v, 31)[0]), (ve, S8.encode(v, 31)[1])):
        assert np.array_equal(got, want)
    back = torch.empty_like(wide)
    P.fl_state_convert(narrow, back)
    got = back.cpu().numpy()
    assert np.array_equal(got[:n], S8.decode(mc, me, 15), equal_nan=True)
    assert np.array_equal(got[n:], S8.decode(vc, ve, 31), equal_nan=True)
    assert (got[n:][np.abs(x) > 0] != 0).all()


def test_every_code_and_exponent(env):
    """All 256 codes at every exponent byte that is ever written; a value that is held is
    held unchanged, whatever its block's largest is."""
    torch, P = env["torch"], env["P"]
    codes = np.tile(np.arange(256, dtype=np.uint8), 512)
    exps = np.repeat(np.maximum(np.arange(512) // 2, 12), 4).astype(np.uint8)
    n = len(codes)
    narrow = torch.from_numpy(np.concatenate([codes, codes, exps, exps])).cuda()
    wide = torch.empty(2 * n, device="cuda")
    P.fl_state_convert(narrow, wide)
    got = wide.cpu().numpy()
    m, v = S8.decode(codes, exps, 15), S8.decode(codes, exps, 31)
    assert np.array_equal(got[:n], m, equal_nan=True) and np.array_equal(got[n:], v, equal_nan=True)
    assert np.array_equal(np.signbit(got[:n][~np.isnan(m)]), np.signbit(m[~np.isnan(m)]))
    again, back = torch.empty_like(narrow), torch.empty_like(wide)
    wide = torch.where(wide.isfinite(), wide, torch.zeros_like(wide))
    P.fl_state_convert(wide, again)
    P.fl_state_convert(again, back)
    a, b = wide.cpu().numpy(), back.cpu().numpy()
    for k, top in ((0, 15), (1, 31)):
        x, y = a[k * n:(k + 1) * n].reshape(-1, 64), b[k * n:(k + 1) * n].reshape(-1, 64)
        # (a block of small codes has a lower exponent now, which holds them as well)
        assert np.array_equal(x, y)


def test_a_state_of_zeros_is_positive_zeros(env):
    """Before the first step: no sign in either moment, and exponent bytes below 12, which
    stand for 12."""
    torch, P = env["torch"], env["P"]
    n = 1024
    narrow = torch.zeros(2 * n + n // 32, dtype=torch.uint8, device="cuda")
    wide = torch.full((2 * n,), -7.0, device="cuda")
    P.fl_state_convert(narrow, wide)
    assert not bool(wide.view(torch.int32).any())
    codes = np.tile(np.arange(256, dtype=np.uint8), 4)
    exps = np.arange(16, dtype=np.uint8)
    narrow = torch.from_numpy(np.concatenate([codes, codes, exps, exps])).cuda()
    P.fl_state_convert(narrow, wide)
    got = wide.cpu().numpy()
    low = np.maximum(exps, 12)
    assert np.array_equal(got[:n], S8.decode(codes, low, 15), equal_nan=True)
    assert np.array_equal(got[n:], S8.decode(codes, low, 31), equal_nan=True)
    master = torch.ones(600, device="cuda")
    t = P.Tensors([master])
    state = t.state(8)
    P.fl_adamw_tensors(t, HP, 1, [torch.full((600,), -0.0, device="cuda")], state)
    assert not bool(state[:2 * n].any())       # 0 * beta1 + -0 is 0


def test_draws_are_even_and_the_held_value_is_right_on_average(env):
    """n equal moments between two codes, a quarter of the way up.  What is held is one of
    the two, up in a share of 1/4 that n independent draws miss by 6 sqrt(3/16/n) once in
    10^9; the update of m alone (v's is tested the same way)."""
    torch, P = env["torch"], env["P"]
    n = 1 << 20
    hp = dict(HP, beta1=0.5, beta2=0.5)
    master = torch.zeros(n, device="cuda")
    ts = P.Tensors([master])
    g = torch.full((n,), 2 * (1 + 0.25 / 8), device="cuda")      # m = 1 + 1/32, of steps of 1/8
    g[::64] = 2 * 1.5                                            # the block's largest
    gv = torch.full((n,), math.sqrt(2 * (1 + 0.25 / 8)), device="cuda")
    gv[::64] = math.sqrt(2 * 1.5)
    for grad, first, top in ((g, 0, 15), (gv, 1, 31)):
        shares = []
        for seed, step in ((1, 1), (2, 1), (1, 2), ((1 << 40) + 3, 77)):
            state = ts.state(8)
            P.fl_adamw_tensors(ts, hp, step, [grad], state, seed=seed)
            codes = S8.split(state.cpu().numpy(), n)[first].reshape(-1, 64)[:, 1:]
            low = 8 * top
            assert set(np.unique(codes)) == {low, low + 1}
            up = codes == low + 1
            shares.append(up)
            # (the second moment's place is that of the rounded root's square: within 2^-20)
            assert abs(up.mean() - 0.25) <= 6 * math.sqrt(3 / 16 / up.size) + 2.0 ** -20
        for k in range(1, 4):    # different keys, different draws: both up in 1/16
            both = (shares[0] & shares[k]).mean()
            assert abs(both - 1 / 16) <= 6 * math.sqrt(1 / 16 / shares[0].size)
    state = ts.state(8)
    P.fl_adamw_tensors(ts, hp, 1, [g], state, seed=1)
    other = ts.state(8)
    P.fl_adamw_tensors(ts, hp, 1, [g], other, seed=1)
    assert torch.equal(state, other)


@pytest.mark.parametrize("bits", [8, 32])
def test_tensors_without_a_gradient(env, bits):
    torch, P = env["torch"], env["P"]
    sizes = [700, 5, 512, 0, 1000, 33] * 30
    grp, all_ = Group(torch, sizes), Group(torch, sizes)
    ts, ta = P.Tensors(grp.masters, grp.workings), P.Tensors(all_.masters, all_.workings)
    s, sa = ts.state(bits), ta.state(bits)
    left = [k % 4 == 1 or k in (0, 177) for k in range(len(sizes))]
    before = [m.clone() for m in grp.masters]
    P.fl_adamw_tensors(ts, HP, 1, [None if x else g for x, g in zip(left, grp.grads)], s, seed=4 if bits == 8 else 0)
    P.fl_adamw_tensors(ta, HP, 1, all_.grads, sa, seed=4 if bits == 8 else 0)
    starts, n = grp.starts()
    for k, size in enumerate(sizes):
        want = before[k] if left[k] else all_.masters[k]
        assert torch.equal(grp.masters[k], want)
        u = slice(starts[k], starts[k] + size)
        for part, whole in ((s[:n], sa[:n]), (s[n:2 * n], sa[n:2 * n])):
            assert torch.equal(part[u], torch.zeros_like(part[u]) if left[k] else whole[u])
    P.fl_adamw_tensors(ts, HP, 1, [None] * len(sizes), s)
    assert all(torch.equal(a, b) for k, (a, b) in enumerate(zip(grp.masters, before)) if left[k])


def test_working_copies_may_be_left_out(env):
    torch, P = env["torch"], env["P"]
    a, b = Group(torch, [600, 70]), Group(torch, [600, 70])
    ta, tb = P.Tensors(a.masters, [None, a.workings[1]], a.decays), P.Tensors(b.masters, b.workings, b.decays)
    old = a.workings[0].clone()
    P.fl_adamw_tensors(ta, HP, 1, a.grads, ta.state(8))
    P.fl_adamw_tensors(tb, HP, 1, b.grads, tb.state(8))
    assert torch.equal(a.workings[0], old) and torch.equal(a.workings[1], b.workings[1])
    assert all(torch.equal(x, y) for x, y in zip(a.masters, b.masters))


def test_special_gradients(env):
    """NaN and infinite gradients: the element's own moments and master are lost, and no
    other's."""
    torch, P = env["torch"], env["P"]
    a, b = Group(torch, [1500]), Group(torch, [1500])
    a.grads[0][100], a.grads[0][700] = math.nan, math.inf
    a.grads[0][701] = 1e30                    # its square is no fp32 number
    ta, tb = P.Tensors(a.masters), P.Tensors(b.masters)
    sa, sb = ta.state(8), tb.state(8)
    for step in (1, 2):
        P.fl_adamw_tensors(ta, HP, step, a.grads, sa)
        P.fl_adamw_tensors(tb, HP, step, b.grads, sb)
        a.grads[0][[100, 700, 701]] = 0.0
    wide = torch.empty(2 * 1536, device="cuda")
    P.fl_state_convert(sa, wide)
    lost = wide[:1500].isnan() | wide[1536:1536 + 1500].isnan()
    assert lost.nonzero().flatten().tolist() == [100, 700, 701]
    same = torch.ones(1500, dtype=torch.bool, device="cuda")
    same[640:704] = False                     # (their block's exponent is another: 1e29)
    same[[100]] = False
    assert torch.equal(a.masters[0][same], b.masters[0][same])
    assert bool(a.masters[0].isnan()[[100, 700]].all())
    assert int(a.masters[0].isnan().sum()) <= 3


def test_a_tensor_past_32_bits(env):
    """More than 2^32 elements: the first and the last ones against a small tensor with
    the same values."""
    torch, P = env["torch"], env["P"]
    n = (1 << 32) + 1029
    master = torch.zeros(n, device="cuda")
    grad = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    ends = [slice(0, 2048), slice((1 << 32) - 1024, n)]     # whole units
    small = []
    for e in ends:
        k = grad[e].numel()
        grad[e] = (torch.randn(k, generator=g, device="cuda") * 1e-2).bfloat16()
        master[e] = torch.randn(k, generator=g, device="cuda")
        small.append((master[e].clone(), grad[e].clone()))
    ts = P.Tensors([master])
    state = ts.state(8)
    P.fl_adamw_tensors(ts, HP, 1, [grad], state, seed=9)
    state_n = ts.n_state
    for e, (m0, g0) in zip(ends, small):
        t = P.Tensors([m0])
        s = t.state(8)
        P.fl_adamw_tensors(t, HP, 1, [g0], s)
        assert torch.equal(master[e], m0)
        k = g0.numel()
        lay = P.Layout([0, k])
        m, v, mm = torch.zeros(k, device="cuda"), torch.zeros(k, device="cuda"), m0.clone()
        P.fl_adamw_step(lay, HP, 1, g0.float(), mm, m, v)
        torch.cuda.synchronize()
        lay.close()
        full = -(-k // 512) * 512
        dm, _ = S8.draws(full, 9, 1, e.start)
        mn = np.pad(m.cpu().numpy(), (0, full - k))
        want = S8.encode(mn, 15, dm)[0]
        assert np.array_equal(state[e.start:e.start + full].cpu().numpy(), want)
    assert not bool(master[2048:1 << 20].any())
    assert state.numel() == 2 * state_n + state_n // 32


def test_streams_and_graphs(env):
    torch, P = env["torch"], env["P"]
    sizes = [3000, 17, 4096] + [100] * 120
    a, b = Group(torch, sizes, "bf16"), Group(torch, sizes, "bf16")
    ta, tb = P.Tensors(a.masters, a.workings), P.Tensors(b.masters, b.workings)
    sa, sb = ta.state(8), tb.state(8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    P.fl_adamw_tensors(ta, HP, 1, a.grads, sa, seed=3, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    P.fl_adamw_tensors(tb, HP, 1, b.grads, sb, seed=3)
    assert torch.equal(sa, sb) and torch.equal(a.mflat, b.mflat)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.fl_adamw_tensors(ta, HP, 2, a.grads, sa, seed=3)
    for _ in range(4):
        a.new_grads()
        b.gflat.copy_(a.gflat)
        graph.replay()
        P.fl_adamw_tensors(tb, HP, 2, b.grads, sb, seed=3)
        torch.cuda.synchronize()
        assert torch.equal(sa, sb) and torch.equal(a.mflat, b.mflat) and torch.equal(a.wflat, b.wflat)


def test_refusals(env):
    torch, P = env["torch"], env["P"]
    grp = Group(torch, [100, 50])
    ts = P.Tensors(grp.masters, grp.workings)
    state = ts.state(8)
    flat = torch.zeros(200, device="cuda")
    for args in (([flat[:100], flat[99:150]],), ([flat, flat],), ([flat.bfloat16()],),
                 ([flat.cpu()],), ([flat[::2]],), ([flat], [flat.bfloat16()[:99]]),
                 ([flat], [flat]), ([flat], None, [1, 0]), ([flat], [None, None])):
        with pytest.raises(ValueError):
            P.Tensors(*args)
    with pytest.raises(ValueError):
        ts.state(16)
    good = grp.grads
    for grads in ([good[0]], good + [flat], [good[0], good[1][:49]], [good[0], good[1].bfloat16()],
                  [good[0], good[1].cpu()], [good[0].half(), good[1].half()]):
        with pytest.raises(ValueError):
            P.fl_adamw_tensors(ts, HP, 1, grads, state)
    for bad in (state[:-1], state.float(), state.int(), ts.state(32)[1:]):
        with pytest.raises(ValueError):
            P.fl_adamw_tensors(ts, HP, 1, good, bad)
    for kw in (dict(step=0), dict(grad_scale=math.nan), dict(hp=dict(HP, eps=0.0)),
               dict(state=ts.state(32), seed=1), dict(grads=[grp.masters[0], good[1]])):
        a = dict(dict(hp=HP, step=1, grads=good, state=state), **kw)
        with pytest.raises(P.FlError):
            P.fl_adamw_tensors(ts, a.pop("hp"), a.pop("step"), a.pop("grads"), a.pop("state"), **a)
    for seed in (-1, 1 << 64):
        with pytest.raises(ValueError):
            P.fl_adamw_tensors(ts, HP, 1, good, state, seed=seed)
    wide = torch.zeros(2 * ts.n_state, device="cuda")
    for src, dst in ((state, state.clone()), (wide, wide.clone()), (state, wide[2:]),
                     (state[1:], wide), (state, wide.half())):
        with pytest.raises(ValueError):
            P.fl_state_convert(src, dst)
    empty = P.Tensors([])
    P.fl_adamw_tensors(empty, HP, 1, [], torch.zeros(0, device="cuda"))


def test_a_parameter_that_moves(env):
    """A master or a working copy that was given other memory, or whose memory was given
    back: the step says so, and writes nowhere."""
    torch, P = env["torch"], env["P"]

    def resized(t):
        t.untyped_storage().resize_(0)

    def replaced(t):
        t.data = t.data.clone()

    for which in (0, 1):
        for move in (replaced, resized):
            masters = [torch.ones(n, device="cuda") for n in (100, 700, 0)]
            workings = [torch.nn.Parameter(m.bfloat16()) for m in masters]
            grads = [torch.ones_like(m) for m in masters]
            ts = P.Tensors(masters, workings)
            state = ts.state(8)
            P.fl_adamw_tensors(ts, HP, 1, grads, state)
            before = [t.detach().clone() for t in masters + workings]
            move((masters, workings)[which][1])
            kept = state.clone()
            with pytest.raises(ValueError, match="moved"):
                P.fl_adamw_tensors(ts, HP, 2, grads, state)
            assert torch.equal(state, kept)
            if move is replaced:
                assert all(torch.equal(a, b) for a, b in zip(masters + workings, before))
                P.fl_adamw_tensors(P.Tensors(masters, workings), HP, 2, grads, state)
                assert not torch.equal(masters[1], before[1]) and not torch.equal(state, kept)
                assert torch.equal(masters[0].bfloat16(), workings[0])


def test_many_gradients_some_left_out(env):
    """Addresses of gradients past the first launch's, with some left out on both sides."""
    torch, P = env["torch"], env["P"]
    sizes = [3] * 250
    a, b = Group(torch, sizes, "bf16"), Group(torch, sizes, "bf16")
    ta, tb = P.Tensors(a.masters), P.Tensors(b.masters)
    left = {0, 1, 95, 96, 97, 200, 249}
    before = [m.clone() for m in a.masters]
    P.fl_adamw_tensors(ta, HP, 1, [None if k in left else g for k, g in enumerate(a.grads)], ta.state(32))
    P.fl_adamw_tensors(tb, HP, 1, b.grads, tb.state(32))
    for k in range(250):
        assert torch.equal(a.masters[k], before[k] if k in left else b.masters[k]), k
