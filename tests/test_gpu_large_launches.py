"""Outputs, tables and states so large that one launch would take 2^32 threads or more,
which HIP refuses: such a call takes several.  (The largest array of a test is 64 GiB.)"""
import math

import numpy as np
import pytest

import state8 as S8
from test_gpu_embed import env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_back(env):  # noqa: F811
    yield
    env["torch"].cuda.synchronize()
    env["torch"].cuda.empty_cache()


def test_embed_of_64_gib(env):  # noqa: F811
    """2^32 chunks of 16 bytes."""
    torch, P = env["torch"], env["P"]
    T, V, D = 1 << 20, 7, 1 << 15
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    w = torch.randn(V, D, generator=g, device="cuda").bfloat16()
    ids = torch.randint(-1, V + 1, (T,), generator=g, device="cuda")
    out = torch.full((T, D), -7.0, dtype=torch.bfloat16, device="cuda")
    P.fl_embed(ids, w, out)
    rows = torch.cat([w, torch.full((1, D), math.nan, dtype=w.dtype, device="cuda"),
                      torch.zeros(1, D, dtype=w.dtype, device="cuda")])    # of V and of -1
    for t in range(0, T, 1 << 15):
        got, want = out[t:t + (1 << 15)], rows[ids[t:t + (1 << 15)]]
        assert bool(((got == want) | (got.isnan() & want.isnan())).all()), t


@pytest.mark.parametrize("extra", [0, 5])
def test_embed_grad_of_a_table_of_64_gib(env, extra):  # noqa: F811
    """2^32 chunks of zeros, and some rows more; all values are whole and small."""
    torch, P = env["torch"], env["P"]
    V, D = (1 << 20) + extra, 1 << 15
    half, last = 1 << 19, V - 1
    ids = torch.tensor([0, half - 1, half, last] * 150 + [last, 77, -1, V], device="cuda")
    d = torch.ones(ids.numel(), D, dtype=torch.bfloat16, device="cuda")
    dw = torch.full((V, D), 3.0, dtype=torch.bfloat16, device="cuda")
    P.fl_embed_grad(ids, d, dw, scale=0.5)
    for v, want in ((0, 75.0), (half - 1, 75.0), (half, 75.0), (last, 75.5), (77, 0.5)):
        assert bool((dw[v] == want).all()), v
        dw[v] = 0.0
    for v in range(0, V, 1 << 15):
        assert not bool(dw[v:v + (1 << 15)].any()), v


def test_convert_past_32_bits(env):  # noqa: F811
    """A state of more elements than one launch takes, both ways: its first and last codes
    and those where the launches meet."""
    torch, P = env["torch"], env["P"]
    n, k = (1 << 32) + 1024, 1024
    narrow = torch.zeros(2 * n + n // 32, dtype=torch.uint8, device="cuda")
    rng = np.random.RandomState(2)
    starts = (0, (1 << 32) - k, n - k)
    want = {}
    for at in starts:
        codes = [rng.randint(0, 8 * top + 7, k).astype(np.uint8) for top in (15, 31)]
        exps = [rng.randint(100, 140, k // 64).astype(np.uint8) for _ in range(2)]
        for c, e in zip(codes, exps):   # a block's exponent is that of its largest
            c[::64] = 8 * (15 if c is codes[0] else 31)
        for i, (c, e) in enumerate(zip(codes, exps)):
            narrow[i * n + at:i * n + at + k] = torch.from_numpy(c).cuda()
            first = 2 * n + i * (n // 64) + at // 64
            narrow[first:first + k // 64] = torch.from_numpy(e).cuda()
            want[i, at] = S8.decode(c, e, 15 if i == 0 else 31)
    wide = torch.full((2 * n,), -7.0, device="cuda")
    P.fl_state_convert(narrow, wide)
    for (i, at), x in want.items():
        part = wide[i * n + at:i * n + at + k]
        assert np.array_equal(part.cpu().numpy(), x), (i, at)
    back = torch.full_like(narrow, 99)
    P.fl_state_convert(wide, back)
    for (i, at), x in want.items():
        c, e = S8.encode(x, 15 if i == 0 else 31)
        first = 2 * n + i * (n // 64) + at // 64
        assert np.array_equal(back[i * n + at:i * n + at + k].cpu().numpy(), c), (i, at)
        assert np.array_equal(back[first:first + k // 64].cpu().numpy(), e), (i, at)
        wide[i * n + at:i * n + at + k] = 0.0
    for at in range(0, 2 * n, 1 << 30):
        assert not bool(wide[at:at + (1 << 30)].any()), at
