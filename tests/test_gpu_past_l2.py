"""The embedding, the norm and their gradients on arrays of more than 32 MiB, which are read
and written past the caches by kernels of their own: the checks and tolerances of
test_gpu_embed.py and test_gpu_norm.py at such sizes, each number of waves and chunks to a
row among them."""
import pytest

import test_gpu_embed as E
from test_gpu_embed import env, framed  # noqa: F401
from test_gpu_norm import Case

pytestmark = pytest.mark.gpu

PAST = 32 << 20


def size(dtype):
    return 2 if dtype == "bf16" else 4


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [8, 640, 2001, 4096])
@pytest.mark.parametrize("scale,pad", [(1.0, 0), (3.7, 3)])
def test_embed(env, D, dtype, scale, pad):  # noqa: F811
    torch, P = env["torch"], env["P"]
    V, T = 3000, min(1 << 20, PAST // (D * size(dtype)) + 77)
    if D == 8:
        T = 1 << 20                # (16 MiB of bf16: the largest of 8 columns)
    ids, w, _ = E.make(torch, T, V, D, dtype, pad=pad)
    out, untouched = framed(torch, (T, D), w.dtype)
    P.fl_embed(ids, w, out, scale=scale)
    rows = (w[ids.clamp(0, V - 1)].float() * scale).to(w.dtype)
    ok = torch.where((ids < 0)[:, None], out == 0.0, out == rows)
    assert bool(torch.where((ids >= V)[:, None], out.isnan(), ok).all())
    untouched()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("T,V", [(9000, 300), (700, 9000), (9000, 9000), (20000, 9001)])
@pytest.mark.parametrize("D", [1000, 2001])
def test_embed_grad(env, T, V, D, dtype, add):  # noqa: F811
    """Gradients of the output, the table, or both, past the caches (or, in fp32, with 1000
    columns; in bf16 those of 2001)."""
    ids, _, d = E.make(env["torch"], T, V, D, dtype, pad=5)
    E.check_grad(env, ids, d, V, 1.0, add)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("D", [64, 250, 500, 1000, 1601, 2048, 2500, 4096, 5000, 8192])
def test_norm(env, D, rms, dtype):  # noqa: F811
    R = PAST // (D * size(dtype)) + 33
    c = Case(env["torch"], R, D, dtype, rms, pad=3 if D % 8 else 0)
    c.check_forward(env["P"])
    c.check_backward(env["P"])
