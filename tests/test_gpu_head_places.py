"""The output head with inputs at places of their own: a weight that starts
between two 16-byte boundaries, hidden states far apart."""
import pytest

from test_gpu_head import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_20359_amd as P

    P.lib()
    return dict(torch=torch, P=P)


@pytest.mark.parametrize("K", [0, 5])
@pytest.mark.parametrize("off", [1, 3, 8, 65])
@pytest.mark.parametrize("V,D,ld", [(500, 65, 65), (300, 64, 67), (700, 31, 32)])
def test_weight_rows_off_sixteen_bytes(env, V, D, ld, off, K):
    """A head inside a flat array, as a shard's segment is: rows that are copied
    are taken from any element on."""
    torch = env["torch"]
    c = Case(torch, 40, V, D, K=K)
    flat = torch.full((off + V * ld,), float("nan"), dtype=torch.bfloat16, device="cuda")
    view = flat[off:].view(V, ld)[:, :D]
    view.copy_(c.w)
    c.w = view
    c.check(env["P"])


@pytest.mark.parametrize("K", [0, 5])
def test_last_tokens_of_long_sequences(env, K):
    """hidden[:, -1] of 3-D states: rows a whole sequence apart, some of them
    past 32 bits of bytes."""
    torch = env["torch"]
    T, D, length = 40, 64, 1 << 20
    c = Case(torch, T, 300, D, K=K)
    states = torch.empty(T, length, D, dtype=torch.bfloat16, device="cuda")
    states[:, -1] = c.h
    c.h = states[:, -1]
    assert c.h.stride(0) == length * D > 1 << 22
    c.check(env["P"])
