"""Attention over values that are not finite, in the kernel with the masks and in the
main one, against the definition: a row without weight is 0; a key without weight
gives 0 x inf; what a row does not see does not count."""
import pytest
import torch

from pages_common import Both, check_attend

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")
# head dim, page; both of the main kernel's page forms
FORMS = [(BF, 64, 32), (BF, 128, 64), (BF, 128, 32), (BF, 64, 256), (F32, 64, 64), (F32, 128, 32)]


def _attend(ldr, c, q, before=5.0):
    """Outputs of layer 0, checked but for rows that K leaves undefined."""
    shape = q.shape
    out = torch.full(shape, before, dtype=c.dtype, device="cuda")
    lse = torch.full(shape[:3], before, device="cuda")
    ldr.attend(c.g.plan(shape[2], shape[1]), 0, q, out=out, lse=lse)
    torch.cuda.synchronize()
    assert c.g.status() == ldr.LDR_OK
    check_attend(c, shape[1], q, out, lse, 0, shape[3] ** -0.5, before)
    return out, lse


def _cache(ldr, dtype, d, page, n, new, K, V, seed=0):
    """One sequence of n rows, then new open ones; K and V hold all of them."""
    c = Both(ldr, 1, 2, d, page, (n + new) // page + 2, 1, (n + new) // page + 2, dtype, seed=seed)
    c.append([n], K=K[:, :n].contiguous(), V=V[:, :n].contiguous())
    c.append([new], K=K[:, n:].contiguous(), V=V[:, n:].contiguous())
    return c


def _rand(dtype, *shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype,d,page", FORMS)
@pytest.mark.parametrize("n", [40, 1100])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_rows_without_weight_are_zero(gpu_lib, dtype, d, page, n, bad):
    """Every score -inf and values that are not finite, at a key that only the last kernel
    takes, at one of the main kernel's (n = 1100) and at an open row's."""
    new = 5
    K = torch.full((1, n + new, 1, 2, d), -INF, dtype=dtype, device="cuda")
    for at in (7, n - 1, n + 2):
        V = _rand(dtype, 1, n + new, 1, 2, d)
        V[0, at, 0, 1, ::3] = bad
        c = _cache(gpu_lib, dtype, d, page, n, new, K, V)
        q = torch.ones(1, new, 4, d, dtype=dtype, device="cuda")
        out, lse = _attend(gpu_lib, c, q)
        assert torch.all(out == 0) and torch.all(lse == -INF)
