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
    if n:
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


@pytest.mark.parametrize("dtype,d,page", FORMS)
@pytest.mark.parametrize("n", [40, 1100])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_keys_without_weight(gpu_lib, dtype, d, page, n, bad):
    """One key's score is -inf and some of its values are not finite: 0 x inf is NaN, in
    whichever kernel the key is; the other values of the rows are as without the key."""
    new = 5
    for at in (7, n - 1, n + 2):
        K, V = _rand(dtype, 1, n + new, 1, 2, d, seed=1), _rand(dtype, 1, n + new, 1, 2, d, seed=2)
        K[0, at] = -INF
        V[0, at, 0, 1, ::3] = bad
        c = _cache(gpu_lib, dtype, d, page, n, new, K, V)
        q = _rand(dtype, 1, new, 4, d, seed=3).abs() + 0.1
        out, _ = _attend(gpu_lib, c, q)
        sees = max(0, at - n)                        # the first open row that sees the key
        assert torch.isnan(out[0, sees:, 2:, ::3]).all()
        assert torch.isfinite(out[0, :sees]).all() and torch.isfinite(out[0, :, :2]).all()


@pytest.mark.parametrize("dtype,d,page", FORMS)
@pytest.mark.parametrize("n,new,which,bad", [
    (n, new, w, x) for n, new in ((40, 5), (1100, 5)) for w in ("K", "V", "KV") for x in (INF, -INF, NAN)
] + [(n, new, w, x) for n, new in ((1100, 150), (0, 700)) for w, x in (("K", NAN), ("V", INF), ("KV", -INF))])
def test_keys_that_are_not_finite(gpu_lib, dtype, d, page, n, new, bad, which):
    """A key or values of a long past (the main kernel's) and of open rows: every row
    against the definition, with few rows, several tiles of them, and a fresh prompt. A
    score of inf or NaN leaves NaN in the rows that see it."""
    K, V = _rand(dtype, 1, n + new, 1, 2, d, seed=4), _rand(dtype, 1, n + new, 1, 2, d, seed=5)
    for at in ([n // 2] if n else [new // 2]) + [n + new // 3]:
        if "K" in which:
            K[0, at, 0, 0] = bad
        if "V" in which:
            V[0, at, 0, 0, 1::5] = bad
    c = _cache(gpu_lib, dtype, d, page, n, new, K, V)
    q = _rand(dtype, 1, new, 4, d, seed=6).abs() + 0.1
    out, _ = _attend(gpu_lib, c, q)
    assert torch.isfinite(out[0, :, 2:]).all()       # the other K/V head


def test_queries_in_the_place_of_the_results(gpu_lib):
    """Values that are not finite, and o over q: as into a buffer of its own."""
    n, new, d = 40, 40, 128
    K, V = _rand(BF, 1, n + new, 1, 2, d, seed=7), _rand(BF, 1, n + new, 1, 2, d, seed=8)
    K[0, 60], V[0, 60, 0, :, ::2], V[0, 50, 0, :, 1] = -INF, INF, NAN
    c = _cache(gpu_lib, BF, d, 64, n, new, K, V)
    q = _rand(BF, 1, new, 8, d, seed=9).abs() + 0.1
    out, _ = _attend(gpu_lib, c, q)
    gpu_lib.attend(c.g.plan(8, new), 0, q, out=q)
    torch.cuda.synchronize()
    assert torch.equal(q.view(torch.int16), out.view(torch.int16))
