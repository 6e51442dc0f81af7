"""The main attention kernel on every page size over some thousand keys, shared and of a
sequence's own, with lengths off its units, one row to several tiles of them; and over the
last pages of a pool of more than 4 GB."""
import numpy as np
import pytest
import torch

from oracle import pages as OP
from pages_common import Both, check_attend, i32

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _run(ldr, c, hq, new, groups=None):
    q = c.rand(c.batch, new, hq, c.g.d)
    out = torch.full_like(q, 2.0)
    lse = torch.full(q.shape[:3], 2.0, device="cuda")
    ldr.attend(c.g.plan(hq, new, groups=groups), 0, q, out=out, lse=lse)
    torch.cuda.synchronize()
    assert c.g.status() == ldr.LDR_OK
    check_attend(c, new, q, out, lse, 0, c.g.d ** -0.5, 2.0)


@pytest.mark.parametrize("dtype,d,page", [
    (BF, 128, 32), (BF, 64, 32), (BF, 128, 64), (BF, 64, 128), (BF, 128, 256), (BF, 64, 256),
    (F32, 128, 256), (F32, 64, 32)])
@pytest.mark.parametrize("hq,hkv,new", [(4, 1, 1), (4, 2, 17), (8, 1, 70)])
def test_long_fronts_and_long_rests(gpu_lib, dtype, d, page, hq, hkv, new):
    """Three samples of 2999 rows, two of them more than a thousand rows further, beside a
    stranger of 2300 rows and a fresh prompt."""
    c = Both(gpu_lib, 1, hkv, d, page, 12800 // page, 5, 6400 // page, dtype, seed=page + new)
    c.append([2999, 0, 0, 2300, 0])
    c.fork([0, 0, 0, 3, 4])
    c.append([1283, 7, 1100, 0, 0])
    c.append([new, max(1, new - 1), new, new, new])
    _run(gpu_lib, c, hq, new)
    _run(gpu_lib, c, hq, new, groups=i32([-1] * 5))


@pytest.mark.parametrize("dtype,d,page", [(BF, 128, 32), (BF, 128, 64), (BF, 64, 256), (F32, 64, 64)])
def test_fresh_prompts(gpu_lib, dtype, d, page):
    """Nothing but open rows: eight tiles of 256 with masks at every length, and one row."""
    c = Both(gpu_lib, 1, 1, d, page, 2048 // page + 2, 2, 2048 // page, dtype, seed=1)
    c.append([1021, 1])
    _run(gpu_lib, c, 2, 1021)


def test_last_pages_of_a_large_pool(gpu_lib):
    """Keys and values behind 2^32 bytes of the pool, and of its layer."""
    p = gpu_lib.Pages(2, 8, 128, 256, 10240, 1, 16).init()
    assert p.pool[0].numel() * 2 > 1 << 32
    p.refs[:10236] = 1                   # all but the last four pages are taken
    K, V = (torch.randn(1, 1000, 2, 8, 128, device="cuda").to(BF) for _ in range(2))
    p.append(i32([995]), K[:, :995].contiguous(), V[:, :995].contiguous())
    p.append(i32([5]), K[:, 995:].contiguous(), V[:, 995:].contiguous())
    assert p.table[0, :4].tolist() == [10236, 10237, 10238, 10239]
    q = torch.randn(1, 5, 8, 128, device="cuda").to(BF)
    plan = p.plan(8, 5)
    f = lambda x: x.double().cpu().numpy()  # noqa: E731
    for layer in range(2):
        got = f(gpu_lib.attend(plan, layer, q))[0]
        want, _ = OP.attend(f(q)[0], f(K)[0, :, layer], f(V)[0, :, layer], 128 ** -0.5)
        size, _ = OP.attend(f(q)[0], f(K)[0, :, layer], np.abs(f(V)[0, :, layer]), 128 ** -0.5)
        # probabilities and result to bf16, half a step each; 1.1e-3 for all sums and scores in
        # fp32 (1000 keys, scores below 20: 2 (1000 + 3 x 134 x 20) 2^-24 = 1.1e-3, an upper bound)
        assert np.all(np.abs(got - want) <= (2.0 ** -8 + 1.1e-3) * size + 2.0 ** -8 * np.abs(want))
    assert p.status() == gpu_lib.LDR_OK
