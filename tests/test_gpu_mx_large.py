"""Coded pools and logits of more bytes than 32 bits count."""
import numpy as np
import pytest
import torch

from oracle import pages as OP
from pages_common import i32

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_pages_behind_4_gb(gpu_lib):
    """A pool of 9 GB whose sequences have its last pages: rows in, rows out, attention."""
    n_pages, page, hkv, d = 70000, 64, 8, 128
    p = gpu_lib.Pages(1, hkv, d, page, n_pages, 2, 20, codes="mxfp8").init()
    assert p.pool.numel() > 2 * (1 << 32)
    # all pages but the last thirty are held by somebody
    p.refs[:n_pages - 30] = 1
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = [900, 333]
    K, V = (torch.randn(2, 900, 1, hkv, d, generator=g, device="cuda").to(BF) for _ in range(2))
    p.append(i32(rows), K, V)
    assert p.table[0, 0] == n_pages - 30 and p.status() == gpu_lib.LDR_OK
    k, v = p.read(i32([0, 0]), i32(rows), 900)
    for got, x in ((k, K), (v, V)):
        for b, n in enumerate(rows):
            ref = OP.mx_values(x[b, :n].double().cpu().numpy(), 8)
            assert np.array_equal(got[b, :n].double().cpu().numpy(), ref)
    # the same rows in a small pool: the same bits
    s = gpu_lib.Pages(1, hkv, d, page, 30, 2, 20, codes="mxfp8").init()
    s.append(i32(rows), K, V)
    for c in (p, s):
        c.keep(i32([900, 333]))
    new, q = i32([3, 3]), torch.randn(2, 3, 16, d, generator=g, device="cuda").to(BF)
    more = torch.randn(2, 3, 1, hkv, d, generator=g, device="cuda").to(BF)
    outs = []
    for c in (p, s):
        c.append(new, more, more)
        outs.append(gpu_lib.attend(c.plan(16, 3), 0, q))
    torch.cuda.synchronize()
    assert torch.equal(*outs) and bool(outs[0].any())


def test_rows_of_logits_behind_4_gb(gpu_lib):
    """Rows 2^28 entries apart."""
    V, far = 5003, 1 << 28
    z = torch.empty(4 * far + V, device="cuda")
    rows = torch.as_strided(z, (1, 5, V), (5 * far, far, 1))
    rows.copy_(torch.randn(1, 5, V, device="cuda"))
    y = i32([[1, 2, 3, 4, 5]])
    a = gpu_lib.logprobs(rows, y, top_n=5)
    b = gpu_lib.logprobs(rows.contiguous(), y, top_n=5)
    torch.cuda.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(a, b)) and bool(a[0].all())
