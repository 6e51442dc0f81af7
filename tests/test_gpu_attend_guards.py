"""What an attention refuses on the device: plans of another cache, of another
handle, and of a cache that was reset in between. Each leaves the output as it was
and sets the status."""
import ctypes

import pytest
import torch

from pages_common import Both, check_attend

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _cache(ldr, batch, dtype, d=64, hkv=1, page=32, seed=0):
    """A cache that has counted as many changes as any other made here."""
    c = Both(ldr, 1, hkv, d, page, 40 * batch, batch, 40, dtype, seed=seed)
    c.g.state.zero_()
    c.g.init()
    c.append([700 + b for b in range(batch)])
    c.append([3] * batch)
    return c


def _refused(ldr, c, plan, q):
    out = torch.full(q.shape, 3.0, dtype=c.dtype, device="cuda")
    lse = torch.full(q.shape[:3], 3.0, device="cuda")
    assert c.g.status(clear=True) == ldr.LDR_OK
    ldr.attend(plan, 0, q, out=out, lse=lse)
    assert c.g.status(clear=True) == ldr.LDR_EINVAL
    assert torch.all(out == 3.0) and torch.all(lse == 3.0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("other", [dict(batch=2), dict(batch=7), dict(batch=2, page=256),
                                   dict(batch=2, d=128, hkv=2)])
def test_plan_of_another_cache(gpu_lib, dtype, other):
    """Two caches that went through the same calls share a workspace."""
    a, b = _cache(gpu_lib, 2, dtype, seed=1), _cache(gpu_lib, dtype=dtype, seed=2, **other)
    hq = 4
    ws = torch.empty(max(x.g.attend_workspace_bytes(hq, 3) for x in (a, b)), dtype=torch.uint8,
                     device="cuda")
    plan_a = a.g.plan(hq, 3, workspace=ws)
    q = a.rand(2, 3, hq, a.g.d)
    out = torch.zeros_like(q)
    gpu_lib.attend(plan_a, 0, q, out=out)
    torch.cuda.synchronize()
    check_attend(a, 3, q, out, None, 0, a.g.d ** -0.5)
    plan_b = b.g.plan(hq, 3, workspace=ws)
    _refused(gpu_lib, a, plan_a, q)
    q = b.rand(b.batch, 3, hq, b.g.d)
    out = torch.zeros_like(q)
    gpu_lib.attend(plan_b, 0, q, out=out)
    assert b.g.status() == gpu_lib.LDR_OK
    check_attend(b, 3, q, out, None, 0, b.g.d ** -0.5)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_plan_kept_over_a_reset(gpu_lib, dtype):
    """As many calls after the reset as before the plan: a new handle of the same object,
    and the old handle of a state that another one reset."""
    a = _cache(gpu_lib, 2, dtype)
    plan = a.g.plan(4, 3)
    q = a.rand(2, 3, 4, 64)
    a.g.init()
    n = torch.tensor([300, 300], dtype=torch.int32, device="cuda")
    for _ in range(2):
        a.g.reserve(n, 300)
    _refused(gpu_lib, a, plan, q)
    a = _cache(gpu_lib, 2, dtype)
    plan = a.g.plan(4, 3)
    h, lib = ctypes.c_void_p(), gpu_lib.lib()
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    assert lib.ldr_pages_init(ctypes.byref(h), ctypes.byref(a.g.cfg), ptr(a.g.pool), ptr(a.g.state),
                              stream) == gpu_lib.LDR_OK
    for _ in range(2):
        assert lib.ldr_pages_reserve(h, ptr(n), 300, stream) == gpu_lib.LDR_OK
    _refused(gpu_lib, a, plan, q)
    torch.cuda.synchronize()
    lib.ldr_pages_destroy(h)


def test_plan_of_a_state_put_back(gpu_lib):
    """A state that was saved goes on where it was, on a handle made since then too; its
    attention needs a plan of that handle."""
    a = _cache(gpu_lib, 2, BF)
    saved = a.g.state.clone()
    q = a.rand(2, 3, 4, 64)
    old = a.g.plan(4, 3)
    a.g.init()
    a.g.state.copy_(saved)
    _refused(gpu_lib, a, old, q)
    out = torch.zeros_like(q)
    gpu_lib.attend(a.g.plan(4, 3), 0, q, out=out)
    assert a.g.status() == gpu_lib.LDR_OK
    check_attend(a, 3, q, out, None, 0, 0.125)


def test_scales(gpu_lib):
    """A scale whose product with log2(e) is no fp32 number is refused; the largest ones
    that are not give what the definition does."""
    a = _cache(gpu_lib, 2, F32)
    q = a.rand(2, 3, 4, 64)
    out = torch.full_like(q, 3.0)
    for scale in (3e38, 2.0 ** 127 * 1.5):
        with pytest.raises(gpu_lib.LdrError) as e:
            gpu_lib.attend(a.g.plan(4, 3), 0, q, out=out, scale=scale)
        assert e.value.code == gpu_lib.LDR_EINVAL and torch.all(out == 3.0)
    q *= 2.0 ** -120
    out = torch.zeros_like(q)
    gpu_lib.attend(a.g.plan(4, 3), 0, q, out=out, scale=2.0 ** 117)
    torch.cuda.synchronize()
    check_attend(a, 3, q, out, None, 0, 2.0 ** 117)
    gpu_lib.attend(a.g.plan(4, 3), 0, q * 0, out=out, scale=2.0 ** 127)
    torch.cuda.synchronize()
    check_attend(a, 3, q * 0, out, None, 0, 2.0 ** 127)
