"""The binding refuses memory of another device than the current one for reads of cache rows,
coded caches and log probabilities, as for the other calls (test_binding_device.py)."""
import torch

from test_binding_device import _refused, ldr  # noqa: F401


def test_memory_of_another_device(ldr):  # noqa: F811
    B, i32 = 3, torch.zeros(3, dtype=torch.int32)
    for codes in (None, "mxfp4", "mxfp8"):
        p = ldr.Pages(2, 2, 64, 32, 8, B, 4, device="cpu", codes=codes)
        K = torch.zeros(B, 4, 2, 2, 64, dtype=torch.bfloat16)
        _refused(ldr, p.init)
        _refused(ldr, lambda: p.read(i32, i32, 4))
        _refused(ldr, lambda: p.read(i32, i32, out=(K, K.clone())))
        _refused(ldr, lambda: p.append(i32, K, K))
    z, y = torch.zeros(2, 3, 70), torch.zeros(2, 3, dtype=torch.int32)
    _refused(ldr, lambda: ldr.logprobs(z, y, top_n=5))
    _refused(ldr, lambda: ldr.logprobs(z, y))
