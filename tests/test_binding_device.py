"""The binding refuses memory of another device than the current one, and a stream of
another, before it calls the library: the kernels would run on the wrong GPU."""
import types

import pytest
import torch


@pytest.fixture
def ldr(monkeypatch):
    """The binding, with a current device that no memory here is on."""
    from paper_2609_37029_amd import ldr as L
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(L, "_on_gpu", lambda *a: None)
    return L


def _refused(L, call):
    with pytest.raises(L.LdrError, match="current device 3") as e:
        call()
    assert e.value.code == L.LDR_EINVAL


def test_memory_of_another_device(ldr):
    L, B = ldr, 3
    p = L.Pages(2, 2, 64, 32, 8, B, 4, torch.float32, device="cpu")
    i32 = torch.zeros(B, dtype=torch.int32)
    K = torch.zeros(B, 4, 2, 2, 64)
    for call in (p.init, lambda: p.reserve(i32, 4), lambda: p.write(K, K), lambda: p.append(i32, K, K),
                 lambda: p.keep(i32), lambda: p.fork(i32), p.compact, p.status,
                 lambda: p.plan(4, 4, groups=i32)):
        _refused(L, call)
    plan = types.SimpleNamespace(pages=p, n_q_heads=4, max_new=4, workspace=torch.zeros(1))
    q = torch.zeros(B, 4, 4, 64)
    _refused(L, lambda: L.attend(plan, 0, q))
    P, y, u = torch.zeros(2, 4, 9), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 4)
    _refused(L, lambda: L.verify_probs(P, None, y, u))
    v = types.SimpleNamespace(batch=B, arena=K, _stream=None, _h=None)
    _refused(L, lambda: L.Views.fork(v, i32))


def test_stream_of_another_device(ldr):
    L = ldr
    dev, s = torch.device("cuda", 3), types.SimpleNamespace(device_index=2, cuda_stream=64)
    _refused(L, lambda: L._stream(s, dev))
    s.device_index = 3
    assert L._stream(s, dev).value == 64
    _refused(L, lambda: L._stream(s, torch.device("cuda", 2)))
    assert L._stream(s).value == 64
