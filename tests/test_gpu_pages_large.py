"""Tables and pools of more words and bytes than 32 bits count."""
import pytest
import torch

from pages_common import i32

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_tables_of_more_than_2_32_words(gpu_lib):
    """A state of 17 GB is reset to its end, and its last sequence gets pages."""
    b, most = 129, (1 << 25) - 1
    p = gpu_lib.Pages(1, 1, 64, 32, 8, b, most, BF)
    assert p.table.numel() > 1 << 32
    p.state.fill_(7)
    p.init()
    assert p.status() == gpu_lib.LDR_OK
    for at in range(0, b, 43):
        assert int(p.table[at:at + 43].max()) == -1 == int(p.table[at:at + 43].min())
    assert not p.rows.any() and not p.open.any() and not p.refs.any()
    n = i32([0] * (b - 1) + [40])
    K = torch.randn(b, 40, 1, 1, 64, device="cuda").to(BF)
    p.append(n, K, -K)
    p.fork(i32([b - 1] + list(range(1, b))))
    assert p.status() == gpu_lib.LDR_OK
    assert p.rows.tolist() == [40] + [0] * (b - 2) + [40] and p.refs[:3].tolist() == [2, 2, 0]
    for at in (0, b - 1):
        assert p.table[at, :3].tolist() == [0, 1, -1]
    k = p.k(0)[:2].transpose(1, 2).reshape(64, 1, 64)[:40]
    assert torch.equal(k, K[b - 1, :, 0])
