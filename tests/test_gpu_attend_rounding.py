"""Rounding of the running softmax that a long row would add up."""
import pytest
import torch

from pages_common import i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("raw", [56440.0, 63384.0])
def test_equal_scores_of_a_long_row(gpu_lib, d, raw):
    """512 rows, each alone, over the same 16384 keys of one score, and values k / n: the
    result is their mean. Scores are dyadic, so exact, and every key's weight is the same
    number; what is left are the sums, of 16384 / 4 keys each before the waves and parts are
    joined: (n / 4 + 64) 2^-24 relative of either, and the division."""
    n, b = 16384, 512
    p = gpu_lib.Pages(1, 1, d, 64, 256 + b, b, 256, torch.float32).init()
    v = (torch.arange(n, device="cuda") / n).view(n, 1, 1, 1).expand(n, 1, 1, d)
    V = torch.zeros(b, n - 1, 1, 1, d, device="cuda")
    V[0] = v[:n - 1]
    p.append(i32([n - 1] + [0] * (b - 1)), torch.full_like(V, raw / d), V)
    del V
    p.fork(i32([0] * b))
    p.append(i32([1] * b), torch.full((b, 1, 1, 1, d), raw / d, device="cuda"),
             v[n - 1].expand(b, 1, 1, 1, d).contiguous())
    q = torch.ones(b, 1, 1, d, device="cuda")
    out = gpu_lib.attend(p.plan(1, 1, groups=i32([-1] * b)), 0, q, scale=0.125)
    assert p.status() == gpu_lib.LDR_OK
    mean = (n - 1) / (2 * n)
    off = (out.double() - mean).abs().max().item()
    assert off <= mean * (2 * (n / 4 + 64) + 2) * 2.0 ** -24, off
