"""Rows into a coded cache and back, exactly as the oracle codes them; reads of
any cache; forks, releases and compactions of coded pages; refused ranges."""
import numpy as np
import pytest
import torch

from mx_common import BothCoded
from pages_common import Both, i32

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

SHAPES = [(1, 64, 32), (2, 128, 64), (3, 64, 128), (1, 128, 256)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hkv,d,page", SHAPES)
def test_rows_come_back_as_their_codes(gpu_lib, bits, hkv, d, page):
    """Appends that begin and end anywhere in a page and in a run of 16 positions."""
    c = BothCoded(gpu_lib, bits, 2, hkv, d, page, 64, 5, 14, seed=bits)
    for n in ([1, 15, 16, 17, 0], [31, 32, 33, 7, 1], [0, 1, 100, 70, 16], [5, 0, 3, 2, 300 % page]):
        c.append(n)
        c.check()
    assert c.g.status() == gpu_lib.LDR_OK


@pytest.mark.parametrize("bits", [4, 8])
def test_values_at_the_edges_of_the_codes(gpu_lib, bits):
    """Every half-way point between two codes and its neighbours, blocks of one value
    a binade and more, zeros of both signs, the smallest and the largest numbers."""
    from oracle import pages as OP
    grid, limit, lowest, top = OP.MX[bits]
    mid = [(a + b) / 2 for a, b in zip(grid, grid[1:])] + [limit]
    rows = []
    for s in (1.0, 2.0 ** -100, 2.0 ** 60):
        for t in mid + grid:
            for f in (1.0, 1 - 2.0 ** -8, 1 + 2.0 ** -7):
                row = np.zeros(64)
                row[0], row[1], row[2] = grid[-1] * s, t * f * s, -t * s
                row[32], row[33] = t * f * s, -t * f * s / 3
                rows.append(row)
    tiny = float(np.float32(2.0 ** -133))
    for a in (0.0, tiny, 5 * tiny, 2.0 ** -126, 3 * 2.0 ** -126, 2.0 ** (lowest - 1), 2.0 ** lowest,
              limit * 2.0 ** lowest, 2.0 ** 127, 1.5 * 2.0 ** 127, 1.875 * 2.0 ** 127,
              1.9921875 * 2.0 ** 127):
        row = np.zeros(64)
        row[5], row[6], row[40] = a, -a, -a / 2
        rows.append(row)
    rows.append(np.full(64, -0.0))
    X = torch.tensor(np.stack(rows)).to(BF)
    n = len(X)
    K = X.view(1, n, 1, 1, 64).cuda()
    c = BothCoded(gpu_lib, bits, 1, 1, 64, 64, n // 64 + 2, 1, n // 64 + 2)
    c.append([n], n, K, -K)
    c.check()
    k, v = c.g.read(i32([0]), i32([n]), n)
    assert bool(torch.isfinite(k).all()) and torch.equal(k, -v)
    # half a step at most
    half = 2.0 ** (-2 if bits == 4 else -4)
    err = (k - K).abs().double().view(n, 2, 32)
    big = K.abs().double().view(n, 2, 32)
    within = big <= top
    low = big.amax(-1, keepdim=True).clamp(min=limit * 2.0 ** lowest) / limit * 2.0
    step = torch.maximum(half * big, low * (0.25 if bits == 4 else 2.0 ** -10))
    assert bool((err <= step)[within].all())


@pytest.mark.parametrize("bits", [4, 8])
def test_values_that_are_not_finite(gpu_lib, bits):
    """Their block is NaN, the others of the row and of its page are not."""
    c = BothCoded(gpu_lib, bits, 1, 2, 128, 32, 8, 1, 8)
    K, V = c.rand(1, 40, 1, 2, 128), c.rand(1, 40, 1, 2, 128)
    K[0, 3, 0, 1, 40] = float("nan")
    K[0, 33, 0, 0, 0] = float("inf")
    V[0, 4, 0, 0, 127] = -float("inf")
    V[0, 5, 0, 1, 64:] = float("nan")
    c.append([40], 40, K, V)
    c.check()
    k, v = c.g.read(i32([0]), i32([40]), 40)
    assert int(k.isnan().sum()) == 64 and int(v.isnan().sum()) == 32 + 64


@pytest.mark.parametrize("bits", [4, 8])
def test_forks_releases_and_compactions(gpu_lib, bits):
    """Whole pages move with their scales; a sharer's rows do not touch the others'."""
    c = BothCoded(gpu_lib, bits, 2, 2, 64, 32, 60, 4, 12, seed=3)
    c.append([70, 40, 0, 5])
    c.fork([0, 1, 0, 0])
    c.append([9, 3, 20, 40])
    c.check()
    c.keep([2, 0, 20, 7])
    c.check()
    c.append([40, 1, 0, 33])
    c.fork([0, -1, 2, 3])
    c.check()
    c.compact()
    c.check()
    c.append([3, 30, 3, 3])
    c.check()


@pytest.mark.parametrize("bits", [4, 8])
def test_layers_apart(gpu_lib, bits):
    """Layers written one by one are as those written together."""
    c = BothCoded(gpu_lib, bits, 3, 2, 128, 64, 20, 2, 8, seed=4)
    n, K, V = [21, 90], c.rand(2, 90, 3, 2, 128), c.rand(2, 90, 3, 2, 128)
    c.g.reserve(i32(n), 90)
    c.o.reserve(n, 90)
    for at, m in ((2, 1), (0, 2)):
        k, v = K[:, :, at:at + m].contiguous(), V[:, :, at:at + m].contiguous()
        c.g.write(k, v, layer=at)
        c.o.write(k.double().cpu().numpy(), v.double().cpu().numpy(), at)
    c.check()
    k, v = c.g.read(i32([0, 0]), i32(n), 90, layer=1, n_layers=1)
    k2, v2 = c.g.read(i32([0, 0]), i32(n), 90)
    assert torch.equal(k, k2[:, :, 1:2]) and torch.equal(v, v2[:, :, 1:2])


def test_a_row_does_not_depend_on_others(gpu_lib):
    """One row a call, or all in one."""
    got = []
    for each in (1, 37):
        c = BothCoded(gpu_lib, 4, 1, 1, 64, 32, 4, 1, 4, seed=5)
        K, V = c.rand(1, 37, 1, 1, 64), c.rand(1, 37, 1, 1, 64)
        for at in range(0, 37, each):
            c.append([each], each, K[:, at:at + each].contiguous(), V[:, at:at + each].contiguous())
        c.check()
        got.append(c.g.read(i32([0]), i32([37]), 37))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("held", [BF, F32, 4, 8])
@pytest.mark.parametrize("d,page", [(64, 32), (128, 64), (64, 256)])
def test_reads_of_ranges(gpu_lib, held, d, page):
    """Ranges that begin and end anywhere, of none and of one row; what lies behind them
    in the outputs stays."""
    if held in (4, 8):
        c = BothCoded(gpu_lib, held, 2, 2, d, page, 40, 6, 10, seed=6)
    else:
        c = Both(gpu_lib, 2, 2, d, page, 40, 6, 10, held, seed=6)
    c.append([100, 200, 1, 64, 33, 0])
    for first, n in (([0, 0, 0, 0, 0, 0], [100, 200, 1, 64, 33, 0]),
                     ([99, 57, 0, 31, 32, 0], [1, 101, 1, 33, 1, 0]),
                     ([17, 200, 1, 63, 5, 0], [48, 0, 0, 1, 9, 0])):
        most = max(n) + 3
        out = tuple(torch.full((6, most, 2, 2, d), 9.0, dtype=c.dtype, device="cuda")
                    for _ in range(2))
        K, V = c.g.read(i32(first), i32(n), out=out)
        for layer in range(2):
            for b in range(6):
                ok, ov = c.o.sequence(layer, b)
                for got, ref in ((K, ok), (V, ov)):
                    x = got[b, :, layer].double().cpu().numpy()
                    assert np.array_equal(x[:n[b]], ref[first[b]:first[b] + n[b]]), (layer, b)
                    assert np.all(x[n[b]:] == 9.0), b
    assert c.g.status() == gpu_lib.LDR_OK


@pytest.mark.parametrize("held", [BF, 4])
def test_ranges_outside_a_sequence_are_left_out(gpu_lib, held):
    c = (BothCoded(gpu_lib, 4, 1, 1, 64, 32, 20, 4, 4) if held == 4
         else Both(gpu_lib, 1, 1, 64, 32, 20, 4, 4, held))
    c.append([40, 40, 40, 40])
    big = 2 ** 31 - 1
    for first, n in (([-1, 0, 0, 0], [2, 4, 4, 4]), ([37, 0, 0, 0], [4, 4, 4, 4]),
                     ([0, 0, 0, 0], [-1, 4, 4, 4]), ([0, 0, 0, 0], [9, 4, 4, 4]),
                     ([big, 0, 0, 0], [8, 4, 4, 4]), ([-big, 0, 0, 0], [8, 4, 4, 4])):
        K, V = c.g.read(i32(first), i32(n), 8)
        assert not K[0].any() and not V[0].any()
        ok, ov = c.o.sequence(0, 2)
        assert np.array_equal(K[2, :4, 0].double().cpu().numpy(), ok[:4])
        assert np.array_equal(V[2, :4, 0].double().cpu().numpy(), ov[:4])
        assert c.g.status(clear=True) == gpu_lib.LDR_ERANGE
    assert c.g.status() == gpu_lib.LDR_OK


def test_reads_over_each_other_are_refused(gpu_lib):
    c = BothCoded(gpu_lib, 4, 1, 1, 64, 32, 8, 1, 4)
    c.append([5])
    both = torch.zeros(1, 9, 1, 1, 64, dtype=BF, device="cuda")
    for K, V in ((both[:, :5], both[:, :5]), (both[:, :5], both[:, 4:]), (both[:, 4:], both[:, :5])):
        with pytest.raises(gpu_lib.LdrError) as e:
            c.g.read(i32([0]), i32([5]), out=(K, V))
        assert e.value.code == gpu_lib.LDR_EINVAL
    c.g.read(i32([0]), i32([4]), out=(both[:, :4], both[:, 4:8]))
    torch.cuda.synchronize()
    assert bool(both[:, :8].any()) and not both[:, 8].any()
