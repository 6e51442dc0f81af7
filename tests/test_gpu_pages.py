"""The paged cache on the GPU against its plain form: tables, counts and every
row, bit for bit (the calls copy and count)."""
import numpy as np
import pytest
import torch

from oracle import pages as OP
from pages_common import Both, i32

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype,d,page,hkv,layers", [
    (BF, 128, 64, 2, 2), (F32, 64, 32, 4, 1), (BF, 64, 256, 1, 3), (F32, 128, 128, 3, 2)])
def test_history(gpu_lib, dtype, d, page, hkv, layers):
    """Rounds, forks and compactions in a pool that runs short now and then."""
    rng = np.random.default_rng(page)
    b = 7
    c = Both(gpu_lib, layers, hkv, d, page, 26, b, 5, dtype)
    for step in range(40):
        op = rng.integers(6)
        if op < 4:
            c.append(rng.integers(0, (1, 18, 2 * page, 70)[op] + 1, b))
            c.check(False)
            if op:
                c.keep([rng.integers(0, o + 1) for o in c.o.open])
        elif op == 4:
            src = np.arange(b)
            src[rng.integers(b, size=3)] = rng.integers(-1, b, 3)
            c.fork(src)
        else:
            c.compact()
        c.check(step % 4 == 3)
    c.check()
    want = {OP.ERANGE: gpu_lib.LDR_ERANGE, OP.EPAGES: gpu_lib.LDR_EPAGES}
    flags = {want[f] for f in c.o.flags}
    got = c.g.status(clear=True)
    assert got in flags if flags else got == gpu_lib.LDR_OK
    assert c.g.status() == gpu_lib.LDR_OK


def test_shortage_is_refused_in_order(gpu_lib):
    c = Both(gpu_lib, 1, 1, 64, 32, 4, 4, 3, BF)
    c.append([32, 70, 32, 0])            # 1 + 3 pages; none is left for the third
    c.check()
    assert c.o.rows == [32, 70, 0, 0] and c.g.status(clear=True) == gpu_lib.LDR_EPAGES
    c.append([1, 0, 0, 0], 70)           # nothing free: unchanged, and nothing is written
    c.check()
    assert c.g.status(clear=True) == gpu_lib.LDR_EPAGES
    c.append([0, 26, 0, 0])              # room in its own page
    c.check()
    assert c.g.status() == gpu_lib.LDR_OK
    c.append([0, 1, 0, 0])               # its table is full
    assert c.g.status(clear=True) == gpu_lib.LDR_EPAGES


def test_counts_out_of_range(gpu_lib):
    c = Both(gpu_lib, 1, 1, 64, 32, 16, 4, 4, BF)
    c.append([5, -1, 9, 3], 8)           # -1 and 9 are outside [0, 8]
    c.check()
    assert c.o.rows == [5, 0, 0, 3] and c.g.status(clear=True) == gpu_lib.LDR_ERANGE
    for kept in ([6, 0, 0, 3], [-1, 0, 0, 3], [5, 1, 0, 3]):
        c.keep(kept)
        c.check()
        assert c.g.status(clear=True) == gpu_lib.LDR_ERANGE
    for src in ([0, 4, 2, 3], [0, -2, 2, 3], [1, 0, 2, 3], [1, 1, 1, 2], [-1, 0, 2, 3]):
        c.fork(src)
        c.check()
        assert c.g.status(clear=True) == gpu_lib.LDR_ERANGE
    assert c.o.rows.count(5) <= 1


def test_shared_page_is_copied_by_each_that_writes(gpu_lib):
    """One prompt, several samples: the partial page is copied, the whole ones stay shared."""
    c = Both(gpu_lib, 2, 2, 128, 64, 24, 5, 8, BF)
    c.append([150, 0, 0, 0, 0])
    c.fork([0, 0, 0, 0, 4])
    c.check()
    c.append([1, 17, 0, 2, 3])
    c.check()
    t = c.o.tables()
    assert np.all(t[:4, :2] == t[0, :2]) and len({t[b, 2] for b in (0, 1, 2, 3)}) == 4
    c.append([3, 3, 3, 3, 3])            # sequence 2 holds the old page alone by now
    c.check()
    c.fork([0, -1, 0, -1, -1])
    c.check()
    c.compact()
    c.check()
    assert all(r > 0 for r in c.o.refs[:3]) and not any(c.o.refs[3:])


def test_write_after_a_fork_changes_nothing(gpu_lib):
    """A fork closes the open rows: they may be shared now."""
    c = Both(gpu_lib, 1, 1, 64, 32, 8, 2, 4, F32)
    c.append([10, 0])
    c.fork([0, 0])
    K = c.rand(2, 10, 1, 1, 64)
    c.g.write(K, K)
    c.check()
    c.keep([0, 0])
    c.check()


def test_layers_apart_and_a_narrow_write(gpu_lib):
    """Layer by layer gives what all at once gives; rows beyond the write's
    max_new stay as they were."""
    a, b = (Both(gpu_lib, 3, 2, 64, 32, 12, 3, 4, BF, seed=1) for _ in range(2))
    n = [40, 0, 33]
    K, V = a.rand(3, 40, 3, 2, 64), a.rand(3, 40, 3, 2, 64)
    a.append(n, K=K, V=V)
    b.g.reserve(i32(n), 40)
    for layer in (2, 0, 1):
        b.g.write(K[:, :, layer:layer + 1].contiguous(), V[:, :, layer:layer + 1].contiguous(),
                  layer)
    torch.cuda.synchronize()
    assert torch.equal(a.g.pool.view(torch.int16), b.g.pool.view(torch.int16))
    before = b.g.pool.clone()
    b.g.write(K[:, :0 + 7].contiguous() * 2, V[:, :7].contiguous(), 0)
    torch.cuda.synchronize()
    k, old = b.g.k(0)[b.g.table[0, 0].long()], before[0, 0, b.g.table[0, 0].long()].view(2, 32, 64)
    assert torch.equal(k[:, :7], K[0, :7, 0].transpose(0, 1) * 2) and torch.equal(k[:, 7:], old[:, 7:])


def test_many_sequences_and_a_long_prefill(gpu_lib):
    """1024 sequences; and one that takes most of the pool at once."""
    rng = np.random.default_rng(3)
    c = Both(gpu_lib, 1, 1, 64, 32, 3000, 1024, 4, BF)
    c.append(rng.integers(0, 70, 1024))
    src = np.arange(1024)
    src[::3] = 1
    c.fork(src)
    c.append(rng.integers(0, 40, 1024))
    c.check(False)
    c = Both(gpu_lib, 1, 1, 64, 32, 3000, 2, 2500, BF)
    c.append([2000 * 32 + 5, 7])
    c.check()
    c.fork([0, 0])
    c.append([1, 900 * 32], 900 * 32)    # the second finds no room: 1 + 901 pages of 999
    c.check(False)


def test_pool_beyond_32_bit_offsets(gpu_lib):
    """A pool of 5.4 GB: the last pages of the last layer hold their rows."""
    g = gpu_lib.Pages(2, 8, 128, 256, 5120, 1, 5120).init()
    assert g.pool.numel() * 2 > 1 << 32
    g.refs[:5118] = 1                    # all but the last two pages are taken
    K = torch.randn(1, 300, 2, 8, 128, device="cuda").bfloat16()
    g.append(i32([300]), K, -K)
    torch.cuda.synchronize()
    assert g.table[0, :2].tolist() == [5118, 5119]
    for layer in range(2):
        k = g.k(layer)[5118:].transpose(1, 2).reshape(-1, 8, 128)[:300]
        v = g.v(layer)[5118:].permute(0, 3, 1, 2).reshape(-1, 8, 128)[:300]
        assert torch.equal(k, K[0, :, layer]) and torch.equal(v, -K[0, :, layer])


def test_captured_round(gpu_lib):
    """A round in a graph, replayed with other counts and rows, with eager calls
    and waits in between; undone by putting the state back."""
    c = Both(gpu_lib, 2, 1, 64, 32, 20, 3, 5, BF)
    c.append([40, 3, 0])
    n, kept = i32([0, 0, 0]), i32([0, 0, 0])
    K = torch.zeros(3, 17, 2, 1, 64, dtype=BF, device="cuda")
    s = torch.cuda.Stream()
    c.g._stream = s
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        c.g.reserve(n, 17)
        c.g.write(K, K)
        c.g.keep(kept)
        c.g.compact()
    c.g._stream = None
    rng = np.random.default_rng(4)
    for _ in range(4):
        nn = rng.integers(0, 18, 3)
        kk = [rng.integers(0, x + 1) for x in nn]
        n.copy_(i32(nn))
        kept.copy_(i32(kk))
        K.copy_(c.rand(*K.shape))
        graph.replay()
        c.o.reserve(nn, 17)
        c.o.write(K.double().cpu().numpy(), K.double().cpu().numpy())
        c.o.keep(kk)
        c.o.compact()
        c.check()
        saved = c.g.state.clone()
        c.g.fork(i32([0, 0, 0]))
        c.g.state.copy_(saved)
        c.check()
    assert c.g.status() == gpu_lib.LDR_OK


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_copied_page_is_whole(gpu_lib, dtype):
    """A part-filled page that two sequences hold: who gets one of its own gets what
    lies behind the rows too."""
    c = Both(gpu_lib, 2, 3, 64, 64, 9, 3, 3, dtype)
    g = c.g
    g.pool.view(torch.uint8).random_(0, 120)          # finite in both types
    c.append([70, 0, 5])
    c.fork([0, 0, 2])
    old, before = int(g.table[0, 1]), g.pool.clone()
    g.reserve(i32([1, 1, 1]), 1)
    a, b = int(g.table[0, 1]), int(g.table[1, 1])
    assert a != b and a != old and b != old
    for to in (a, b):
        assert torch.equal(g.pool[:, :, to], before[:, :, old])


def test_wants_of_more_than_an_int(gpu_lib):
    """66 sequences that each want all of a table of 2^25 - 1 pages, 2^31 and more
    together, of a pool of 4: none of them gets any, whatever is behind it."""
    b, most = 66, (1 << 25) - 1
    p = gpu_lib.Pages(1, 1, 64, 32, 4, b, most, BF).init()
    n = i32([most * 32] * (b - 1) + [1])
    p.reserve(n, most * 32)
    assert p.status(clear=True) == gpu_lib.LDR_EPAGES
    assert not p.rows.any() and not p.open.any() and not p.refs.any()
    n[:-1] = 0
    p.reserve(n, 1)
    assert p.status() == gpu_lib.LDR_OK
    assert p.rows.tolist() == [0] * (b - 1) + [1] and p.refs.tolist() == [1, 0, 0, 0]
    assert int(p.table[b - 1, 0]) == 0
