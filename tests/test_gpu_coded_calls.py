"""Calls on coded caches and of log probabilities that a server makes at the edges of their
sizes: as many sequences as a cache can have, many heads a group, far fewer rows than room for
them, nothing at all, and two at once on streams of their own."""
import numpy as np
import pytest
import torch

from mx_common import BothCoded
from pages_common import check_attend, i32
from test_gpu_logprobs import _check, _z
from test_gpu_mx_attend import _run

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("bits", [4, 8])
def test_1024_sequences(gpu_lib, bits):
    """Lengths of none to 900, a front that every other one shares."""
    c = BothCoded(gpu_lib, bits, 1, 1, 64, 32, 1024 * 8, 1024, 40, seed=1)
    c.append([512] + [0] * 1023)
    c.fork([0 if i % 2 == 0 else i for i in range(1024)])
    c.append([(37 * i) % 61 if i % 100 else 600 for i in range(1024)])
    c.append([i % 3 for i in range(1024)], 2)
    _run(gpu_lib, c, 2, 2, before=6.0)


@pytest.mark.parametrize("bits,d", [(4, 128), (8, 64)])
@pytest.mark.parametrize("rep", [48, 80, 96, 200, 300])
def test_many_heads_of_a_group(gpu_lib, bits, d, rep):
    """One query's heads are more rows than a tile."""
    c = BothCoded(gpu_lib, bits, 1, 1, d, 64, 60, 2, 30, seed=rep)
    c.append([1200, 100])
    c.append([2, 1])
    _run(gpu_lib, c, rep, 2)


def test_far_more_room_than_rows(gpu_lib):
    """A batch planned for 700 rows a sequence of which few are open, or none."""
    c = BothCoded(gpu_lib, 4, 1, 2, 128, 64, 80, 3, 30, seed=2)
    c.append([900, 0, 5])
    c.append([1, 0, 30], 700)
    _run(gpu_lib, c, 8, 700, before=2.0)


def test_nothing_to_do(gpu_lib):
    """No open rows, no rows to read, no rows of logits: outputs stay, no flag is set."""
    c = BothCoded(gpu_lib, 8, 1, 2, 64, 32, 20, 2, 9)
    _run(gpu_lib, c, 4, 3, before=5.0)
    c.append([70, 9])
    c.append([0, 0], 3)
    _run(gpu_lib, c, 4, 3, before=5.0)
    out = tuple(torch.full((2, 4, 1, 2, 64), 5.0, dtype=BF, device="cuda") for _ in range(2))
    c.g.read(i32([70, 0]), i32([0, 0]), out=out)
    assert c.g.status() == gpu_lib.LDR_OK and all(bool((t == 5).all()) for t in out)
    _check(gpu_lib, _z((2, 3, 900), 1), [[1, 2, 3]] * 2, 4, n=[0, 0], before=9.0)


def test_two_at_once(gpu_lib):
    """Caches, workspaces and outputs of their own on two streams, in turn without waiting."""
    work = []
    for k in range(2):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            c = BothCoded(gpu_lib, (4, 8)[k], 1, 2, 128, 64, 80, 2, 40, seed=k, stream=s)
            c.append([1500, 700])
            c.append([3, 2], 3)
            q = c.rand(2, 3, 8, 128)
            z = _z((2, 3, 50000), k)
        s.synchronize()
        work.append((s, c, q, z))
    y, got = i32([[1, 2, 3], [4, 5, 6]]), []
    for _ in range(3):
        for s, c, q, z in work:
            with torch.cuda.stream(s):
                lse = torch.zeros(2, 3, 8, device="cuda")
                o = gpu_lib.attend(c.g.plan(8, 3), 0, q, lse=lse)
                rows = c.g.read(i32([10, 600]), i32([40, 90]), 90)
                got.append((c, q, z, o, lse, rows,
                            gpu_lib.logprobs(z, y, top_n=6, n_rows=c.g.open, stream=s)))
    torch.cuda.synchronize()
    for c, q, z, o, lse, (K, V), lp in got:
        check_attend(c, 3, q, o, lse, 0, 128 ** -0.5)
        for b, (lo, n) in enumerate(((10, 40), (600, 90))):
            for x, r in zip((K, V), c.o.sequence(0, b)):
                assert np.array_equal(x[b, :n, 0].double().cpu().numpy(), r[lo:lo + n])
        ref = gpu_lib.logprobs(z, y, top_n=6, n_rows=c.g.open)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(lp, ref))
