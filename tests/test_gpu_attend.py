"""Attention over the paged cache against its fp64 definition, within the bound
of its arithmetic (pages_common.check_attend): head layouts, lengths, pages and
steps that end anywhere, shared fronts, masked values, strides, graphs."""
import numpy as np
import pytest
import torch

from pages_common import Both, check_attend, i32

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _run(ldr, c, hq, new, layer=0, groups=None, scale=None, q=None, before=0.0):
    d = c.g.d
    q = c.rand(c.batch, new, hq, d) if q is None else q
    scale = d ** -0.5 if scale is None else scale
    out = torch.full((c.batch, new, hq, d), before, dtype=c.dtype, device="cuda")
    lse = torch.full((c.batch, new, hq), before, device="cuda")
    plan = c.g.plan(hq, new, groups=groups)
    ldr.attend(plan, layer, q, out=out, lse=lse, scale=scale)
    torch.cuda.synchronize()
    assert c.g.status() == ldr.LDR_OK
    check_attend(c, new, q, out, lse, layer, scale, before)
    return q, out, lse


LAYOUTS = [(BF, 128, 8, 2, 64), (BF, 64, 4, 4, 32), (F32, 64, 4, 4, 32), (F32, 128, 6, 2, 64),
           (BF, 128, 8, 1, 128), (BF, 64, 5, 1, 256), (BF, 128, 3, 3, 64)]


@pytest.mark.parametrize("dtype,d,hq,hkv,page", LAYOUTS)
@pytest.mark.parametrize("new", [1, 2, 17, 40])
def test_lengths(gpu_lib, dtype, d, hq, hkv, page, new):
    """No row, one row, the edges of steps and pages, a few chunks; some
    sequences have fewer open rows than others, or none."""
    rows = [0, 1, 31, 32, 33, 63, 65, 300]
    c = Both(gpu_lib, 2, hkv, d, page, 40, 8, 12, dtype, seed=new)
    c.append(rows)
    c.append([min(new, n) for n in (new, 1, new, 0, 3, new, new - 1, new)], new)
    for layer in (0, 1):
        _run(gpu_lib, c, hq, new, layer, before=7.0)


@pytest.mark.parametrize("dtype,d,hq,hkv,page", LAYOUTS[:5])
@pytest.mark.parametrize("new", [1, 9])
def test_shared_fronts(gpu_lib, dtype, d, hq, hkv, page, new):
    """Two prompts with samples of their own lengths, a stranger between them,
    in slots in no order: the same with any grouping."""
    c = Both(gpu_lib, 1, hkv, d, page, 120, 9, 30, dtype, seed=5)
    prompt = 4 * max(page, 64) + 11
    c.append([prompt, 0, 0, 500, 0, 0, 0, 0, 70])
    c.fork([0, 3, 0, 3, 0, 0, 3, 7, 8])
    c.append([3, 40, 0, 2, 70, 33, 1, 0, 5])
    c.append([new, new, new, 1, new, 0, new, 2 if new > 1 else 1, new], new)
    q, o1, l1 = _run(gpu_lib, c, hq, new)
    for groups in (list(range(9)), [-1] * 9, [0] * 9, [4, 7, 4, 7, 4, 4, 7, 4, 1 << 30]):
        _, o2, l2 = _run(gpu_lib, c, hq, new, groups=i32(groups), q=q)


def test_group_members_that_part_early(gpu_lib):
    """A fork of a fork and a sample that parted inside the front: the group
    shares what all of it has in common."""
    c = Both(gpu_lib, 1, 2, 128, 32, 160, 5, 40, BF, seed=6)
    c.append([300, 0, 0, 0, 0])
    c.fork([0, 0, 0, 0, 4])
    c.append([200, 1, 1, 0, 0], 200)
    c.fork([0, 1, 2, 0, 4])
    c.append([4, 4, 4, 4, 4])
    _run(gpu_lib, c, 8, 4)
    _run(gpu_lib, c, 8, 4, groups=i32([3, 3, 3, 3, 3]))


def test_long_cache_and_many_rows(gpu_lib):
    """Many chunks a row, and more query rows than a tile."""
    c = Both(gpu_lib, 1, 1, 64, 64, 300, 2, 200, BF, seed=7)
    c.append([5000, 777])
    c.append([130, 1])
    _run(gpu_lib, c, 4, 130)


@pytest.mark.parametrize("dtype,extra", [(BF, 0), (F32, 0), (BF, 80)])
def test_masked_values_do_not_count(gpu_lib, dtype, extra):
    """NaN and infinities in the rows behind a query: later open rows, and what
    free parts of a page hold (NaN, by the test's pool). The rows that see them
    take them."""
    for bad in (float("nan"), float("inf"), -float("inf")):
        for which in ("K", "V", "KV"):
            c = Both(gpu_lib, 1, 2, 64, 32, 40, 2, 10, dtype, seed=8)
            c.append([70, 20])
            new = 9 + extra              # with more rows, of another kernel
            K, V = c.rand(2, new, 1, 2, 64), c.rand(2, new, 1, 2, 64)
            if "K" in which:
                K[0, 5] = bad
            if "V" in which:
                V[0, 5, 0, 1, 3:40] = bad
                V[1, 8] = bad
            c.append([new, new], new, K, V)
            q = c.rand(2, new, 4, 64).abs() + 0.1    # K = -inf: the key has no weight
            d = c.g.d
            out = torch.zeros(2, new, 4, d, dtype=dtype, device="cuda")
            gpu_lib.attend(c.g.plan(4, new), 0, q, out=out)
            torch.cuda.synchronize()
            if which == "V" or bad != bad:
                check_attend(c, new, q, out, None, 0, d ** -0.5)
            else:                                    # rows before it are as if it were not there
                assert torch.isfinite(out[0, :5]).all()


def test_rows_without_weight(gpu_lib):
    """Scores of -inf only: no result, 0 and -inf."""
    c = Both(gpu_lib, 1, 1, 64, 32, 8, 1, 4, F32, seed=9)
    K = torch.full((1, 3, 1, 1, 64), -float("inf"), device="cuda")
    c.append([3], 3, K, c.rand(1, 3, 1, 1, 64))
    q = torch.ones(1, 3, 2, 64, device="cuda")
    _, o, lse = _run(gpu_lib, c, 2, 3, q=q)
    assert torch.all(o == 0) and torch.all(lse == -float("inf"))


def test_large_scores(gpu_lib):
    """Scores of thousands: the maximum is taken out before the exponential."""
    for dtype in (BF, F32):
        c = Both(gpu_lib, 1, 1, 64, 32, 40, 1, 30, dtype, seed=10)
        c.append([600], K=c.rand(1, 600, 1, 1, 64) * 40)
        c.append([5])
        _run(gpu_lib, c, 2, 5, q=c.rand(1, 5, 2, 64) * 8)


def test_strided_queries_and_streams(gpu_lib):
    """Queries inside a fused projection's rows; another stream than the current."""
    s = torch.cuda.Stream()
    c = Both(gpu_lib, 1, 2, 128, 64, 20, 3, 4, BF, seed=11)
    c.append([100, 3, 64])
    c.append([5, 5, 5])
    qkv = c.rand(3, 5, (8 + 4) * 128)
    q = qkv[..., :8 * 128].unflatten(-1, (8, 128))
    _, ref, rl = _run(gpu_lib, c, 8, 5, q=q.contiguous())
    out = gpu_lib.attend(c.g.plan(8, 5), 0, q)
    torch.cuda.synchronize()
    assert torch.equal(out, ref)
    s.wait_stream(torch.cuda.current_stream())
    c.g._stream = s
    out = gpu_lib.attend(c.g.plan(8, 5), 0, q)
    s.synchronize()
    assert torch.equal(out, ref)
    with pytest.raises(gpu_lib.LdrError):       # heads apart
        gpu_lib.attend(c.g.plan(8, 5), 0, qkv.view(3, 5, 12, 128)[:, :, ::2][:, :, :8])
    with pytest.raises(gpu_lib.LdrError):
        gpu_lib.attend(c.g.plan(8, 5), 0, q.float())
    with pytest.raises(gpu_lib.LdrError):
        gpu_lib.attend(c.g.plan(8, 5), 1, q)    # no such layer
    for scale in (0.0, -1.0, 1e-40, float("nan"), float("inf")):
        with pytest.raises(gpu_lib.LdrError):
            gpu_lib.attend(c.g.plan(8, 5), 0, q, scale=scale)


def test_plan_of_another_state(gpu_lib):
    """A plan serves the state it was made from: afterwards nothing is written
    and the status says so."""
    c = Both(gpu_lib, 1, 1, 64, 32, 20, 2, 8, BF, seed=12)
    c.append([50, 40])
    q = c.rand(2, 40, 2, 64)
    plan = c.g.plan(2, 40)
    c.keep([1, 1])
    out = torch.full((2, 40, 2, 64), 3.0, dtype=BF, device="cuda")
    gpu_lib.attend(plan, 0, q, out=out)
    assert c.g.status(clear=True) == gpu_lib.LDR_EINVAL and torch.all(out == 3.0)
    other = c.g.plan(2, 4, workspace=plan.workspace)      # the workspace holds another plan
    gpu_lib.attend(plan, 0, q, out=out)
    assert c.g.status(clear=True) == gpu_lib.LDR_EINVAL and torch.all(out == 3.0)
    gpu_lib.attend(other, 0, q[:, :4].contiguous())
    assert c.g.status() == gpu_lib.LDR_OK
    with pytest.raises(gpu_lib.LdrError):
        c.g.plan(2, 40, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))


def test_rows_beyond_the_plans(gpu_lib):
    """More open rows than max_new: the first max_new of them have queries."""
    c = Both(gpu_lib, 1, 1, 64, 32, 20, 2, 8, F32, seed=13)
    c.append([50, 9])
    _run(gpu_lib, c, 2, 6)


def test_captured_layers(gpu_lib):
    """Plan and layers in a graph, replayed over a growing cache."""
    c = Both(gpu_lib, 2, 2, 64, 32, 60, 3, 20, BF, seed=14)
    c.append([200, 0, 31])
    c.fork([0, 0, 2])
    n = i32([4, 4, 4])
    K = torch.zeros(3, 4, 2, 2, 64, dtype=BF, device="cuda")
    q = torch.zeros(2, 3, 4, 4, 64, dtype=BF, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(2, 3, 4, 4, device="cuda")
    ws = torch.empty(c.g.attend_workspace_bytes(4, 4), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    c.g._stream = s
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        c.g.append(n, K, K)
        plan = c.g.plan(4, 4, workspace=ws)
        for layer in range(2):
            gpu_lib.attend(plan, layer, q[layer], out=out[layer], lse=lse[layer])
    c.g._stream = None
    for step in range(4):
        K.copy_(c.rand(*K.shape))
        q.copy_(c.rand(*q.shape))
        graph.replay()
        c.o.reserve([4, 4, 4], 4)
        c.o.write(K.double().cpu().numpy(), K.double().cpu().numpy())
        torch.cuda.synchronize()
        for layer in range(2):
            check_attend(c, 4, q[layer], out[layer], lse[layer], layer, 0.125)
        if step == 1:
            c.append([30, 1, 0])     # eager work in between
    assert c.g.status() == gpu_lib.LDR_OK


def test_same_bits_every_time(gpu_lib):
    c = Both(gpu_lib, 1, 2, 128, 64, 200, 4, 60, BF, seed=15)
    c.append([3000, 0, 0, 50])
    c.fork([0, 0, 0, 3])
    c.append([17, 17, 17, 17])
    q, o, lse = _run(gpu_lib, c, 8, 17)
    for _ in range(3):
        out = gpu_lib.attend(c.g.plan(8, 17), 0, q)
        torch.cuda.synchronize()
        assert torch.equal(out, o)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("hq,new", [(1, 1), (2, 1), (3, 1), (1, 7), (8, 1), (4, 5), (8, 4)])
def test_few_rows_of_many_parts(gpu_lib, dtype, d, hq, new):
    """1 to 32 rows over enough keys for some twenty parts each, which are joined
    side by side; one sequence has none, one a single part."""
    c = Both(gpu_lib, 1, 1, d, 64, 200, 3, 90, dtype, seed=hq)
    c.append([5000, 100, 600])
    c.append([new, new, new])
    _run(gpu_lib, c, hq, new)


def test_a_thousand_sequences(gpu_lib):
    """As many sequences as a cache takes, in groups of one prompt, strangers and empty
    ones between them."""
    b = 1024
    c = Both(gpu_lib, 1, 1, 64, 32, 4096, b, 24, F32, seed=9)
    src = np.array([i % 8 if i % 7 < 5 else i for i in range(b)])
    c.append([[300, 520, 33, 700, 31, 256, 290, 0][i] if i < 8 else 0 for i in range(b)], 700)
    c.fork(src)
    c.append([i % 3 for i in range(b)], 2)
    _run(gpu_lib, c, 2, 2)
