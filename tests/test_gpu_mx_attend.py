"""Attention over a coded cache against its fp64 definition over the values that the
codes stand for, within the bound of its arithmetic (pages_common.check_attend)."""
import pytest
import torch

from mx_common import BothCoded
from pages_common import check_attend, i32

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _run(ldr, c, hq, new, layer=0, groups=None, scale=None, q=None, before=0.0):
    d = c.g.d
    q = c.rand(c.batch, new, hq, d) if q is None else q
    scale = d ** -0.5 if scale is None else scale
    out = torch.full((c.batch, new, hq, d), before, dtype=BF, device="cuda")
    lse = torch.full((c.batch, new, hq), before, device="cuda")
    plan = c.g.plan(hq, new, groups=groups)
    ldr.attend(plan, layer, q, out=out, lse=lse, scale=scale)
    torch.cuda.synchronize()
    assert c.g.status() == ldr.LDR_OK
    check_attend(c, new, q, out, lse, layer, scale, before)
    return q, out, lse


LAYOUTS = [(4, 128, 8, 2, 64), (8, 128, 8, 2, 64), (4, 64, 4, 4, 32), (8, 64, 4, 4, 32),
           (4, 128, 8, 1, 128), (8, 64, 5, 1, 256), (4, 128, 3, 3, 32), (8, 128, 2, 1, 32)]


@pytest.mark.parametrize("bits,d,hq,hkv,page", LAYOUTS)
@pytest.mark.parametrize("new", [1, 2, 17, 40])
def test_lengths(gpu_lib, bits, d, hq, hkv, page, new):
    """No row, one row, the edges of steps and pages; some sequences have fewer open rows
    than others, or none. The last kernel alone."""
    rows = [0, 1, 31, 32, 33, 63, 65, 300]
    c = BothCoded(gpu_lib, bits, 2, hkv, d, page, 40, 8, 12, seed=new)
    c.append(rows)
    c.append([min(new, n) for n in (new, 1, new, 0, 3, new, new - 1, new)], new)
    for layer in (0, 1):
        _run(gpu_lib, c, hq, new, layer, before=7.0)


@pytest.mark.parametrize("bits,d,hq,hkv,page", LAYOUTS)
@pytest.mark.parametrize("new", [1, 7, 33, 70])
def test_items(gpu_lib, bits, d, hq, hkv, page, new):
    """Keys enough for items: of up to 32 rows, of up to 128, of more, and several tiles."""
    n = 1100 // page * page
    c = BothCoded(gpu_lib, bits, 1, hkv, d, page, 3 * (-(-1600 // page)) + 3, 3, 1700 // page + 1,
                  seed=new)
    c.append([n, 777, 1500])
    c.append([new, new, max(1, new - 5)], new)
    _run(gpu_lib, c, hq, new, before=3.0)


@pytest.mark.parametrize("bits,d,hq,hkv,page", [LAYOUTS[i] for i in (0, 1, 2, 3, 6, 7)])
@pytest.mark.parametrize("new", [1, 9])
def test_shared_fronts(gpu_lib, bits, d, hq, hkv, page, new):
    """Two prompts with samples of their own lengths, a stranger between them, in slots in
    no order: the same with any grouping."""
    c = BothCoded(gpu_lib, bits, 1, hkv, d, page, 120, 9, 30, seed=5)
    prompt = 4 * max(page, 64) + 11
    c.append([prompt, 0, 0, 500, 0, 0, 0, 0, 70])
    c.fork([0, 3, 0, 3, 0, 0, 3, 7, 8])
    c.append([3, 40, 0, 2, 70, 33, 1, 0, 5])
    c.append([new, new, new, 1, new, 0, new, 2 if new > 1 else 1, new], new)
    q, o1, l1 = _run(gpu_lib, c, hq, new)
    for groups in (list(range(9)), [-1] * 9, [0] * 9, [4, 7, 4, 7, 4, 4, 7, 4, 1 << 30]):
        _run(gpu_lib, c, hq, new, groups=i32(groups), q=q)


@pytest.mark.parametrize("bits,d", [(4, 128), (8, 128), (4, 64), (8, 64)])
@pytest.mark.parametrize("hq", [8, 64])
def test_many_sequences(gpu_lib, bits, d, hq):
    """More items than run at once, and more rows than one workgroup a compute unit; items
    of one tile, of two, and of 72 rows, which are two items."""
    c = BothCoded(gpu_lib, bits, 1, 8, d, 64, 560, 40, 14, seed=hq)
    c.append([0, 1, 63, 600, 700] + [513 + 3 * i for i in range(35)])
    c.append([9 - i % 3 for i in range(40)], 9)
    _run(gpu_lib, c, hq, 9, before=2.0)


@pytest.mark.parametrize("bits", [4, 8])
def test_many_rows(gpu_lib, bits):
    """More query rows than a tile, the last tile of one row, many chunks."""
    c = BothCoded(gpu_lib, bits, 1, 1, 64, 64, 100, 2, 60, seed=7)
    c.append([2500, 777])
    c.append([129, 1])
    _run(gpu_lib, c, 4, 129)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("extra", [0, 80])
def test_masked_values_do_not_count(gpu_lib, bits, extra):
    """A block of NaN in the rows behind a query, and what free parts of a page hold (NaN,
    by the test's pool). The rows that see it take it."""
    for which in ("K", "V", "KV"):
        c = BothCoded(gpu_lib, bits, 1, 2, 64, 32, 40, 2, 10, seed=8)
        c.append([70, 20])
        new = 9 + extra
        K, V = c.rand(2, new, 1, 2, 64), c.rand(2, new, 1, 2, 64)
        if "K" in which:
            K[0, 5, 0, 1, 3] = float("inf")
        if "V" in which:
            V[0, 5, 0, 1, 3:40] = float("nan")
            V[1, 8] = -float("inf")
        c.append([new, new], new, K, V)
        _run(gpu_lib, c, 4, new)


@pytest.mark.parametrize("new", [1, 40])
def test_nan_within_an_item(gpu_lib, new):
    """A V block of NaN among the keys that all rows see: those dimensions of every row."""
    c = BothCoded(gpu_lib, 4, 1, 1, 128, 64, 40, 2, 20, seed=9)
    K, V = c.rand(2, 700, 1, 1, 128), c.rand(2, 700, 1, 1, 128)
    V[0, 130, 0, 0, 33] = float("nan")
    K[1, 200, 0, 0, 5] = float("nan")
    c.append([700, 700], 700, K, V)
    c.append([new, new], new)
    q, o, _ = _run(gpu_lib, c, 4, new)
    assert bool(o[0, :, :, 32:64].isnan().all()) and not bool(o[0, :, :, :32].isnan().any())
    assert bool(o[1].isnan().all())


@pytest.mark.parametrize("bits", [4, 8])
def test_scales_and_large_scores(gpu_lib, bits):
    """Scores that grow along the keys (the maximum moves in every step), that shrink, and
    that are all equal; scales far from 1 / sqrt(d)."""
    for make in ("grow", "shrink", "same"):
        c = BothCoded(gpu_lib, bits, 1, 1, 64, 32, 60, 1, 50, seed=10)
        K, V = c.rand(1, 1300, 1, 1, 64) * 0.05, c.rand(1, 1300, 1, 1, 64)
        t = torch.arange(1300, device="cuda") / 1300
        K[..., 0] += ({"grow": t, "shrink": 1 - t, "same": 0 * t}[make] * 4)[None, :, None, None].to(BF)
        if make == "same":
            K[:] = K[:, :1]
        c.append([1300], 1300, K.contiguous(), V)
        c.append([3], 3)
        q = c.rand(1, 3, 4, 64).abs() + 0.5
        _run(gpu_lib, c, 4, 3, q=q, scale=1.0)
        _run(gpu_lib, c, 4, 3, q=q, scale=2.0 ** -10)


def test_strided_queries_and_results_in_place(gpu_lib):
    c = BothCoded(gpu_lib, 4, 1, 2, 128, 64, 40, 3, 20, seed=11)
    c.append([600, 40, 900])
    c.append([5, 5, 5])
    wide = c.rand(3, 5, 12, 128)
    q = wide[:, :, 2:10]
    _run(gpu_lib, c, 8, 5, q=q)
    q, o, _ = _run(gpu_lib, c, 8, 5, q=q.contiguous())
    plan = c.g.plan(8, 5)
    gpu_lib.attend(plan, 0, q, out=q)
    assert torch.equal(q, o)


def test_graph_replays_and_another_stream(gpu_lib):
    """A captured round (rows, plan, attention) replayed on changing inputs, eager work and
    synchronizations in between, on a stream of its own."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = BothCoded(gpu_lib, 4, 1, 2, 64, 32, 80, 3, 30, seed=12, stream=s)
        c.append([800, 33, 0])
        n = i32([2, 3, 1])
        K, V = c.rand(3, 3, 1, 2, 64), c.rand(3, 3, 1, 2, 64)
        q, out = c.rand(3, 3, 4, 64), torch.zeros(3, 3, 4, 64, dtype=BF, device="cuda")
        lse = torch.zeros(3, 3, 4, device="cuda")
        ws = torch.empty(c.g.attend_workspace_bytes(4, 3), dtype=torch.uint8, device="cuda")
        back = tuple(torch.zeros(3, 3, 1, 2, 64, dtype=BF, device="cuda") for _ in range(2))

        def round_():
            first = c.g.rows.clone()
            c.g.append(n, K, V)
            gpu_lib.attend(c.g.plan(4, 3, workspace=ws), 0, q, out=out, lse=lse)
            c.g.read(first, n, out=back)

        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        before = c.g.state.clone()
        round_()                       # once before the capture
        c.g.state.copy_(before)
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            round_()
        for k in range(4):
            K.copy_(c.rand(*K.shape))
            V.copy_(c.rand(*V.shape))
            q.copy_(c.rand(*q.shape))
            out.zero_()
            lse.zero_()
            graph.replay()
            s.synchronize()
            c.o.reserve([2, 3, 1], 3)
            c.o.write(K.double().cpu().numpy(), V.double().cpu().numpy())
            c.check()
            check_attend(c, 3, q, out, lse, 0, 64 ** -0.5)
            assert torch.equal(back[0][1], c.g.read(c.g.rows - n, n, 3)[0][1])
        assert c.g.status() == gpu_lib.LDR_OK


def test_same_answer_twice_and_beside_other_sequences(gpu_lib):
    """Bits do not change from call to call."""
    c = BothCoded(gpu_lib, 8, 1, 2, 128, 64, 90, 4, 40, seed=13)
    c.append([2000, 300, 1, 900])
    c.append([4, 4, 4, 4])
    q, o, l = _run(gpu_lib, c, 8, 4)
    for _ in range(3):
        _, o2, l2 = _run(gpu_lib, c, 8, 4, q=q)
        assert torch.equal(o, o2) and torch.equal(l, l2)
