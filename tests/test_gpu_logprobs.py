"""Log probabilities, entropies, ranks and alternatives against their fp64 definition.

With e = 2^-24 (half a step of fp32), x_v = (z_v - m) / T and V entries: an exponent
x log2(e) has the rounding of the difference, of the factor and of the product, 3 e |x|
(absolute, natural units), the power of two 2 e (a step); a sum of V positive terms adds
(32 + log2 V) e relative (32 terms of a thread, then trees, pieces one after the other:
V / 2048 more) and its logarithm 4 e. The terms far below the maximum have little weight, so
|x| is averaged over p: the error of log S is at most
  dS = e (3 E|x| + 40 + V / 2048 + log2 V),  E|x| = sum p |x|,
plus 4 e |log S|; log p adds 3 e |x| of its own and 2 e |log p|. The entropy's second part
has the same relative errors in every product, 3 e |x| + 4 e + those of the sums:
  dH = dS + e (3 E x^2 + (48 + V / 2048 + log2 V) E|x|) + 4 e H."""
import numpy as np
import pytest
import torch

from oracle import pages as OP
from pages_common import i32

pytestmark = pytest.mark.gpu


def _check(ldr, z, y, top, T=1.0, n=None, before=None, **kw):
    batch, rows, V = z.shape
    out = None
    if before is not None:
        out = (torch.full((batch, rows), before, device="cuda"),
               torch.full((batch, rows), before, device="cuda"),
               torch.full((batch, rows), int(before), dtype=torch.int32, device="cuda"),
               torch.full((batch, rows, top), int(before), dtype=torch.int32, device="cuda"),
               torch.full((batch, rows, top), before, device="cuda"))
    got = ldr.logprobs(z, i32(y), top_n=top, temperature=T, n_rows=None if n is None else i32(n),
                       out=out, **kw)
    torch.cuda.synchronize()
    g = [t.double().cpu().numpy() for t in got]
    zs = z.double().cpu().numpy()
    e = 2.0 ** -24
    T = float(np.float32(T))
    for b in range(batch):
        for i in range(rows):
            at = (b, i)
            if n is not None and i >= n[b]:
                for t in g:
                    assert np.all(t[at] == (before or 0)), at
                continue
            lp, ent, rank, order, tl = OP.logprobs(zs[at], int(y[b][i]), T, top)
            assert g[2][at] == rank, (at, g[2][at], rank)
            assert list(g[3][at]) == list(order), at
            if np.isnan(ent):
                assert np.isnan(g[0][at]) and np.isnan(g[1][at]) and np.isnan(g[4][at]).all(), at
                continue
            zf = zs[at]
            x = (zf - zf.max()) / T if np.isfinite(zf.max()) else np.zeros(V)
            p = np.exp(x) / np.exp(x).sum()
            fin = p > 0
            ex, ex2 = (p[fin] * -x[fin]).sum(), (p[fin] * x[fin] ** 2).sum()
            ds = e * (3 * ex + 40 + V / 2048 + np.log2(V)) + 4 * e * np.log(np.exp(x).sum())
            for a, r in [(g[0][at], lp)] + list(zip(g[4][at], tl)):
                if np.isneginf(r):
                    assert np.isneginf(a), at
                else:
                    assert abs(a - r) <= ds + e * 5 * (abs(r) + np.log(V)), (at, a, r)
            dh = ds + e * (3 * ex2 + (48 + V / 2048 + np.log2(V)) * ex) + 4 * e * ent
            assert abs(g[1][at] - ent) <= dh, (at, g[1][at], ent, dh)
    return got


def _z(shape, seed, spread=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda") * spread


@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1023, 2048, 2049, 5003, 20000, 151936])
@pytest.mark.parametrize("top", [0, 1, 5, 64])
def test_vocabularies(gpu_lib, V, top):
    top = min(top, V)
    z = _z((2, 3, V), V + top)
    y = np.random.default_rng(V).integers(0, V, (2, 3))
    y[0, 0] = int(z[0, 0].argmax())
    _check(gpu_lib, z, y, top, before=5.0)


@pytest.mark.parametrize("T", [0.1, 0.7, 1.0, 4.0, 1e-20, 1e20])
def test_temperatures(gpu_lib, T):
    _check(gpu_lib, _z((1, 4, 3001), 3), [[0, 5, 3000, 77]], 7, T)


def test_many_rows_take_larger_pieces(gpu_lib):
    """Enough rows for pieces of 8192 entries, the last of them short."""
    V = 16500
    z = _z((190, 1, V), 4)
    y = np.random.default_rng(1).integers(0, V, (190, 1))
    _check(gpu_lib, z, y, 20)


@pytest.mark.parametrize("top", [1, 20, 64])
def test_many_rows_are_picked_by_fewer_waves(gpu_lib, top):
    """More than 512 rows; vocabularies whose maxima are more than a workgroup holds."""
    z = _z((3, 171, 700), top)
    z[0, :50] = torch.round(z[0, :50])
    z[1, 7, ::2] = -float("inf")
    z[1, 8] = float("nan")
    _check(gpu_lib, z, np.random.default_rng(top).integers(0, 700, (3, 171)), top)


def test_large_vocabularies(gpu_lib):
    V = 4096 * 64 + 700
    z = _z((1, 2, V), 31)
    z[0, 1] -= 40.0 * (torch.arange(V, device="cuda") // 64 % 16 == 5)
    z[0, 1, -3:] += 60.0
    _check(gpu_lib, z, [[V - 1, 4]], 64)


def test_ties_go_to_the_lowest_index(gpu_lib):
    z = torch.zeros(1, 4, 5000, device="cuda")
    z[0, 1, ::7] = 1.0
    z[0, 2, 4000:] = -0.0
    z[0, 3] = torch.arange(5000, device="cuda") // 100 % 3
    _check(gpu_lib, z, [[4999, 700, 4500, 250]], 64)


def test_the_largest_entries_close_together_or_apart(gpu_lib):
    """All of them in one group of neighbours, one a group, in order and in reverse."""
    V = 9000
    z = _z((1, 5, V), 6, 0.1)
    z[0, 0, 640:704] += 50
    z[0, 1, ::128] += 50
    z[0, 2] = torch.arange(V, device="cuda") / 10
    z[0, 3] = -torch.arange(V, device="cuda") / 10
    z[0, 4, -3:] += 9
    _check(gpu_lib, z, [[650, 128, 0, 0, V - 1]], 64)


def test_one_wave_with_nothing_but_small_entries(gpu_lib):
    """Every fourth (eighth, sixteenth) group, or entry, far below the others: no threshold
    leaves few candidates."""
    V = 151936
    at = torch.arange(V, device="cuda")
    for w in (4, 8, 16):
        z = _z((1, 3, V), 61, 1.0)
        z[0, 0] -= 100.0 * (at // 64 % w == 3)
        z[0, 1] -= 100.0 * (at % w == w - 1)
        z[0, 2] = torch.where((at // 64 % w == 0) | (at % w == 0), -50.0, 1.0)
        _check(gpu_lib, z, [[5, 6, 7]], 64)
        _check(gpu_lib, z, [[5, 6, 7]], 17)


def test_one_wave_of_four_with_nothing_but_small_entries(gpu_lib):
    """The same where many rows are picked by four waves."""
    V = 20000
    at = torch.arange(V, device="cuda")
    z = _z((2, 300, V), 62, 1.0)
    z[0] -= 100.0 * (at // 64 % 4 == 3)
    z[1] -= 100.0 * (at % 4 == 1)
    _check(gpu_lib, z, np.zeros((2, 300), int), 30)


def test_masked_entries(gpu_lib):
    """-inf: entries without probability; rows with one entry left, and with none."""
    z = _z((1, 6, 4100), 7)
    inf = float("inf")
    z[0, 0, ::2] = -inf
    z[0, 1, 1:] = -inf
    z[0, 2, :-1] = -inf
    z[0, 3] = -inf
    z[0, 4, :3000] = -inf
    z[0, 5] = torch.finfo(torch.float32).min
    got = _check(gpu_lib, z, [[0, 0, 4099, 17, 5, 9]], 8)
    assert got[0][0, 1] == 0 and got[1][0, 1] == 0


def test_values_that_are_not_numbers(gpu_lib):
    """NaN or +inf: the row's probabilities are NaN, its order stands."""
    z = _z((1, 6, 3000), 8)
    nan, inf = float("nan"), float("inf")
    z[0, 0, 5] = nan
    z[0, 1, 1000:] = nan
    z[0, 2] = nan
    z[0, 3, 64:128] = nan
    z[0, 3, :64] = -inf
    z[0, 3, 128:] = -inf
    z[0, 4, 2999] = inf
    z[0, 5, :2990] = nan
    z[0, 5, 2990:] = -inf
    _check(gpu_lib, z, [[5, 3, 7, 70, 2, 2995]], 64)


def test_tokens_outside_the_vocabulary(gpu_lib):
    z = _z((1, 4, 777), 9)
    lp, _, rank, _, _ = _check(gpu_lib, z, [[-1, 777, 2 ** 31 - 1, -2 ** 31]], 2)
    assert bool((lp == -float("inf")).all()) and bool((rank == 777).all())


def test_nearly_certain_tokens_keep_their_digits(gpu_lib):
    """log p near 0: 2^-17 or less of it off, which 1 - p alone would lose."""
    z = torch.zeros(1, 3, 4096, device="cuda")
    z[0, 0, 9], z[0, 1, 9], z[0, 2, 9] = 20.0, 25.0, 30.0
    lp, ent, _, _, _ = gpu_lib.logprobs(z, i32([[9, 9, 9]]))
    for i in range(3):
        r = OP.logprobs(z[0, i].double().cpu().numpy(), 9, 1.0, 0)
        assert abs(lp[0, i].item() - r[0]) <= 2.0 ** -17 * abs(r[0])
        assert abs(ent[0, i].item() - r[1]) <= 2.0 ** -16 * abs(r[1])


def test_rows_behind_the_last_and_counts_out_of_range(gpu_lib):
    z = _z((4, 3, 2500), 10)
    y = np.arange(12).reshape(4, 3)
    _check(gpu_lib, z, y, 3, n=[0, 3, 1, 2], before=8.0)
    _check(gpu_lib, z, y, 3, n=[-5, 2 ** 31 - 1, 3, 4], before=8.0)


def test_padded_rows_and_odd_places(gpu_lib):
    """Rows a stride apart, that begin at any multiple of four bytes."""
    wide = _z((2, 3, 5020), 11)
    wide[..., 5003:] = 1e9
    for lo in (0, 1, 2, 3):
        _check(gpu_lib, wide[..., lo:5003], [[1, 2, 3], [4, 5, 6]], 9)
    _check(gpu_lib, wide[:, 1:2, :5001], [[1], [4]], 9)


def test_workspace_contents_and_reuse(gpu_lib):
    """Whatever a workspace holds; two calls on one workspace, one after the other."""
    ws = torch.full((gpu_lib.logprobs_workspace_bytes(2, 2, 6000, 10),), 255, dtype=torch.uint8,
                    device="cuda")
    for seed in (1, 2):
        _check(gpu_lib, _z((2, 2, 6000), seed), [[1, 2], [3, 4]], 10, workspace=ws)


def test_graph_replays(gpu_lib):
    z, y = _z((2, 2, 30000), 12), i32([[5, 6], [7, 8]])
    n = i32([2, 1])
    out = gpu_lib.logprobs(z, y, top_n=5, n_rows=n)
    ws = torch.empty(gpu_lib.logprobs_workspace_bytes(2, 2, 30000, 5), dtype=torch.uint8,
                     device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gpu_lib.logprobs(z, y, top_n=5, n_rows=n, out=out, workspace=ws)
    for k in range(4):
        z.copy_(_z((2, 2, 30000), 20 + k))
        graph.replay()
        torch.cuda.synchronize()
        ref = gpu_lib.logprobs(z, y, top_n=5, n_rows=n)
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
        _check(gpu_lib, z, y.tolist(), 5, n=[2, 1])
