"""The kinds of items and of last kernels of the attention over a coded cache, at the numbers of
rows where one gives way to the next, against the fp64 definition (check_attend)."""
import pytest
import torch

from mx_common import BothCoded
from pages_common import check_attend, i32
from test_gpu_mx_attend import _run

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("bits,d,page", [(4, 128, 32), (8, 128, 32), (4, 128, 64), (8, 128, 64),
                                         (4, 64, 32), (8, 64, 64)])
@pytest.mark.parametrize("rows", [32, 33, 64, 65, 72, 96, 97, 112, 128, 129, 132, 160, 255, 256, 257])
def test_rows_of_an_item(gpu_lib, bits, d, page, rows):
    """One tile of 32, two, two tiles of 64 and of the rest, 128 in two groups over a half of
    the keys each, 256, and one row more than each: a query head a K/V head, so that rows are
    queries. The first sequence has the items, the second its last kernel alone."""
    c = BothCoded(gpu_lib, bits, 1, 1, d, page, 3 * (1800 // page), 2, 1800 // page + 2, seed=rows)
    c.append([1300, 40])
    c.append([rows, 3], rows)
    _run(gpu_lib, c, 1, rows, before=4.0)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rep,new", [(4, 16), (4, 17), (4, 24), (4, 25), (4, 32), (4, 33), (4, 40),
                                     (5, 13), (7, 14)])
def test_rows_of_several_heads_on_small_pages(gpu_lib, bits, d, rep, new):
    """The same numbers of rows as heads of a group, a tile's edge within a query's heads,
    pages of half a stage."""
    c = BothCoded(gpu_lib, bits, 1, 2, d, 32, 130, 3, 50, seed=new)
    c.append([900, 1100, 5])
    c.append([new, new - 1, new], new)
    _run(gpu_lib, c, 2 * rep, new, before=1.0)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("page", [32, 128])
@pytest.mark.parametrize("new", [2, 3, 4, 6, 9])
def test_rows_of_a_shared_front(gpu_lib, bits, page, new):
    """A front whose rows, eight sequences of four heads a group, are 64, 96, 128, 192 and
    288: items of the front in every kind."""
    c = BothCoded(gpu_lib, bits, 1, 1, 128, page, 160, 8, 50, seed=new)
    c.append([8 * 128] + [0] * 7)
    c.fork([0] * 8)
    c.append([3, 70, 0, 1, 33, 300, 12, 128])
    c.append([new] * 8, new)
    q, o, _ = _run(gpu_lib, c, 4, new)
    _run(gpu_lib, c, 4, new, groups=i32([0, 0, 0, 0, 1, 1, 1, 1]), q=q)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sequences", [16, 17, 20, 32, 33])
def test_workgroups_of_the_last_kernel(gpu_lib, bits, d, sequences):
    """Eight K/V heads, a row a sequence: at most half as many workgroups as compute units (two
    for the dimensions), at most as many, and more; parts of some sequences to join."""
    c = BothCoded(gpu_lib, bits, 1, 8, d, 64, 14 * sequences, sequences, 13, seed=sequences)
    c.append([(511, 700, 3, 90)[i % 4] + i for i in range(sequences)])
    c.append([1] * sequences)
    _run(gpu_lib, c, 8, 1)


@pytest.mark.parametrize("bits,d", [(4, 128), (8, 128), (8, 64)])
@pytest.mark.parametrize("sequences", [3, 40])
def test_results_in_place(gpu_lib, bits, d, sequences):
    """o is q: no workgroup writes over queries that another reads; closed rows stay."""
    c = BothCoded(gpu_lib, bits, 1, 2, d, 64, 12 * sequences + 20, sequences, 20, seed=11)
    c.append([(600, 40, 900)[i % 3] if i < 9 else 100 + i for i in range(sequences)])
    c.append([5 - i % 2 for i in range(sequences)], 5)
    q = c.rand(sequences, 5, 8, d)
    kept = q.clone()
    lse = torch.zeros(sequences, 5, 8, device="cuda")
    gpu_lib.attend(c.g.plan(8, 5), 0, q, out=q, lse=lse)
    torch.cuda.synchronize()
    closed = torch.arange(5, device="cuda")[None] >= c.g.open[:, None]
    assert torch.equal(q[closed], kept[closed]) and not lse[closed].any()
    out = torch.where(closed[..., None, None], torch.zeros_like(q), q)
    check_attend(c, 5, kept, out, lse, 0, d ** -0.5)


@pytest.mark.parametrize("bits", [4, 8])
def test_a_sequence_alone_and_beside_others(gpu_lib, bits):
    """How a sequence's keys are cut, and so the order of its sums and which of its
    probabilities have 16 bits, follows from the batch: both answers are within the bound
    of the definition, their lse within that of its sums, and each batch's own repeats
    itself bit for bit."""
    got = []
    for others in (0, 30):
        c = BothCoded(gpu_lib, bits, 1, 2, 128, 64, 60 + 60 * others, 1 + others, 60, seed=3)
        K, V = c.rand(1 + others, 3000, 1, 2, 128), c.rand(1 + others, 3000, 1, 2, 128)
        g = torch.Generator(device="cuda").manual_seed(5)
        K[0] = torch.randn(K[0].shape, generator=g, device="cuda").to(BF)
        V[0] = torch.randn(K[0].shape, generator=g, device="cuda").to(BF)
        c.append([3000] * (1 + others), 3000, K, V)
        k, v, q = (torch.randn(1, 4, *x, generator=g, device="cuda").to(BF)
                   for x in ((1, 2, 128), (1, 2, 128), (8, 128)))
        k, v, q = (x.repeat(1 + others, *[1] * (x.dim() - 1)) for x in (k, v, q))
        c.append([4] * (1 + others), 4, k, v)
        _, o, l = _run(gpu_lib, c, 8, 4, q=q)
        for _ in range(2):
            o2 = torch.zeros_like(o)
            l2 = torch.zeros_like(l)
            gpu_lib.attend(c.g.plan(8, 4), 0, q, out=o2, lse=l2)
            assert torch.equal(o, o2) and torch.equal(l, l2)
        got.append((o[0].double(), l[0].double(), c.o.sequence(0, 0)))
    (o1, l1, kv1), (o2, l2, kv2) = got
    assert all((a == b).all() for a, b in zip(kv1, kv2))
    # a bf16 probability each: 2^-8 of sum p |v|, with |v| at most its largest; results are
    # rounded to bf16 twice, 2^-8 each; sums of 3004 keys
    most = float(abs(kv1[1]).max())
    assert (o1 - o2).abs().max() <= (2.0 ** -8 * 2 + 3100 * 2.0 ** -23) * most + 2.0 ** -7 * o1.abs().max()
    assert (l1 - l2).abs().max() <= 2 * (3100 * 2.0 ** -24 + 2.0 ** -20 * l1.abs().max())
