"""Rows in codes and log probabilities: the oracle against closed forms and torch, sizes
and refusals of the calls on the host."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pages as OP


@pytest.mark.parametrize("bits", [4, 8])
def test_codes_are_the_nearest_of_the_smallest_scale(bits):
    grid, limit, lowest, top = OP.MX[bits]
    rng = np.random.default_rng(bits)
    x = rng.standard_normal((200, 64)) * np.exp2(rng.integers(-20, 20, (200, 1)))
    v = OP.mx_values(x, bits)
    a = np.abs(x).reshape(200, 2, 32)
    # of the three scales around, none smaller can hold the block, and no code is nearer
    for r in range(200):
        for k in range(2):
            block, got = x[r, 32 * k:32 * k + 32], v[r, 32 * k:32 * k + 32]
            e = int(np.ceil(np.log2(a[r, k].max() / limit)))
            s = 2.0 ** e
            assert a[r, k].max() <= limit * s and a[r, k].max() > limit * s / 2
            codes = np.array(sorted([-g * s for g in grid] + [g * s for g in grid]))
            assert np.all(np.isin(got, codes))
            assert np.all(np.abs(got - block) <= np.abs(block[:, None] - codes).min(1))
    # half a step of the value's binade, and of the smallest
    half = 2.0 ** (-2 if bits == 4 else -4)
    small = a.max(-1, keepdims=True) / limit * 2 * (0.25 if bits == 4 else 2.0 ** -10)
    err = np.abs(v - x).reshape(200, 2, 32)
    assert np.all(err <= np.maximum(half * a, small))


def test_codes_of_8_bits_are_those_of_torch():
    grid = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().tolist()
    assert grid == OP.MX[8][0]
    x = torch.randn(50, 64, dtype=torch.float64)
    x[:, ::32] = 448.0                    # the scale is 1
    ref = x.float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(OP.mx_values(x.float().double().numpy(), 8), ref)


@pytest.mark.parametrize("bits", [4, 8])
def test_codes_at_the_edges(bits):
    grid, limit, lowest, top = OP.MX[bits]
    x = np.zeros(32)
    assert np.array_equal(OP.mx_values(x, bits), x)
    x[0] = limit                          # held as the largest code
    assert OP.mx_values(x, bits)[0] == grid[-1]
    x[0] = limit * 1.0001                 # one scale more
    assert OP.mx_values(x, bits)[0] == 2 * grid[np.argmin(np.abs(np.array(grid) - limit * 1.0001 / 2))]
    x[0] = 1.99 * 2.0 ** 127
    assert OP.mx_values(x, bits)[0] == top and np.isfinite(np.float32(top))
    x[0] = 2.0 ** -133                    # below half of the smallest code
    assert OP.mx_values(x, bits)[0] == 0.0
    for bad in (np.nan, np.inf, -np.inf):
        y = np.zeros(64)
        y[3] = bad
        v = OP.mx_values(y, bits)
        assert np.isnan(v[:32]).all() and not v[32:].any()
    # every value is a bf16 number, and coded again it is itself
    x = np.random.default_rng(0).standard_normal((100, 32)) * np.exp2(np.arange(100) * 2.4 - 120)[:, None]
    v = OP.mx_values(np.clip(x, -top, top), bits)
    t = torch.tensor(v)
    assert torch.equal(t.to(torch.bfloat16).double(), t)
    assert np.array_equal(OP.mx_values(v, bits), v)


@pytest.mark.parametrize("T", [1.0, 0.5])
def test_logprobs_are_those_of_torch(T):
    z = torch.randn(900, dtype=torch.float64) * 3
    lp = torch.log_softmax(z / T, 0)
    for y in (0, 899, int(z.argmax())):
        got = OP.logprobs(z.numpy(), y, T, 10)
        assert got[0] == pytest.approx(lp[y].item(), rel=1e-12)
        assert got[1] == pytest.approx(-(lp.exp() * lp).sum().item(), rel=1e-12)
        assert got[2] == int((z > z[y]).sum())
        assert list(got[3]) == torch.topk(z, 10)[1].tolist()
        assert np.allclose(got[4], torch.topk(lp, 10)[0].numpy(), rtol=1e-12)


def test_logprobs_at_the_edges():
    inf, nan = np.inf, np.nan
    assert OP.logprobs([0.0], 0, 1.0, 1)[:4] == (0.0, 0.0, 0, [0])
    lp, h, r, order, tl = OP.logprobs([1.0, 1.0, -inf, 1.0], 3, 1.0, 4)
    assert lp == pytest.approx(-np.log(3)) and h == pytest.approx(np.log(3)) and r == 2
    assert order == [0, 1, 3, 2] and tl[3] == -inf
    lp, h, r, order, tl = OP.logprobs([-inf] * 3, 1, 1.0, 2)
    assert lp == -inf and h == 0 and r == 1 and order == [0, 1] and list(tl) == [-inf] * 2
    lp, h, r, order, _ = OP.logprobs([nan, 1.0, nan, 2.0], 2, 1.0, 4)
    assert np.isnan(lp) and np.isnan(h) and r == 3 and order == [3, 1, 0, 2]
    assert OP.logprobs([0.0, 1.0], 2, 1.0, 0)[0] == -inf
    assert OP.logprobs([0.0, 1.0], -1, 1.0, 0)[2] == 2


# ------------------------------------------------------- refusals, on the host

@pytest.fixture(scope="module")
def L():
    from paper_2609_37029_amd import ldr
    return ldr


GOOD = dict(n_layers=5, n_kv_heads=8, head_dim=128, page=64, n_pages=2048, batch=16,
            max_pages=600)


@pytest.mark.parametrize("bits,dtype", [(4, 4), (8, 8)])
@pytest.mark.parametrize("d,page", [(64, 32), (128, 64), (64, 256), (128, 128)])
def test_coded_pool_sizes(L, bits, dtype, d, page):
    c = ctypes.byref(L.PagesConfig(**{**GOOD, "head_dim": d, "page": page}, dtype=dtype))
    row = d * bits // 8 + d // 32
    assert L.lib().ldr_pages_pool_bytes(c) == 5 * 2 * 2048 * 8 * page * row
    assert L.lib().ldr_attend_workspace_bytes(c, 32, 17) > 0
    p = L.Pages(2, 3, d, page, 4, 2, 3, device="cpu", codes=f"mxfp{bits}")
    assert p.pool.shape == (2, 2, 4, 3, page * row) and p.pool.dtype == torch.uint8
    for view in (p.k, p.v):
        with pytest.raises(L.LdrError):
            view(0)


@pytest.mark.parametrize("dtype", [-1, 2, 3, 5, 6, 7, 9, 16])
def test_other_codes_are_refused(L, dtype):
    c = ctypes.byref(L.PagesConfig(**GOOD, dtype=dtype))
    assert L.lib().ldr_pages_pool_bytes(c) == 0


def test_codes_belong_to_caches_alone(L):
    """Drafters and corrections have no coded types."""
    lib, fake = L.lib(), ctypes.c_void_p(1 << 20)
    import synth
    for dtype in (L.LDR_MXFP4, L.LDR_MXFP8):
        cfg = L.config(synth.TINY)
        cfg.dtype = dtype
        assert lib.ldr_config_check(ctypes.byref(cfg)) == L.LDR_EINVAL
        need = lib.ldr_sample_workspace_bytes(2, 64)
        assert lib.ldr_sample_markov(fake, 2, 2, 64, fake, fake, fake, 8, dtype, 1.0, 0, 1, 1, fake,
                                     fake, fake, fake, need, None) == L.LDR_EINVAL


def test_binding_refuses_what_it_would_misread(L):
    for kw in (dict(codes="mxfp6"), dict(codes="mxfp4", dtype=torch.float32), dict(codes="")):
        with pytest.raises(L.LdrError):
            L.Pages(2, 2, 64, 32, 8, 3, 4, device="cpu", **kw)
    p = L.Pages(2, 2, 64, 32, 8, 3, 4, device="cpu", codes="mxfp4")
    i32 = torch.zeros(3, dtype=torch.int32)
    K = torch.zeros(3, 4, 2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(L.LdrError):
        p.write(K.float(), K.float())
    for first, n in ((i32.long(), i32), (i32, i32[:2]), (i32, i32.float())):
        with pytest.raises(L.LdrError):
            p.read(first, n, 4)
    for kw in (dict(), dict(max_rows=0), dict(max_rows=4, layer=2), dict(out=(K, K.float())),
               dict(out=(K, K[:, :3])), dict(out=(K[0], K[0])), dict(out=(K, K), max_rows=3),
               dict(out=(K, K), n_layers=1)):
        with pytest.raises(L.LdrError):
            p.read(i32, i32, **kw)
    # host memory, otherwise as it should be: no handle
    with pytest.raises(Exception):
        p.read(i32, i32, 4)
    z, y = torch.zeros(2, 3, 50), torch.zeros(2, 3, dtype=torch.int32)
    for args, kw in (((z.double(), y), {}), ((z, y.long()), {}), ((z, y[:1]), {}), ((z[0], y), {}),
                     ((z, y), dict(top_n=51)), ((z, y), dict(top_n=65)), ((z, y), dict(top_n=-1)),
                     ((z[..., ::2], y), {}), ((z.transpose(0, 1).contiguous().transpose(0, 1), y), {}),
                     ((z, y), dict(n_rows=torch.zeros(3, dtype=torch.int32))),
                     ((z, y), dict(workspace=torch.zeros(9))),
                     ((z, y), dict(out=(torch.zeros(2, 3),) * 5))):
        with pytest.raises(L.LdrError):
            L.logprobs(*args, **kw)
    with pytest.raises(L.LdrError, match="logprobs on cpu"):
        L.logprobs(z, y, top_n=3)


def test_read_host_refusals(L):
    lib, fake = L.lib(), ctypes.c_void_p(1 << 20)
    assert lib.ldr_pages_read(None, 0, 1, fake, fake, fake, fake, 17, None) == L.LDR_EINVAL


def test_logprobs_host_refusals(L):
    lib, E = L.lib(), L.LDR_EINVAL
    at = lambda i: ctypes.c_void_p((1 << 20) + (i << 16))  # noqa: E731
    need = lib.ldr_logprobs_workspace_bytes(2, 4, 64, 3)
    good = [at(0), 64, at(1), at(2), 2, 4, 64, 1.0, 3, at(3), at(4), at(5), at(6), at(7), at(8), need,
            None]
    assert need > 0
    bad = [(i, None) for i in (0, 2, 9, 10, 11, 12, 13, 14)]
    bad += [(1, 63), (1, (1 << 40) + 1), (4, 0), (4, 65536), (5, 0), (5, 65536), (6, 0),
            (6, (1 << 30) + 1), (8, -1), (8, 65), (15, need - 1)]
    bad += [(7, t) for t in (0.0, -1.0, float("nan"), float("inf"), 1e-39, 1e-45, 3e38)]
    bad += [(i, ctypes.c_void_p((1 << 24) + 2)) for i in (0, 2, 3, 9, 10, 11, 12, 13)]
    bad += [(14, ctypes.c_void_p((1 << 24) + 128))]
    bad += [(i, at(0)) for i in (9, 10, 11, 12, 13, 14)]          # over the logits
    bad += [(i, at(1)) for i in (9, 14)] + [(i, at(2)) for i in (10, 14)]
    bad += [(10, at(3)), (12, at(4)), (13, at(6)), (14, at(7))]   # over each other
    for i, x in bad:
        assert lib.ldr_logprobs(*good[:i], x, *good[i + 1:]) == E, (i, x)
    for sizes in ((0, 4, 64, 3), (65536, 4, 64, 3), (2, 0, 64, 3), (2, 65536, 64, 3), (2, 4, 0, 0),
                  (2, 4, (1 << 30) + 1, 3), (2, 4, 64, -1), (2, 4, 64, 65), (2, 4, 5, 6)):
        assert lib.ldr_logprobs_workspace_bytes(*sizes) == 0
