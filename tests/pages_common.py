"""A GPU cache and its plain form driven by the same calls, and the error bound
of the attention kernels."""
import numpy as np
import torch

from oracle import pages as OP

DEV = "cuda"


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Both:
    def __init__(self, ldr, layers, hkv, d, page, n_pages, batch, max_pages, dtype, seed=0,
                 stream=None):
        self.g = ldr.Pages(layers, hkv, d, page, n_pages, batch, max_pages, dtype,
                           stream=stream).init()
        self.o = OP.Cache(layers, hkv, d, page, n_pages, batch, max_pages)
        self.layers, self.dtype, self.batch = layers, dtype, batch
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        # what free pages hold is not defined: NaN, so that a use of it shows
        self.g.pool.fill_(float("nan"))

    def rand(self, *shape):
        return torch.randn(shape, generator=self.gen, device=DEV).to(self.dtype)

    def append(self, n, max_new=None, K=None, V=None):
        max_new = max(1, max(int(x) for x in n)) if max_new is None else max_new
        shape = (self.batch, max_new, self.layers, self.g.hkv, self.g.d)
        K = self.rand(*shape) if K is None else K
        V = self.rand(*shape) if V is None else V
        self.g.append(i32(n), K, V)
        self.o.reserve(n, max_new)
        self.o.write(K.double().cpu().numpy(), V.double().cpu().numpy())

    def keep(self, kept):
        self.g.keep(i32(kept))
        self.o.keep(kept)

    def fork(self, src):
        self.g.fork(i32(src))
        self.o.fork(src)

    def compact(self):
        self.g.compact()
        self.o.compact()

    def check(self, contents=True):
        torch.cuda.synchronize()
        g, o = self.g, self.o
        assert g.rows.tolist() == o.rows and g.open.tolist() == o.open
        assert g.refs.tolist() == o.refs
        assert np.array_equal(g.table.cpu().numpy(), o.tables())
        if not contents:
            return
        for layer in range(self.layers):
            K, V = g.k(layer).double().cpu().numpy(), g.v(layer).double().cpu().numpy()
            for b in range(self.batch):
                if o.rows[b] == 0:
                    continue
                ids, n = o.table[b], o.rows[b]
                k = K[ids].transpose(0, 2, 1, 3).reshape(-1, g.hkv, g.d)[:n]
                v = V[ids].transpose(0, 3, 1, 2).reshape(-1, g.hkv, g.d)[:n]
                ok, ov = o.sequence(layer, b)
                assert np.array_equal(k, ok, equal_nan=True), (layer, b)
                assert np.array_equal(v, ov, equal_nan=True), (layer, b)


def check_attend(both, plan_new, q, out, lse, layer, scale, before=0.0):
    """Every open row within the bound of its arithmetic, the others as before.

    With e = 2^-24 (half a step of fp32): a score is off by at most
    ds = (d + 3) e scale sum_j |q_j k_j| (a sum of d products in any order, the
    scaling) and its exponent by the rounding of the two products subtracted in
    it, 3 e max |s|; a weight by that and the 4 e of the exponential (about one
    step) relative, and by 2^-8 where it is rounded to bf16; the sums over n keys add n e, the
    joining of parts 16 e. Weights and their sum are both off, hence twice. The
    result is rounded to its type."""
    o, lz = both.o, None if lse is None else lse.double().cpu().numpy()
    got, qn = out.double().cpu().numpy(), q.double().cpu().numpy()
    bf16 = both.dtype == torch.bfloat16
    e, half = 2.0 ** -24, 2.0 ** -8 if bf16 else 2.0 ** -24
    worst = 0.0
    for b in range(both.batch):
        m = min(o.open[b], plan_new)
        assert np.all(got[b, m:] == before), b
        if lz is not None:
            assert np.all(lz[b, m:] == before), b
        if m == 0:
            continue
        K, V = o.sequence(layer, b)
        keep = len(K) - (o.open[b] - m)          # rows the plan's queries end at
        K, V = K[:keep], V[:keep]
        ref, rl = OP.attend(qn[b, :m], K, V, scale)
        size, _ = OP.attend(qn[b, :m], K, np.abs(V), scale)
        rep = q.shape[2] // K.shape[1]
        with np.errstate(all="ignore"):
            mass = np.einsum("ihd,khd->ihk", np.abs(qn[b, :m]), np.abs(K).repeat(rep, 1)) * scale
            mass = np.where(np.isfinite(mass), mass, 0.0).max(-1)
        ds = (q.shape[3] + 6) * e * mass
        w = 2 * (ds + 4 * e) + (len(K) + 16) * e
        tol = (w + (half if bf16 else 0.0))[..., None] * size + half * np.abs(ref) + 1e-30
        assert np.array_equal(np.isnan(got[b, :m]), np.isnan(ref)), b
        inf = np.isinf(ref)
        assert np.array_equal(got[b, :m][inf], ref[inf]), b
        fin = np.isfinite(ref)
        assert np.all(np.isfinite(got[b, :m][fin]))
        err = np.abs(got[b, :m][fin] - ref[fin])
        assert np.all(err <= tol[fin]), (b, (err / tol[fin]).max())
        worst = max(worst, (err / tol[fin]).max(initial=0.0))
        if lz is not None:
            ok = np.isfinite(rl)
            diff = np.abs(np.where(ok, lz[b, :m], 0.0) - np.where(ok, rl, 0.0))
            assert np.array_equal(lz[b, :m][np.isneginf(rl)], rl[np.isneginf(rl)])
            lt = ds + (len(K) + 20) * e + 4 * e * np.abs(rl)
            assert np.all(diff[ok] <= lt[ok]), b
    return worst
