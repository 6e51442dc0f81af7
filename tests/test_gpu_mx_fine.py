"""Probabilities of 16 bits where the attention over a coded cache keeps them: in the last
kernel, and in items of at most 32 rows with at most four steps of 32 keys a wave. The rows of
mx_fine are off by some thirty times their bound where that is not so (test_oracle_mx_fine.py)."""
import numpy as np
import pytest
import torch

import mx_fine as F
from mx_common import BothCoded
from oracle import pages as OP

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _check(ldr, bits, d, hkv, rep, page, lengths, new, front=0, in_place=False):
    """Sequences of these lengths, behind `front` rows in common, and `new` rows more each."""
    b, hq = len(lengths), hkv * rep
    per = (front + max(lengths) + new) // page + 2
    c = BothCoded(ldr, bits, 1, hkv, d, page, b * per + 1, b, per)
    rng = np.random.default_rng(7)

    def put(counts):
        most = max(1, max(counts))
        K, V = np.zeros((2, b, most, 1, hkv, d))
        for s in range(b):
            K[s, :, 0], V[s, :, 0] = F.rows(rng, most, hkv, d)
        c.append(counts, most, *(torch.tensor(x).to(BF).cuda() for x in (K, V)))

    if front:
        put([front] + [0] * (b - 1))
        c.fork([0] * b)
    put(lengths)
    put([new] * b)
    q = torch.tensor(F.queries((b, new, hq, d))).to(BF).cuda()
    qn = q.double().cpu().numpy()
    out = ldr.attend(c.g.plan(hq, new), 0, q, out=q if in_place else None, scale=F.SCALE)
    torch.cuda.synchronize()
    assert c.g.status() == ldr.LDR_OK
    got = out.double().cpu().numpy()
    for s in range(b):
        K, V = c.o.sequence(0, s)
        ref, _ = OP.attend(qn[s], K, V, F.SCALE)
        size, _ = OP.attend(qn[s], K, np.abs(V), F.SCALE)
        err, tol = np.abs(got[s] - ref), F.bound(ref, size, len(K), d)
        assert np.all(err <= tol), (s, (err / tol).max())


@pytest.mark.parametrize("bits,d,hkv,rep,page", [
    (4, 128, 2, 4, 64), (8, 128, 2, 4, 64), (4, 64, 4, 1, 32), (8, 64, 4, 1, 32), (4, 128, 3, 1, 32),
    (8, 128, 1, 2, 256)])
@pytest.mark.parametrize("new", [1, 17])
def test_keys_near_the_mask(gpu_lib, bits, d, hkv, rep, page, new):
    """Sequences that leave no keys to items: the last kernel alone, by few workgroups (two for
    the dimensions of 32 rows with head_dim 128)."""
    _check(gpu_lib, bits, d, hkv, rep, page, [1, 33, 300, 470], new)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("sequences", [20, 40])
def test_keys_near_the_mask_of_many_sequences(gpu_lib, bits, sequences):
    """More workgroups than half the compute units, and more than all."""
    _check(gpu_lib, bits, 128, 8, 1, 64, [(37 * i) % 130 + 1 for i in range(sequences)], 1)


@pytest.mark.parametrize("bits", [4, 8])
def test_keys_near_the_mask_in_place(gpu_lib, bits):
    _check(gpu_lib, bits, 128, 2, 4, 64, [100, 5, 300], 9, in_place=True)


@pytest.mark.parametrize("bits,d,hkv,rep,page", [
    (4, 128, 2, 4, 64), (8, 128, 2, 4, 64), (4, 64, 4, 1, 32), (8, 64, 4, 1, 32), (4, 128, 3, 1, 32),
    (8, 128, 1, 2, 256)])
@pytest.mark.parametrize("new", [1, 8])
def test_items_of_few_rows_and_keys(gpu_lib, bits, d, hkv, rep, page, new):
    """Few sequences of some thousand keys: chunks of 256, a step or none a wave."""
    _check(gpu_lib, bits, d, hkv, rep, page, [1100, 777, 2500], new)


@pytest.mark.parametrize("bits", [4, 8])
def test_fronts_of_few_rows_and_keys(gpu_lib, bits):
    """A front of 512 keys that four sequences share, 32 rows a head."""
    _check(gpu_lib, bits, 128, 2, 4, 64, [40, 3, 70, 1], 2, front=512)
