"""Forks of the views, and rounds of the operators together: samples of one
prompt are drafted for, scored over the shared cache, verified from given random
numbers and cut back, with views and cache in step."""
import numpy as np
import pytest
import torch

import synth
from oracle import pages as OP
from pages_common import Both, check_attend, i32

pytestmark = pytest.mark.gpu


def _regions(v):
    r = {"pos": v.pos, "boundary": v.boundary()}
    if v.window() is not None:
        r.update(zip(("k", "v"), v.window()))
    if v.summary() is not None:
        r.update(zip(("m", "eta"), v.summary()))
    if v.pooled() is not None:
        r.update(zip(("pk", "pv"), v.pooled()))
    return {k: t for k, t in r.items() if t is not None}


def _filled(ldr, s, batch, seed=0):
    torch.manual_seed(seed)
    v = ldr.Views(s, batch, synth.make_G(s, device="cuda")).init()
    K, V, h = next(iter(synth.prefix_chunks(s, batch, 200, 200, device="cuda")))
    v.update(i32([200 - 7 * b for b in range(batch)]), K, V, h)
    return v


@pytest.mark.parametrize("shape", [synth.TINY, synth.QWEN3_8B, synth.QWEN3_8B_POOLED],
                         ids=["tiny", "8b", "8b-pooled"])
def test_views_fork(gpu_lib, shape):
    v = _filled(gpu_lib, shape, 6)
    ref = gpu_lib.Views(shape, 6, v.G).init()
    torch.cuda.synchronize()
    empty, before = ref.arena.clone().view(6, -1), v.arena.clone().view(6, -1)
    pos = v.pos.clone()
    src = [0, 0, 2, -1, 2, 5]
    v.fork(i32(src))
    torch.cuda.synchronize()
    got = v.arena.view(6, -1)
    for b, a in enumerate(src):
        assert torch.equal(got[b], before[a] if a >= 0 else empty[b]), b
        assert int(v.pos[b]) == (int(pos[a]) if a >= 0 else 0)
    assert v.status() == gpu_lib.LDR_OK
    for bad in ([1, 0, 2, 3, 4, 5], [0, 6, 2, 3, 4, 5], [0, -2, 2, 3, 4, 5], [-1, 0, 2, 3, 4, 5]):
        was = v.arena.clone().view(6, -1)
        v.fork(i32(bad))
        torch.cuda.synchronize()
        now = v.arena.view(6, -1)
        for b, a in enumerate(bad):
            stays = a < -1 or a >= 6 or (a >= 0 and bad[a] != a)
            if stays:
                assert torch.equal(now[b], was[b]), (bad, b)
        assert v.status(clear=True) == gpu_lib.LDR_ERANGE
    with pytest.raises(gpu_lib.LdrError):
        v.fork(i32([0]))


def test_forked_views_draft_the_same(gpu_lib):
    """A copy proposes what its source proposes, and goes its own way after an update."""
    s = synth.TINY
    v = _filled(gpu_lib, s, 3)
    w = gpu_lib.DraftWeights(synth.make_weights(s, gain_std=0.1, device="cuda"))
    v.fork(i32([0, 1, 0]))
    anchor = i32([5, 6, 5])
    z = gpu_lib.draft_step(v, w, anchor)
    torch.cuda.synchronize()
    assert torch.equal(z[0], z[2]) and not torch.equal(z[0], z[1])
    K, V, h = synth.decode_rows(s, 3, s.block + 1, 0, device="cuda")
    v.update(i32([2, 0, 4]), K, V, h)
    z = gpu_lib.draft_step(v, w, anchor)
    torch.cuda.synchronize()
    assert not torch.equal(z[0], z[2])


@pytest.mark.parametrize("shape", [synth.TINY, synth.TINY.replace(
    name="small", dtype="bf16", n_layers=2, n_kv_heads=2, head_dim=128)], ids=["tiny", "bf16"])
def test_rounds_together(gpu_lib, shape):
    """Four samples of one prompt for three rounds. The target is stood in for by
    the attention's output through a random vocabulary head; every operator is
    compared with its plain form on its own inputs, and the views keep the rows
    that the cache keeps."""
    s, batch, B = shape, 4, shape.block
    dt = s.torch_dtype
    c = Both(gpu_lib, s.n_layers, s.n_kv_heads, s.head_dim, 32, 64, batch, 16, dt, seed=1)
    v = gpu_lib.Views(s, batch, synth.make_G(s, device="cuda")).init()
    w = gpu_lib.DraftWeights(synth.make_weights(s, gain_std=0.1, device="cuda"))
    # the prompt goes into sequence 0 of both, then to every sample
    n = [150, 0, 0, 0]
    K = c.rand(batch, 150, s.n_layers, s.n_kv_heads, s.head_dim)
    V = c.rand(*K.shape)
    h = c.rand(batch, s.n_feat_layers, s.hidden)
    v.update(i32(n), K, V, h)
    c.append(n, 150, K, V)
    v.fork(i32([0] * batch))
    c.fork([0] * batch)
    head = c.rand(s.n_q_heads * s.head_dim, s.vocab).float() * 0.3
    anchor = i32([1, 2, 3, 4])
    for step in range(3):
        z = gpu_lib.draft_step(v, w, anchor)
        tok, _, _ = gpu_lib.sample(z.view(-1, s.vocab), 1.0, 0, 3, step)
        tok = tok.view(batch, B)
        K = c.rand(batch, B + 1, s.n_layers, s.n_kv_heads, s.head_dim)
        V = c.rand(*K.shape)
        c.append([B + 1] * batch, B + 1, K, V)
        plan = c.g.plan(s.n_q_heads, B + 1)
        q = c.rand(batch, B + 1, s.n_q_heads, s.head_dim)
        for layer in range(s.n_layers):
            lse = torch.zeros(batch, B + 1, s.n_q_heads, device="cuda")
            out = gpu_lib.attend(plan, layer, q, lse=lse)
            torch.cuda.synchronize()
            check_attend(c, B + 1, q, out, lse, layer, s.head_dim ** -0.5)
        logits = out.float().reshape(batch * (B + 1), -1) @ head
        target = logits.view(batch, B + 1, -1)
        target[:, :B] += z
        P, Q = target.softmax(-1), z.softmax(-1)
        u = torch.rand(batch, B + 1, generator=c.gen, device="cuda")
        acc, nxt, n_new = gpu_lib.verify_probs(P, Q, tok, u)
        torch.cuda.synchronize()
        for b in range(batch):
            assert (int(acc[b]), int(nxt[b])) == OP.verify_probs(
                P[b].cpu().numpy(), Q[b].cpu().numpy(), tok[b].cpu().numpy(), None,
                u[b].cpu().numpy())
        c.g.keep(n_new)
        c.o.keep(n_new.tolist())
        c.check()
        v.update(n_new, K, V, h)
        torch.cuda.synchronize()
        assert v.pos.tolist() == c.o.rows
        # the window holds the cache's last rows, slot p mod W
        Kw = v.window()[0].double().cpu().numpy()
        for b in range(batch):
            for layer in range(s.n_layers):
                k, _ = c.o.sequence(layer, b)
                for p in range(max(0, len(k) - s.window), len(k)):
                    assert np.array_equal(Kw[b, layer, :, p % s.window], k[p])
        anchor = nxt
    assert c.g.status() == gpu_lib.LDR_OK and v.status() == gpu_lib.LDR_OK
