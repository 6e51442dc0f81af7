"""The operators of a coded cache in rounds, as a server runs them: samples of one prompt are
drafted for, scored over the cache, verified, answered with log probabilities and cut back;
the views that draft for them are made from rows read back from the cache."""
import numpy as np
import pytest
import torch

import synth
from mx_common import BothCoded
from oracle import pages as OP
from pages_common import check_attend, i32

pytestmark = pytest.mark.gpu

SHAPE = synth.TINY.replace(name="small", dtype="bf16", n_layers=2, n_kv_heads=2, head_dim=128)


@pytest.mark.parametrize("bits", [4, 8])
def test_rounds_together(gpu_lib, bits):
    s, batch, B = SHAPE, 4, SHAPE.block
    c = BothCoded(gpu_lib, bits, s.n_layers, s.n_kv_heads, s.head_dim, 32, 64, batch, 16, seed=1)
    v = gpu_lib.Views(s, batch, synth.make_G(s, device="cuda")).init()
    w = gpu_lib.DraftWeights(synth.make_weights(s, gain_std=0.1, device="cuda"))
    n = [150, 0, 0, 0]
    c.append(n, 150)
    # the views of the values that the cache holds
    K, V = c.g.read(c.g.rows - c.g.open, c.g.open, 150)
    h = c.rand(batch, s.n_feat_layers, s.hidden)
    v.update(i32(n), K, V, h)
    v.fork(i32([0] * batch))
    c.fork([0] * batch)
    head = c.rand(s.n_q_heads * s.head_dim, s.vocab).float() * 0.3
    anchor = i32([1, 2, 3, 4])
    for step in range(3):
        z = gpu_lib.draft_step(v, w, anchor)
        tok, _, _ = gpu_lib.sample(z.view(-1, s.vocab), 1.0, 0, 3, step)
        tok = tok.view(batch, B)
        c.append([B + 1] * batch, B + 1)
        K, V = c.g.read(c.g.rows - c.g.open, c.g.open, B + 1)
        plan = c.g.plan(s.n_q_heads, B + 1)
        q = c.rand(batch, B + 1, s.n_q_heads, s.head_dim)
        for layer in range(s.n_layers):
            lse = torch.zeros(batch, B + 1, s.n_q_heads, device="cuda")
            out = gpu_lib.attend(plan, layer, q, lse=lse)
            torch.cuda.synchronize()
            check_attend(c, B + 1, q, out, lse, layer, s.head_dim ** -0.5)
        target = (out.float().reshape(batch * (B + 1), -1) @ head).view(batch, B + 1, -1)
        target[:, :B] += z
        P, Q = target.softmax(-1), z.softmax(-1)
        u = torch.rand(batch, B + 1, generator=c.gen, device="cuda")
        acc, nxt, n_new = gpu_lib.verify_probs(P, Q, tok, u)
        # what was emitted: the accepted tokens, then the next one
        emitted = torch.cat((tok, tok[:, :1]), 1)
        emitted = emitted.scatter(1, acc.long()[:, None], nxt[:, None]).contiguous()
        lp, ent, rank, top, tlp = gpu_lib.logprobs(target, emitted, top_n=4, n_rows=n_new)
        torch.cuda.synchronize()
        zs = target.double().cpu().numpy()
        for b in range(batch):
            assert (int(acc[b]), int(nxt[b])) == OP.verify_probs(
                P[b].cpu().numpy(), Q[b].cpu().numpy(), tok[b].cpu().numpy(), None,
                u[b].cpu().numpy())
            for i in range(B + 1):
                if i >= int(n_new[b]):
                    assert not top[b, i].any() and float(lp[b, i]) == 0
                    continue
                r = OP.logprobs(zs[b, i], int(emitted[b, i]), 1.0, 4)
                assert int(rank[b, i]) == r[2] and top[b, i].tolist() == list(r[3])
                # 2^-24 for each of some 60 roundings (test_gpu_logprobs), of values up to 2^5
                for got, ref in ((lp[b, i], r[0]), (ent[b, i], r[1]), (tlp[b, i, 3], r[4][3])):
                    assert abs(float(got) - ref) <= 60 * 2.0 ** -24 * 32
        c.g.keep(n_new)
        c.o.keep(n_new.tolist())
        c.check()
        v.update(n_new, K, V, h)
        torch.cuda.synchronize()
        assert v.pos.tolist() == c.o.rows
        Kw = v.window()[0].double().cpu().numpy()
        for b in range(batch):
            for layer in range(s.n_layers):
                k, _ = c.o.sequence(layer, b)
                for p in range(max(0, len(k) - s.window), len(k)):
                    assert np.array_equal(Kw[b, layer, :, p % s.window], k[p])
        anchor = nxt
    assert c.g.status() == gpu_lib.LDR_OK and v.status() == gpu_lib.LDR_OK


def test_two_captured_rounds_on_one_cache(gpu_lib):
    """Two graphs with workspaces of their own, replayed in turn with eager calls between."""
    c = BothCoded(gpu_lib, 8, 1, 2, 128, 64, 60, 2, 20, seed=2)
    c.append([700, 90])
    c.append([3, 3])
    qs, outs, graphs, refs = [], [], [], []
    kept = []       # the graphs' workspaces: theirs as long as they are replayed
    for g in range(2):
        q = c.rand(2, 3, 8, 128)
        out = torch.zeros(2, 3, 8, 128, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(c.g.attend_workspace_bytes(8, 3), dtype=torch.uint8, device="cuda")
        gpu_lib.attend(c.g.plan(8, 3, workspace=ws), 0, q, out=out)
        torch.cuda.synchronize()
        refs.append(out.clone())
        kept.append(ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            gpu_lib.attend(c.g.plan(8, 3, workspace=ws), 0, q, out=out)
        qs.append(q), outs.append(out), graphs.append(graph)
    for k in range(4):
        for g in (k % 2, 1 - k % 2):
            outs[g].zero_()
            graphs[g].replay()
            extra = gpu_lib.attend(c.g.plan(8, 3), 0, qs[1 - g])
            torch.cuda.synchronize()
            assert torch.equal(outs[g], refs[g]) and torch.equal(extra, refs[1 - g])


def test_plans_of_another_state_are_refused(gpu_lib):
    """A plan from before a change of the cache writes nothing and says so."""
    c = BothCoded(gpu_lib, 4, 1, 1, 64, 32, 40, 1, 30, seed=3)
    c.append([600])
    c.append([2])
    plan = c.g.plan(2, 2)
    c.append([2])
    q = c.rand(1, 2, 2, 64)
    out = torch.full((1, 2, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    gpu_lib.attend(plan, 0, q, out=out)
    torch.cuda.synchronize()
    assert bool((out == 5.0).all()) and c.g.status(clear=True) == gpu_lib.LDR_EINVAL
