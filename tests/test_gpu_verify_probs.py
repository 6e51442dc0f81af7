"""Verification from given probabilities and random numbers against its plain
form in 64 bits: whole numbers, equal."""
import numpy as np
import pytest
import torch

from oracle import pages as OP

pytestmark = pytest.mark.gpu


def _inputs(batch, B, V, seed, sharp=4.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    y = torch.randint(0, V, (batch, B), generator=g, device="cuda")
    z = torch.randn(batch, B, V, generator=g, device="cuda") * 2
    z.scatter_add_(2, y[..., None], torch.full((batch, B, 1), sharp, device="cuda"))
    t = torch.randn(batch, B + 1, V, generator=g, device="cuda") * 2
    t[:, :B] = z + 0.4 * torch.randn(batch, B, V, generator=g, device="cuda")
    u = torch.rand(batch, B + 1, generator=g, device="cuda")
    return t.softmax(-1), z.softmax(-1), y.to(torch.int32), u


def _check(ldr, P, Q, y, u, n=None):
    acc, tok, n_new = ldr.verify_probs(P, Q, y, u, n_draft=n)
    torch.cuda.synchronize()
    assert torch.equal(n_new, acc + 1)
    for b in range(P.shape[0]):
        want = OP.verify_probs(P[b].cpu().numpy(), None if Q is None else Q[b].cpu().numpy(),
                               y[b].cpu().numpy(), None if n is None else int(n[b]),
                               u[b].cpu().numpy())
        assert (int(acc[b]), int(tok[b])) == want, b
    return acc, tok


@pytest.mark.parametrize("batch,B,V", [(1, 1, 1), (3, 4, 2), (5, 16, 63), (9, 3, 4095), (4, 2, 4097),
                                       (16, 16, 5003), (2, 33, 32000), (3, 8, 151936),
                                       (2, 300, 257)])
@pytest.mark.parametrize("proposal", ["probs", "tokens"])
def test_parity(gpu_lib, batch, B, V, proposal):
    for seed in range(3):
        P, Q, y, u = _inputs(batch, B, V, seed)
        n = torch.randint(-1, B + 2, (batch,), device="cuda", dtype=torch.int32)
        for nn in (None, n):
            _check(gpu_lib, P, Q if proposal == "probs" else None, y, u, nn)


def test_all_stops_occur(gpu_lib):
    """Acceptances, rejections and full blocks, so that the parity covers each."""
    P, Q, y, u = _inputs(64, 4, 500, 7, sharp=8.0)
    acc, _ = _check(gpu_lib, P, Q, y, u)
    assert set(acc.tolist()) == {0, 1, 2, 3, 4}


def test_ties_and_borders(gpu_lib):
    """Dyadic probabilities: sums on the border of u belong to the next token."""
    V = 8192
    P = torch.full((6, 2, V), 1.0 / V, device="cuda")
    Q = P[:, :1].clone()
    y = torch.zeros(6, 1, dtype=torch.int32, device="cuda")
    u = torch.tensor([[0.5, 0.0], [0.5, 0.5], [0.5, 1 / V], [0.5, 1 - 1 / V], [0.5, 0.25],
                      [0.5, 1 - 2.0 ** -24]], device="cuda")
    _, tok = _check(gpu_lib, P, Q, y, u)
    assert tok.tolist() == [0, V // 2, 1, V - 1, V // 4, V - 1]
    u[:, 0] = 1.0                        # u q = p: not below, rejected; the residual is empty
    acc, tok = _check(gpu_lib, P, Q, y, u)
    assert not acc.any() and tok.tolist() == [0, V // 2, 1, V - 1, V // 4, V - 1]


def test_values_that_are_no_probabilities(gpu_lib):
    P, Q, y, u = _inputs(8, 3, 5000, 11)
    P[0, :, 100:200] = float("nan")
    P[1, :, 7] = float("inf")
    P[2, :, ::2] = -1.0
    P[3] = 0.0
    Q[4] = float("nan")
    u[5, -1], u[6, -1], u[7, -1] = float("nan"), 1.0, -0.5
    _check(gpu_lib, P, Q, y, u)
    _check(gpu_lib, P, None, y, u)
    y[:, 0] = torch.tensor([-1, 5000, 1 << 30, -(1 << 31), 3, 4, 5, 6], device="cuda")
    _check(gpu_lib, P, Q, y, u)
    _check(gpu_lib, P, None, y, u)


def test_frequencies(gpu_lib):
    """Tokens of the first position follow the target whatever the draft says:
    within 5 standard deviations."""
    n, V = 20000, 5
    rng = np.random.default_rng(0)
    p, q = rng.dirichlet(np.ones(V)), rng.dirichlet(np.ones(V))
    y = rng.choice(V, size=(n, 1), p=q)
    dev = lambda x, t=torch.float32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    P = dev(p).expand(n, 2, V).contiguous()
    acc, tok, _ = gpu_lib.verify_probs(P, dev(q).expand(n, 1, V).contiguous(), dev(y, torch.int32),
                                       dev(rng.random((n, 2))))
    first = np.where(acc.cpu().numpy() > 0, y[:, 0], tok.cpu().numpy())
    count = np.bincount(first, minlength=V)
    assert np.all(np.abs(count - n * p) < 5 * np.sqrt(n * p * (1 - p)))


def test_rows_off_16_bytes_and_graph(gpu_lib):
    """An odd vocabulary inside a larger buffer; captured and replayed."""
    buf = torch.rand(1 + 2 * 4 * 5003, device="cuda")
    P = buf[1:].view(2, 4, 5003)
    Q = torch.rand(2, 3, 5003, device="cuda")
    y = torch.randint(0, 5003, (2, 3), device="cuda", dtype=torch.int32)
    u = torch.rand(2, 4, device="cuda")
    _check(gpu_lib, P, Q, y, u)
    out = tuple(torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(3))
    ws = torch.empty(gpu_lib.verify_probs_workspace_bytes(2, 3, 5003), dtype=torch.uint8,
                     device="cuda")
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        gpu_lib.verify_probs(P, Q, y, u, out=out, workspace=ws, stream=s)
    for _ in range(3):
        u.copy_(torch.rand(2, 4, device="cuda"))
        graph.replay()
        acc, tok = _check(gpu_lib, P, Q, y, u)
        assert torch.equal(acc, out[0]) and torch.equal(tok, out[1])
