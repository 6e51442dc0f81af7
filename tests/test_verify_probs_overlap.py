"""ldr_verify_probs refuses outputs over its inputs or over one another, on the host. The
addresses are never used: each call is refused before a launch."""
import ctypes

import pytest

BATCH, B, V = 3, 4, 64


@pytest.fixture(scope="module")
def L():
    from paper_2609_37029_amd import ldr
    return ldr


def _regions(L):
    """name -> (address, bytes), a gap of one word between them."""
    ws = L.lib().ldr_verify_probs_workspace_bytes(BATCH, B, V)
    at, r = 1 << 20, {}
    for name, n in (("target", BATCH * (B + 1) * V * 4), ("draft", BATCH * B * V * 4),
                    ("tokens", BATCH * B * 4), ("n_draft", BATCH * 4), ("u", BATCH * (B + 1) * 4),
                    ("accepted", BATCH * 4), ("next", BATCH * 4), ("n_new", BATCH * 4), ("ws", ws)):
        r[name] = (at, n)
        at += (n + 4 + 255) // 256 * 256
    return r


OUT = ("accepted", "next", "n_new", "ws")
IN = ("target", "draft", "tokens", "n_draft", "u")


@pytest.mark.parametrize("out,other", [(o, x) for o in OUT for x in IN + OUT if x != o])
@pytest.mark.parametrize("where", ["same", "last"])
def test_overlaps_are_refused(L, out, other, where):
    r = _regions(L)
    # at the other's start, or on its last word (of its last 16 bytes for the workspace)
    step = 16 if out == "ws" else 4
    at = r[other][0] + (0 if where == "same" else (r[other][1] - 1) // step * step)
    r[out] = (at, r[out][1])
    p = {k: ctypes.c_void_p(v[0]) for k, v in r.items()}
    assert L.lib().ldr_verify_probs(p["target"], p["draft"], p["tokens"], p["n_draft"], p["u"], BATCH,
                                    B, V, p["accepted"], p["next"], p["n_new"], p["ws"], r["ws"][1],
                                    None) == L.LDR_EINVAL
