"""ldr_pages_read refuses outputs over each other, over its inputs, and over the cache it
reads from, on the host. The library's host side is linked with launches that do nothing
(tests/host/pages_stub.cpp); the addresses are never used."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2609_37029_amd import build as B

HOST = os.path.join(os.path.dirname(os.path.abspath(__file__)), "host")
LAYERS, HKV, D, PAGE, N_PAGES, BATCH, MAX_PAGES, ROWS = 2, 2, 64, 32, 5, 3, 4, 7
LAYER, N_LAYERS = 1, 1
EINVAL = -1


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("hipcc is required to build the library's host side")
    out = str(tmp_path_factory.mktemp("stub") / "libpages_host.so")
    r = subprocess.run([B.hipcc()] + B.flags() + ["-I", B.CSRC, "-shared", "-x", "hip",
                        os.path.join(B.CSRC, "api_pages.cpp"), os.path.join(HOST, "pages_stub.cpp"),
                        "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    L = ctypes.CDLL(out)
    L.ldr_pages_pool_bytes.restype = L.ldr_pages_state_bytes.restype = ctypes.c_size_t
    return L


class Rig:
    """A handle, and the regions of one read: name -> (address, bytes), gaps between them."""

    def __init__(self, L, dtype):
        self.L, self.h = L, ctypes.c_void_p()
        cfg = (ctypes.c_int32 * 8)(LAYERS, HKV, D, PAGE, N_PAGES, BATCH, MAX_PAGES, dtype)
        rows = BATCH * ROWS * N_LAYERS * HKV * D * (4 if dtype == 0 else 2)
        at, self.r = 1 << 20, {}
        for name, n in (("pool", L.ldr_pages_pool_bytes(cfg)), ("state", L.ldr_pages_state_bytes(cfg)),
                        ("first", 4 * BATCH), ("n", 4 * BATCH), ("K", rows), ("V", rows)):
            self.r[name] = (at, n)
            at += (n + 16 + 255) // 256 * 256
        assert L.ldr_pages_init(ctypes.byref(self.h), cfg, ctypes.c_void_p(self.r["pool"][0]),
                                ctypes.c_void_p(self.r["state"][0]), None) == 0

    def read(self, **moved):
        p = {k: ctypes.c_void_p(moved.get(k, v[0])) for k, v in self.r.items()}
        return self.L.ldr_pages_read(self.h, LAYER, N_LAYERS, p["first"], p["n"], p["K"], p["V"],
                                     ROWS, None)

    def close(self):
        self.L.ldr_pages_destroy(self.h)


@pytest.fixture(params=[0, 1, 4, 8], ids=["f32", "bf16", "mxfp4", "mxfp8"])
def rig(lib, request):
    r = Rig(lib, request.param)
    yield r
    r.close()


def test_regions_apart_are_read(rig):
    assert rig.read() == 0
    # next to each other, without a gap
    at, n = 1 << 30, rig.r["K"][1]
    assert rig.read(K=at, V=at + n) == 0 and rig.read(K=at, V=at - n) == 0
    # the counts may be words of the state (its rows, its open rows)
    assert rig.read(first=rig.r["state"][0] + 256, n=rig.r["state"][0] + 512) == 0


@pytest.mark.parametrize("out,other", [(o, x) for o in ("K", "V")
                                       for x in ("first", "n", "pool", "state", "K", "V") if x != o])
def test_overlaps_are_refused(rig, out, other):
    """At the other's start, on its last bytes, and with its own last bytes on the other's first."""
    at, n = rig.r[other]
    for to in (at, at + (n - 1) // 16 * 16, at - (rig.r[out][1] - 16)):
        assert rig.read(**{out: to}) == EINVAL, hex(to)
