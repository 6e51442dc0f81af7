"""The digest that counted figures are held against: of the drafting step's sources, and of
no others. Figures counted on other kernels of the step are stale; those of a library that
got another operator are not."""
import json
import os
import re
import shutil

import pytest

import bench
from paper_2609_37029_amd import build as B


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A copy of the sources that bench.py takes the digest of."""
    csrc = tmp_path / "paper_2609_37029_amd" / "csrc"
    shutil.copytree(B.CSRC, csrc)
    shutil.copytree(os.path.join(bench.ROOT, "include"), tmp_path / "include")
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return csrc


def _changes(path):
    before = bench.source_digest()
    with open(path, "a") as f:
        f.write("// a line more\n")
    return bench.source_digest() != before


@pytest.mark.parametrize("name", ["attend.hip", "attend_common.h", "attend_mx.hip", "mx.h", "pages.hip",
                                  "pages_mx.hip", "logprobs.hip", "verify_probs.hip", "verify.hip",
                                  "api_pages.cpp", "api_serve.cpp", "serve_internal.h"])
def test_other_operators_are_not_in_it(tree, name):
    assert not _changes(tree / name)


def test_a_new_operator_is_not_in_it(tree):
    before = bench.source_digest()
    (tree / "another.hip").write_text("// kernels of another operator\n")
    assert bench.source_digest() == before
    assert not _changes(tree.parent.parent / "include" / "ldr.h")


@pytest.mark.parametrize("name", ["api.cpp", "views.hip", "gemm.hip", "draft.hip", "attn.hip",
                                  "sample.hip", "ldr_internal.h", "noise.h"])
def test_the_steps_sources_are_in_it(tree, name):
    assert _changes(tree / name)


def test_every_counted_kernel_is_of_these_sources():
    text = "".join(open(os.path.join(B.CSRC, f)).read() for f in bench.step_files(B.CSRC))
    with open(bench.TRAFFIC_JSON) as f:
        symbols = json.load(f)["symbols"]
    names = {re.match(r"\w+", s.strip()).group() for v in symbols.values() for s in v.split("+")}
    assert names
    for n in names:
        assert re.search(r"\b%s\(" % n, text), n
