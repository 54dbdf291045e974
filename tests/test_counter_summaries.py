"""The counter summaries that bench.py quotes hold while the sources they were
taken on stand: the backward's kernels and the attention's part of the host
sources.  An operator added behind that part does not lose them."""
import os
import shutil

import pytest

import bench

CSRC = os.path.join("paper_2606_01143_amd", "csrc")


@pytest.fixture
def tree(tmp_path, monkeypatch):
    os.makedirs(tmp_path / CSRC)
    for f in bench.BWD_SOURCES:
        shutil.copy(os.path.join(bench.ROOT, CSRC, f), tmp_path / CSRC / f)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path / CSRC


def _edit(path, old, new):
    text = path.read_text()
    assert text.count(old) == 1, (path, old)
    path.write_text(text.replace(old, new))


def test_other_operators_do_not_lose_the_counters(tree):
    before = bench.bwd_source_hash()
    for f, end in bench.ATTENTION_ENDS.items():
        _edit(tree / f, end, end + "hipError_t launch_something_else();\n")
    _edit(tree / "spr_api.hip", '#include "../../include/spr_layer.h"\n',
          '#include "../../include/spr_layer.h"\n#include "../../include/spr_other.h"\n')
    assert bench.bwd_source_hash() == before


@pytest.mark.parametrize("f", bench.BWD_SOURCES)
def test_the_attentions_sources_do(tree, f):
    before = bench.bwd_source_hash()
    text = (tree / f).read_text()
    (tree / f).write_text("constexpr int kOther = 1;\n" + text)
    assert bench.bwd_source_hash() != before
    end = bench.ATTENTION_ENDS.get(f)
    if end:  # up to its end, and without one the whole file
        (tree / f).write_text(text.replace(end, "constexpr int kOther = 1;\n" + end))
        assert bench.bwd_source_hash() != before
        (tree / f).write_text(text.replace(end, ""))
        assert bench.bwd_source_hash() != before


def test_a_summary_of_these_sources_is_read(tree):
    os.makedirs(tree.parent.parent / "profiles")
    with open(bench.traffic_summary("w"), "w") as f:
        f.write("- HBM bytes per launch (calibrated): `1.5e+09`\n- kernel source hash: `%s` (sha256)\n" % bench.bwd_source_hash())
    assert bench.committed_traffic("w")[0] == 1.5e9
    (tree / "tile.hpp").write_text("// other\n")
    assert bench.committed_traffic("w") == (None, "kernel changed since the counters were taken")
