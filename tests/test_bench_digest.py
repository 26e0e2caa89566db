"""The digest that ties a stored traffic record to the kernels it was taken
from covers what the networks run, and nothing else (CPU)."""
import os
import re
import shutil
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import bench  # noqa: E402

CSRC = os.path.join(ROOT, "paper_1511_07376_amd", "csrc")


@pytest.fixture
def copy(tmp_path, monkeypatch):
    at = tmp_path / "paper_1511_07376_amd" / "csrc"
    shutil.copytree(CSRC, at)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return at


def _append(path, text):
    with open(path, "a", encoding="utf-8") as f:
        f.write(text)


@pytest.mark.parametrize("name", ["route.hip", "mx4.hip", "fc_rows.hip", "fc_tiles_kernel.h", "experts.h"])
def test_operators_outside_the_networks_do_not_count(copy, name):
    before = bench.source_digest()
    _append(copy / name, "int another;\n")
    assert bench.source_digest() == before


@pytest.mark.parametrize("name", ["bandwidth.hip", "fc_gemm.hip", "conv_split_kernel.h", "common.h"])
def test_the_networks_kernels_count(copy, name):
    before = bench.source_digest()
    _append(copy / name, "// a comment changes no kernel\n\n")
    assert bench.source_digest() == before
    _append(copy / name, "int another;\n")
    assert bench.source_digest() != before


def test_no_network_source_uses_one_that_is_left_out():
    names = set(os.listdir(CSRC))
    assert set(bench.EXPERT_SOURCES) <= names
    for name in sorted(names - set(bench.EXPERT_SOURCES) - set(bench.HOST_ONLY_SOURCES)):
        with open(os.path.join(CSRC, name), encoding="utf-8") as f:
            used = set(re.findall(r'#include "([^"]+)"', f.read()))
        assert not used & set(bench.EXPERT_SOURCES), (name, used)
