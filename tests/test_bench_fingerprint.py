"""The fingerprint that ties recorded DRAM traffic to the kernels it was measured
on: it follows the sources of the networks' kernels, and those alone."""
import os
import re
import shutil
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_16742_gb300", "csrc")


@pytest.fixture(scope="module")
def bench():
    sys.path.insert(0, ROOT)
    import bench
    return bench


def test_follows_the_networks_kernels_alone(bench, tmp_path):
    shutil.copytree(CSRC, tmp_path / "csrc")
    before = bench.source_fingerprint(str(tmp_path / "csrc"))
    assert before == bench.source_fingerprint()
    for name in sorted(os.listdir(CSRC)):
        path = tmp_path / "csrc" / name
        text = path.read_text()
        path.write_text(text + "// changed\n")
        assert (bench.source_fingerprint(str(tmp_path / "csrc")) == before) == (name in bench.OPERATOR_SOURCES), name
        path.write_text(text)
    (tmp_path / "csrc" / "new_layer.cu").write_text("// a new kernel\n")
    assert bench.source_fingerprint(str(tmp_path / "csrc")) != before


def test_operator_sources_are_apart(bench):
    """The sources left out exist, and the networks' sources include none of them."""
    for name in bench.OPERATOR_SOURCES:
        assert os.path.exists(os.path.join(CSRC, name))
    for name in sorted(os.listdir(CSRC)):
        if name not in bench.OPERATOR_SOURCES:
            text = open(os.path.join(CSRC, name)).read()
            assert not set(re.findall(r'#include "([^"]+)"', text)) & set(bench.OPERATOR_SOURCES), name
