"""The checksum that ties the committed counter summaries to the sources: it covers what the networks run, and nothing that they do not."""
import os
import shutil
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import bench  # noqa: E402
from paper_2108_09413_amd import profile_report  # noqa: E402

CSRC = os.path.join("paper_2108_09413_amd", "csrc")


@pytest.fixture
def tree(tmp_path, monkeypatch):
    os.makedirs(tmp_path / CSRC)
    for name in os.listdir(os.path.join(ROOT, CSRC)):
        if name.endswith((".hip", ".h", ".cpp")):
            shutil.copy(os.path.join(ROOT, CSRC, name), tmp_path / CSRC / name)
    monkeypatch.setattr(profile_report, "ROOT", str(tmp_path))
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path / CSRC


@pytest.mark.parametrize("name", ["distill.hip", "logprobs.hip", "logit_device.h", "logit_rows.h", "logit_api.cpp"])
def test_operators_on_rows_of_logits_are_no_part_of_the_networks(tree, name):
    before = bench.kernel_sources_sha256()
    assert before == profile_report.sources_sha256()
    with open(tree / name, "a") as f:
        f.write("// more\n")
    assert bench.kernel_sources_sha256() == profile_report.sources_sha256() == before


@pytest.mark.parametrize("name", ["conv_igemm.hip", "conv_device.h", "kernels.hip", "plan.cpp", "isr_internal.h", "a_new_kernel.hip"])
def test_all_other_sources_are(tree, name):
    before = bench.kernel_sources_sha256()
    with open(tree / name, "a") as f:
        f.write("// more\n")
    assert bench.kernel_sources_sha256() == profile_report.sources_sha256() != before


def test_no_other_source_uses_the_operators(tree):
    """So leaving them out leaves out nothing of the networks."""
    for name in os.listdir(tree):
        if name not in profile_report.ROW_OPERATOR_SOURCES:
            text = open(tree / name).read()
            assert "logit_rows.h" not in text and "logit_device.h" not in text, name
