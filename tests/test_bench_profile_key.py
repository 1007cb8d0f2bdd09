"""The bench's DRAM traffic figure belongs to the kernel sources that were
captured: the key covers all of their device code, and the profile names it."""
import os
import re
import shutil

import pytest

import bench

CSRC = os.path.join("paper_2512_21857_gb300", "csrc")
SOURCES = ("tree_attn.cu", "tree_attn_wide.cuh", "sm100.cuh", "adt_common.cuh")


@pytest.fixture
def copy(tmp_path, monkeypatch):
    os.makedirs(tmp_path / CSRC)
    for name in SOURCES:
        shutil.copy(os.path.join(bench.ROOT, CSRC, name), tmp_path / CSRC / name)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path / CSRC


def test_the_key_covers_every_source_of_the_attention_kernels(copy):
    first = bench.attn_source_sha()
    for name in SOURCES:
        text = (copy / name).read_text()
        assert set(re.findall(r'#include "(\w+\.cuh)"', text)) <= set(SOURCES)
        (copy / name).write_text("// changed\n" + text)
        assert bench.attn_source_sha() != first, name
        (copy / name).write_text(text)
    (copy / "tree_attn.cu").write_text((copy / "tree_attn.cu").read_text() + "// host code changed\n")
    assert bench.attn_source_sha() == first


def test_the_figure_is_one_that_was_captured():
    with open(os.path.join(bench.ROOT, "profiles", "tree_attn_tc_kernel_128_7b_layer.md")) as f:
        profile = f.read()
    for key, traffic in bench.NCU_TRAFFIC.items():
        assert f"SHA-256 prefix {key}" in profile
        read, write = (int(re.search(rf"dram__bytes_{x}\.sum \| ([\d,]+) B", profile)[1].replace(",", "")) for x in ("read", "write"))
        assert read + write == traffic
