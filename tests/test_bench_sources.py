"""Which sources a stored counter figure of the gather is of (bench.py)."""
import os
import shutil

import pytest

import bench

CSRC = os.path.join("paper_2110_08450_amd", "csrc")


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A copy of the library's sources that bench.py looks at instead."""
    shutil.copytree(os.path.join(bench.ROOT, CSRC), tmp_path / CSRC)
    shutil.copytree(os.path.join(bench.ROOT, "include"), tmp_path / "include")
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path


def append(path, text):
    with open(path, "a", encoding="utf-8") as f:
        f.write(text)


@pytest.mark.parametrize("name", ["train.hip", "kernels_embed.h", "kernels_norm.h", "kernels_clip.h", "elements.h"])
def test_training_operators_leave_the_gathers_figure(tree, name):
    was = bench.source_hash()
    append(tree / CSRC / name, "\nint another;\n")
    assert bench.source_hash() == was


@pytest.mark.parametrize("name", ["csrc/smfg.hip", "csrc/kernels_gather.h", "csrc/device_common.h", "csrc/host_common.h", "include/smfg.h"])
def test_code_of_the_library_changes_it_and_comments_do_not(tree, name):
    path = tree / "include" / "smfg.h" if name.startswith("include") else tree / CSRC / os.path.basename(name)
    was = bench.source_hash()
    append(path, "\n// a comment\n/* another */\n")
    assert bench.source_hash() == was
    append(path, "\nint another;\n")
    assert bench.source_hash() != was
