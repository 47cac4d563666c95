"""The digest by which bench.py knows whether recorded HBM bytes are of the present kernel."""
import os
import shutil

import pytest

import bench


@pytest.fixture
def tree(tmp_path, monkeypatch):
    for p in bench.KERNEL_SOURCES:
        os.makedirs(os.path.dirname(tmp_path / p), exist_ok=True)
        shutil.copy(os.path.join(bench.ROOT, p), tmp_path / p)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path


def _edit(tree, name, old, new):
    path = tree / next(p for p in bench.KERNEL_SOURCES if p.endswith(name))
    text = path.read_text()
    assert old in text
    path.write_text(text.replace(old, new, 1))


def test_other_files_of_the_library_are_not_the_kernel(tree):
    before = bench.kernel_source_digest()
    _edit(tree, "hipbuild.py", 'SOURCES = ["api.hip", ', 'SOURCES = ["api.hip", "another.hip",\n           ')
    _edit(tree, "topk.hip", "#include", "// a comment\n#include")
    assert bench.kernel_source_digest() == before


@pytest.mark.parametrize("name,old,new", [("hipbuild.py", '"-O3"', '"-O2"'), ("topk_kernel.h", "return", "return  (0),"),
                                          ("schedule.h", "return", "return  (0),"), ("topk.hip", "return", "return  (0),"),
                                          ("common.h", "return", "return  (0),"), ("hipbuild.py", "-shared", "-static")])
def test_its_code_and_flags_are(tree, name, old, new):
    before = bench.kernel_source_digest()
    _edit(tree, name, old, new)
    assert bench.kernel_source_digest() != before


def test_bytes_of_another_kernel_are_not_reported(tree):
    os.makedirs(tree / "profiles")
    line = "traffic: workload=w kernel=k_topk source_sha256={} bytes_per_launch=5\n"
    (tree / "profiles" / "w.md").write_text(line.format(bench.kernel_source_digest()))
    assert bench.recorded_traffic("w") == (5.0, os.path.join("profiles", "w.md"))
    assert bench.recorded_traffic("v") == (None, None)
    _edit(tree, "topk.hip", "return", "return  (0),")
    assert bench.recorded_traffic("w") == (None, None)
