"""What a traffic record depends on: the sources that define its kernels and the flags that
they are built with, and nothing else."""
import os
import re

import pytest

from paper_2606_00746_amd import build, profiling

CSRC = os.path.join(os.path.dirname(profiling.__file__), "csrc")


def kernels():
    """(file, name) of every kernel."""
    for f in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, f)).read()
        for m in re.finditer(r"__global__[^;{]*?\bvoid\s+(?:__launch_bounds__\([^)]*\)\s+)?(\w+)\s*\(", text, re.S):
            yield f, m.group(1)


def test_kernels_are_found():
    assert len(list(kernels())) > 60
    assert ("scan_line.hip", "grad_kernel") in kernels() and ("scan_pm.hip", "fwd_pm_kernel") in kernels()


@pytest.mark.parametrize("file,name", sorted(set(kernels())))
def test_a_kernel_depends_on_the_file_that_defines_it(file, name):
    for full in (name, name + "<unsigned short, 4, true>"):
        assert file in [os.path.basename(f) for f in profiling.source_files([full])]


@pytest.mark.parametrize("file,name", sorted((f, n) for f, n in set(kernels()) if not f.startswith("scan_")))
def test_the_scans_calls_have_none_of_the_other_operators_kernels(file, name):
    assert profiling.call_of(f"void gspn::(anonymous namespace)::{name}<unsigned short>(int)") is None


def test_a_source_more_leaves_other_kernels_records_as_they_are(monkeypatch):
    names = ["bwd_med_kernel<64, 64>", "to_blocked_kernel<64>"]
    before = profiling.source_hash(names)
    monkeypatch.setattr(build, "SOURCES", build.SOURCES + ["another.hip"])
    monkeypatch.setitem(build.SOURCE_FLAGS, "another.hip", ["-mllvm", "-x"])
    assert profiling.source_hash(names) == before
    assert "build.py" not in [os.path.basename(f) for f in profiling.source_files(names)]


def test_other_flags_make_another_record(monkeypatch):
    names = ["bwd_med_kernel<64, 64>"]
    before = profiling.source_hash(names)
    monkeypatch.setattr(build, "HIPCC_FLAGS", build.HIPCC_FLAGS + ["-ffast-math"])
    assert profiling.source_hash(names) != before
    monkeypatch.undo()
    assert profiling.source_hash(names) == before
    monkeypatch.setitem(build.SOURCE_FLAGS, "scan_med_64.hip", ["-mllvm", "-x"])
    assert profiling.source_hash(names) != before


def test_the_hash_does_not_depend_on_where_the_tree_lies(monkeypatch):
    names = ["bwd_med_kernel<64, 64>"]
    before = profiling.source_hash(names)
    monkeypatch.setattr(build, "HIPCC_FLAGS", ["/elsewhere/include" if os.path.isabs(f) else f for f in build.HIPCC_FLAGS])
    assert profiling.source_hash(names) == before
