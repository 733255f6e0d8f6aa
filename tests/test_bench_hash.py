"""bench.py prints a kernel's measured DRAM traffic for the sources it was measured on:
their hash follows the benchmark's kernels, not the other operators'."""
import os
import re
import shutil

import bench

CSRC = os.path.join("paper_2602_05774_gb300", "csrc")


def _tree(tmp_path, monkeypatch):
    shutil.copytree(os.path.join(bench.ROOT, CSRC), tmp_path / CSRC)
    shutil.copytree(os.path.join(bench.ROOT, "include"), tmp_path / "include")
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path / CSRC


def _append(path, text):
    with open(path, "a") as f:
        f.write(text)


def test_hash_follows_the_benchmarks_kernels(tmp_path, monkeypatch):
    csrc = _tree(tmp_path, monkeypatch)
    before = bench.kernel_source_hash()
    for f in ("vsd_lmloss.cu", "vsd_topk.cu", "vsd_rowloss.cuh", "vsd_target.cuh", "vsd_pair.cuh",
              "vsd_loss.h"):
        _append(csrc / f, "int another_line;\n")
    assert bench.kernel_source_hash() == before
    for f in ("vsd_kernels_bf16.cu", "vsd_passes.cuh", "vsd_lmhead_bwd.cu", "vsd_tc.cuh",
              "vsd_api.cu"):
        _append(csrc / f, "// a comment\n")
        assert bench.kernel_source_hash() == before
        _append(csrc / f, "int another_line;\n")
        now = bench.kernel_source_hash()
        assert now != before, f
        before = now


def test_sources_left_out_are_the_losses_alone():
    """No kernel of the benchmark is compiled from them (the entry points see their
    launchers' declarations)."""
    csrc = os.path.join(bench.ROOT, CSRC)
    for f in os.listdir(csrc):
        if f in bench.LOSS_SOURCES or f == "vsd_api.cu":
            continue
        with open(os.path.join(csrc, f)) as src:
            named = re.findall(r'#include "([^"]+)"', src.read())
        assert not set(named) & set(bench.LOSS_SOURCES), f
