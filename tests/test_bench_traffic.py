"""bench.py's record of the score kernel's HBM traffic belongs to the sources of the compression step: it holds while those are what it was measured on, whatever the serving operators' sources are."""
import argparse
import os
import shutil

import bench

PLAIN = argparse.Namespace(resident=False, post_rope=False, half_split=False, variant=0, seqs=0, layers=0)


def with_sources(monkeypatch, tmp_path, change):
    csrc = tmp_path / "paper_2604_04921_amd" / "csrc"
    shutil.copytree(os.path.join(bench.ROOT, "paper_2604_04921_amd", "csrc"), csrc)
    with open(csrc / change, "a") as f:
        f.write("// more\n")
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return bench.kernel_sources_sha16()


def test_other_sources(monkeypatch, tmp_path):
    here = bench.kernel_sources_sha16()
    assert with_sources(monkeypatch, tmp_path / "a", "tri_attend.hip") == here
    monkeypatch.undo()
    assert with_sources(monkeypatch, tmp_path / "b", "tri_score_lane.hip") != here
    monkeypatch.undo()
    assert with_sources(monkeypatch, tmp_path / "c", "tri_internal.h") != here


def test_the_record_holds():
    """(A change to the compression's sources wants the counters read again, or this record taken out.)"""
    assert bench.measured_traffic("c3_model", "dense", PLAIN) == bench.MEASURED_TRAFFIC["c3_model/dense"]["bytes"]
