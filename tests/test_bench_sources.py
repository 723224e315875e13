"""Which sources a measured traffic figure of the bench is tied to."""
import os
import shutil
import sys

from conftest import ROOT


def test_traffic_is_tied_to_the_decode_steps_sources_and_their_header(tmp_path, monkeypatch):
    sys.path.insert(0, ROOT)
    import bench
    for d in ("include", os.path.join("paper_2504_18583_gb300", "csrc")):
        shutil.copytree(os.path.join(ROOT, d), tmp_path / d)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    csrc, start = tmp_path / "paper_2504_18583_gb300" / "csrc", bench.kernel_source_hash()

    def changed(path):
        kept = path.read_bytes()
        path.write_bytes(kept + b"\n")
        now = bench.kernel_source_hash()
        path.write_bytes(kept)
        return now != start

    # the header that internal.h includes, and with it every kernel file
    assert 'include/pard.h"' in (csrc / "internal.h").read_text() and changed(tmp_path / "include" / "pard.h")
    for name in os.listdir(csrc):
        if name.endswith((".cu", ".cuh", ".h")):
            assert changed(csrc / name) == (name not in bench.TREE_SOURCES), name
