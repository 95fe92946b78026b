"""The digest of the kernel sources that a committed profile names: of what the measured kernels are made of, and of nothing else."""
import os
import shutil

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name,counts", [("svip_kernels.hip", True), ("draft_kernels.h", True), ("wave_ops.h", True), ("exchange.h", True), ("loop_round.h", True),
                                         ("svip_head.hip", False), ("head_kernels.h", False), ("head_tile.h", False), ("svip_loop.hip", False),
                                         ("marshal.cpp", False)])
def test_digest_follows_the_sources_of_the_measured_kernels(tmp_path, monkeypatch, name, counts):
    import bench

    csrc = os.path.join("paper_2411_18462_amd", "csrc")
    shutil.copytree(os.path.join(ROOT, csrc), tmp_path / csrc)
    before = bench.sources_digest()
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.sources_digest() == before
    with open(tmp_path / csrc / name, "a") as f:
        f.write("// changed\n")
    assert (bench.sources_digest() != before) == counts
