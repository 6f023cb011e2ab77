"""Which sources the counter figures on file belong to: those of the step's kernels, no others."""
import os
import shutil

import bench

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_other_calls_sources_do_not_count(tmp_path, monkeypatch):
    for d in (os.path.join("paper_1901_01544_amd", "csrc"), "include"):
        shutil.copytree(os.path.join(ROOT, d), tmp_path / d)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    csrc = tmp_path / "paper_1901_01544_amd" / "csrc"
    want = bench.kernel_source_hash()

    def with_line(path):
        text = path.read_text()
        path.write_text(text + "// a line more\n")
        h = bench.kernel_source_hash()
        path.write_text(text)
        return h

    for name in ("iwp_losses.hip", "iwp_head.hpp", "iwp_matrix.hpp", "iwp_balance.hpp", "call.cpp"):
        assert with_line(csrc / name) == want, name
    (csrc / "iwp_another.hpp").write_text("// of another call\n")
    assert bench.kernel_source_hash() == want
    for path in (csrc / "iwp_api.hip", csrc / "iwp_host.hpp", csrc / "iwp_common.hpp", csrc / "iwp_stream.hpp", csrc / "iwp_sum.hpp",
                 tmp_path / "include" / "iwp.h"):
        assert with_line(path) != want, path.name
    assert bench.kernel_source_hash() == want
