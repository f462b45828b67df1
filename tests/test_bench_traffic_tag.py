"""Which source changes make bench.py forget the DRAM counters on file."""
import os
import shutil

import bench


def test_the_tag_follows_the_sources_of_the_timed_kernels(tmp_path, monkeypatch):
    csrc = tmp_path / "csrc"
    shutil.copytree(os.path.join(bench.ROOT, "paper_2603_06626_b200", "csrc"), csrc)
    tag = bench.kernel_source_tag()
    monkeypatch.setattr(bench, "CSRC", str(csrc))
    assert bench.kernel_source_tag() == tag

    def with_line(name, line):
        path = csrc / name
        before = path.read_text() if path.exists() else None
        path.write_text((before or "") + line)
        changed = bench.kernel_source_tag()
        path.write_text(before) if before is not None else path.unlink()
        return changed

    for other in ("norm.cu", "adamw.cu", "balance.cu", "new_operator.cu"):      # kernels that the layer's step does not launch
        assert with_line(other, "int another;\n") == tag, other
    for used in ("plan.cu", "permute.cu", "gemm.cu", "api.cu", "ptx.cuh", "common.cuh", "vec.cuh"):      # those of the step, and what they include
        assert with_line(used, "int another;\n") != tag, used
        assert with_line(used, "// a comment\n\n") == tag, used
