"""The sources that the benchmark's traffic measurement is tied to: those of the kernels that it launches, not the 4-bit operators'."""
import os
import shutil

import bench

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_hash_covers_the_benchmarks_kernels_alone(tmp_path, monkeypatch):
    for part in (os.path.join("paper_2512_22804_amd", "csrc"), "include"):
        shutil.copytree(os.path.join(ROOT, part), tmp_path / part)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    csrc = tmp_path / "paper_2512_22804_amd" / "csrc"
    before = bench.csrc_sha256()
    (csrc / "mx_product.hip").write_text("// another one\n")
    (csrc / "mx_new.h").write_text("// and one more\n")
    assert bench.csrc_sha256() == before
    with open(csrc / "mor_device.h", "a") as f:
        f.write("// a change\n")
    changed = bench.csrc_sha256()
    assert changed != before
    with open(tmp_path / "include" / "mor.h", "a") as f:
        f.write("// a change\n")
    assert bench.csrc_sha256() != changed
