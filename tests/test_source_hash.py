"""The digest that ties a stored capture to the kernels it was taken of."""
import os
import shutil

from paper_2607_12789_b200 import build


def test_it_follows_the_forward_s_sources_and_their_headers_alone(tmp_path, monkeypatch):
    csrc = tmp_path / "csrc"
    shutil.copytree(build.CSRC, csrc)
    before = build.source_hash()
    monkeypatch.setattr(build, "CSRC", str(csrc))
    assert build.source_hash() == before
    for name in ("avq_cache.cu", "avq_exact.cuh", "avq_tc_cached.cu", "avq_update.cu"):   # other kernels
        assert os.path.exists(csrc / name)
        (csrc / name).write_text((csrc / name).read_text() + "// more\n")
        assert build.source_hash() == before
    seen = {before}
    for name in ("avq_tc_attend.cu", "avq_tc_aggregate.cu", "avq_tc_assign.cu", "avq_tc_common.cuh", "avq_internal.h"):
        (csrc / name).write_text((csrc / name).read_text() + "// more\n")
        seen.add(build.source_hash())
    assert len(seen) == 6
