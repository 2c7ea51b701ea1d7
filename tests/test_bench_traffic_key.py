"""The key of the bench line's DRAM traffic covers the device headers that the
prefill kernel is built from (CPU): an edit of a header's code makes the bench
report null, an edit of its comments does not."""
import os
import shutil
import sys

from test_boundary_cpu import ROOT

CSRC = os.path.join("paper_2608_15171_gb300", "csrc")


def test_key_follows_the_device_headers(tmp_path, monkeypatch):
    sys.path.insert(0, ROOT)
    import bench
    assert bench.PREFILL_TRAFFIC.get(bench._src_hash("attn_prefill.cu")) is not None
    (tmp_path / "paper_2608_15171_gb300").mkdir()
    shutil.copytree(os.path.join(ROOT, CSRC), tmp_path / CSRC)
    real = bench._src_hash("attn_prefill.cu")
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench._src_hash("attn_prefill.cu") == real
    for header, code, other in (("ppas_device.cuh", "fma.rn.f32x2", "fma.rz.f32x2"),
                                ("attn_decode_body.cuh", "kDecodeStages", "kOtherStages")):
        path = tmp_path / CSRC / header
        text = path.read_text(encoding="utf-8")
        assert code in text
        path.write_text(text.replace(code, other, 1), encoding="utf-8")
        assert bench._src_hash("attn_prefill.cu") != real, header
        path.write_text("// a remark\n" + text, encoding="utf-8")
        assert bench._src_hash("attn_prefill.cu") == real, header
        path.write_text(text, encoding="utf-8")
