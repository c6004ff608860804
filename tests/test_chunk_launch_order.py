"""The chunk attention's tensor-memory kernel lets the next kernel of the stream start only after its allocation (why, and the
check: test_dependent_launch_order.py, which reads the .cu files; this kernel stands in a .cuh)."""
import glob
import os

import test_dependent_launch_order as order


def test_trigger_follows_the_allocation(monkeypatch, tmp_path):
    for path in glob.glob(os.path.join(order.CSRC, "*.cuh")):
        text = open(path).read()
        if "__global__" in text:
            (tmp_path / (os.path.basename(path) + ".cu")).write_text(text)
    monkeypatch.setattr(order, "CSRC", str(tmp_path))
    found = order.kernels()
    assert [p.id for p in found] == ["attention_chunk_tc.cuh.cu:chunk_tc_kernel"]
    order.test_trigger_follows_the_allocation(found[0].values[0])
