"""A check takes the error word on the stream that it is given: cudaMemset works on the legacy stream and returns before it has
run, and streams that do not wait for that one (PyTorch's side streams) may set bits before the clearing lands, which are lost.
When that happens cannot be arranged, so the calls are read from the sources."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_03700_gb300", "csrc")


def body(path, name):
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(os.path.join(CSRC, path)).read(), flags=re.S)
    m = re.search(r"\b%s\([^;{]*\)\s*\{" % name, text)
    depth, end = 1, m.end()
    while depth:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
    return text[m.end():end]


@pytest.mark.parametrize("path,name", [("kv_ops.cu", "adept_kv_check"), ("runtime.cu", "adept_check_device_status")])
def test_no_check_uses_the_legacy_stream(path, name):
    calls = body(path, name)
    assert "take_error_word(" in calls
    assert not re.search(r"\bcudaMem(set|cpy)\s*\(", calls)
    cleared = calls.find("cudaMemsetAsync(")   # (counters besides: waited for)
    assert cleared < 0 or calls.find("cudaStreamSynchronize(", cleared) > 0


def test_the_word_is_read_and_cleared_on_the_stream():
    calls = body("kernels_misc.cu", "take_error_word")
    read, wait = calls.index("cudaMemcpyAsync("), calls.index("cudaStreamSynchronize(")
    clear = calls.index("clear_bits_kernel")
    assert read < wait < clear < calls.rindex("cudaStreamSynchronize(")
    assert not re.search(r"\bcudaMem(set|cpy)\s*\(", calls)
    assert re.search(r"atomicAnd\(word, ~bits\)", body("kernels_misc.cu", "clear_bits_kernel"))
