"""What a workgroup tells the others of its launch must be there before it says
that it is done.  A barrier does not wait for the memory operations of the other
waves, so every wave waits for its own first.  (Read from the source: the loss
depends on timing and cannot be shown by running the kernels.)"""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_09800_amd", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def body(src, name):
    """Source text of the function `name`, up to the brace in column 0 that ends it."""
    at = re.search(r"\b%s\([^;{]*\{" % name, src).start()
    return src[at:src.index("\n}\n", at)]


def test_a_plan_s_errors_are_there_before_its_arrival():
    text = body(source("hbf_kv.hip"), "plan_done")
    assert re.search(r"atomicOr\(&ctl->err, err\);\s*stores_done\(\);\s*__syncthreads\(\);", text)
    assert text.index("stores_done()") < text.index("atomicAdd(&ctl->arrived")


@pytest.mark.parametrize("file", ["hbf_attn.hip", "hbf_moe.hip"])
def test_every_last_of_comes_after_a_wait(file):
    src = source(file)
    calls = [m.start() for m in re.finditer(r"if \(!?last_of\(", src)]
    assert calls
    for at in calls:
        before = src[:at]
        assert before.rfind("stores_done();") > max(before.rfind("hand_over("), before.rfind("__hip_atomic_store("))
