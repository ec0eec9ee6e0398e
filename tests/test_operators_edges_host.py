"""Host side of the learner-side operators where it meets more than one device or stream; nothing here needs a GPU."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2104_11125_b200", "csrc")


def _code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def test_nothing_of_a_device_is_kept_for_the_process():
    """What a call asks of the runtime (attributes it sets, blocks that fit) holds for the device it was asked on. A variable of static
    storage that is initialised by such a call would hand the first device's answer to a handle on another."""
    for name in ("operators.cu", "layer_norm.cuh", "ns_small.cuh", "ffn_tokens.cuh", "tc_product.cuh", "operand_prep.cuh", "ops_common.cuh"):
        for line in re.findall(r"\bstatic\b[^;{]*=[^;]*;", _code(name)):
            assert not re.search(r"\bcuda[A-Z]\w*\s*\(|\bresident\s*\(|\bo->", line), "%s: %s" % (name, line.strip())
    # and the limit that the layer norm's backward pass needs is raised where a handle is made
    create = _code("operators.cu").split("int scalecom_ops_create(")[1].split("void scalecom_ops_destroy(")[0]
    for kind in ("float", "__half", "__nv_bfloat16"):
        assert "ln_attributes<%s>()" % kind in create
