"""The paged kernels start beside the end of the kernel in front of them, which writes what they read: no load of theirs may count on data that nobody writes."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_03383_b200", "csrc")


@pytest.mark.parametrize("name", ["paged.cu", "attention_paged.cu", "attention_paged_fp8.cu", "paged_attn.cuh", "paged_common.cuh", "fp8.cuh"])
def test_no_load_as_of_constants(name):
    code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    assert "__ldg" not in code and ".nc" not in code and "__restrict__" not in code
