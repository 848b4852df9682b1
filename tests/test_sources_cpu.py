"""What no run shows, read from the sources of the 4-bit layers and of the log probabilities."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_19509_b200", "csrc")
FILES = ["cluster.cuh", "conv_mxfp4.cu", "conv_mxfp4_pair.cu", "logprobs.cu", "mxfp4.cu", "mxfp4.cuh", "mxfp4_mma.cuh"]
# Barriers that all lanes of a warp have to execute together (bar.sync and bar.red are short for their aligned forms).
ALIGNED = re.compile(r"\b(barrier\.cluster\.(arrive|wait)[\w.]*\.aligned|bar\.(sync|red|arrive))\b")


@pytest.mark.parametrize("name", FILES)
def test_lanes_meet_before_aligned_barriers(name):
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    code = re.sub(r"//[^\n]*", lambda m: " " * len(m.group()), text)
    for hit in ALIGNED.finditer(code):
        body = code[code.rfind("\n__device__", 0, hit.start()):hit.start()]
        assert "__syncwarp();" in body, f"{name}: {hit.group()} in a function that does not bring the lanes together"
