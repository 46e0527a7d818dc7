"""The example runs the operators together as a server would: chunks, then captured steps."""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


# A rounded code is off by up to half a step: a step is 1/127 of a page's largest value (int8; about 1/29 of a standard
# deviation of normal rows, so an error of 0.01 of it) or 2^-3 of the value itself (e4m3: 0.036 of it on average over a binade).
# The weights' errors are of the same size; the output, an average of about as many values as weights count, keeps both.
# Twice the sum of the two is allowed.
@pytest.mark.parametrize("code,dtype,allowed", [("int8", "bf16", 0.05), ("int8", "fp16", 0.05), ("e4m3", "bf16", 0.15)])
def test_serving_loop(code, dtype, allowed):
    import block_cache
    assert block_cache.main(["--code", code, "--dtype", dtype, "--prompts", "2500", "300", "17", "--steps", "20"]) < allowed
