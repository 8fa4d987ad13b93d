"""The stored traffic of the two dominant kernels belongs to the sources that hold them: the record names these files."""
import json
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2412_14590_amd", "csrc")


@pytest.mark.parametrize("key,kernel", [("decode_m1_gate_up", "linear_decode_split_kernel"), ("prefill_m2048_gate_up", "linear_prefill_kernel")])
def test_the_record_names_the_kernels_sources(key, kernel):
    sources = json.load(open(os.path.join(ROOT, "profiles", "hbm_traffic.json")))[key]["sources"]
    text = {n: open(os.path.join(CSRC, n)).read() for n in sources}
    assert any(re.search(r"__global__[^;{]*\b" + kernel + r"\(", t) for t in text.values())
    # ... and what those include, but for the epilogue, which the plain kernels have none of
    included = {n for t in text.values() for n in re.findall(r'#include "([^"]+)"', t)}
    assert included - set(sources) <= {"epilogue.h", "mixllm.h"}
