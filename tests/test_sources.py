"""Every source of the library is one that its build compiles."""
import os

from paper_2512_22560_amd import build


def test_no_source_lies_beside_the_build():
    compiled = {s.partition(":")[0] for s in build.SOURCES} | {"bench_peaks.hip", "host_calls.cpp"}
    assert {f for f in os.listdir(build.CSRC) if f.endswith((".hip", ".cpp"))} == compiled
