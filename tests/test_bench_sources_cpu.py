"""bench.py takes measured HBM traffic from counters that were recorded on the sweeps' present sources: those of
the sequence operators are no part of them."""
import os
import re

import bench


def includes(name):
    return set(re.findall(r'^#include "(\w+\.h)"', open(os.path.join(bench.CSRC, name)).read(), re.M))


def test_sources_of_the_sequence_operators_are_no_part_of_the_sweeps():
    sources = {n for n in os.listdir(bench.CSRC) if n.endswith((".hip", ".h"))}
    headers = {"sequence.h"}  # and those that include it
    while more := {n for n in sources - headers if n.endswith(".h") and includes(n) & headers}:
        headers |= more
    operators = headers | {n for n in sources if includes(n) & headers}
    operators.discard("api.hip")  # the library's last error, for both
    assert bench.OTHER_SOURCES == operators


def test_the_default_workloads_counters_are_of_the_present_sources():
    assert bench.measured_traffic("full_1000990x624961_d20", "k_gram_ne")
