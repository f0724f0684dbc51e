"""What the header says of the table of gaps is what the kernels hold."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_last_bound_of_a_table():
    gap = open(os.path.join(ROOT, "paper_1108_2580_amd", "csrc", "gap.h")).read()
    header = open(os.path.join(ROOT, "include", "als.h")).read()
    gaps = int(re.search(r"constexpr int kTableGaps = (\d+);", gap).group(1))
    assert int(re.search(r"\(Up to (\d+) a table in LDS", header).group(1)) == gaps - 1
