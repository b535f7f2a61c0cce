"""Limits that the binding states are those of the header."""
import os
import re

from paper_2507_19131_b200 import binding as mq

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mixaq.h")


def test_the_widest_row_of_a_norm():
    assert int(re.search(r"#define MIXAQ_NORM_MAX_DIM (\d+)", open(HEADER).read())[1]) == mq.NORM_MAX_DIM
