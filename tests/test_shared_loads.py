"""Instructions written by hand that read shared memory which the same kernel also writes in C++ say so to the compiler ("memory"): nothing else keeps it
from moving the one past the other.  Read off the source of the decode steps over rows."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_20787_b200", "csrc")


def test_hand_written_loads_of_the_decode_steps_name_memory():
    text = open(os.path.join(CSRC, "decode_rows_mma.cuh")).read()
    loads = re.findall(r'asm volatile\("ld\.shared[^;]*;"[^;]*;', text)
    assert len(loads) >= 4
    assert [x for x in loads if '"memory"' not in x] == []
