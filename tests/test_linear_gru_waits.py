"""The linear GRU's waits along its chain of tiles, checked in the source (no GPU needed).

A tile of time waits in a loop for the state before it.  A queue can be taken off the device for any
time in the middle of that, so the loop must not be bounded by a clock: on return it would give up,
with NaN, on words that its neighbours are about to write."""
import os
import re

from paper_1810_09958_amd import build as B


def test_waits_do_not_read_a_clock():
    with open(os.path.join(B.CSRC, "linear_gru.hip")) as f:
        source = f.read()
    assert "s_sleep" in source
    assert not re.search(r"clock|s_memtime|s_memrealtime|SHADER_CYCLES", source)
