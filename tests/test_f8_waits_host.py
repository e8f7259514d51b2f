"""Waits of the 8-bit floating-point linear layers, as far as their source shows them."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1806_08342_b200", "csrc")


def test_the_last_waits_do_not_end_with_an_earlier_one():
    """What a CTA has under way when it ends is waited for even where another wait has run out: by the wait itself, not by the form that
    polls once from then on."""
    found = 0
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            calls = re.findall(r"(mbar_wait\w*)\((?:[^;]*?)kDrainBudget", f.read())
        found += len(calls)
        assert set(calls) <= {"mbar_wait"}, (name, calls)
    assert found >= 8
