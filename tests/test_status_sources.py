"""How kernels record errors, whatever the tests on a GPU happen to see."""
import os
import re

from tests.test_body_sources import CSRC, _code


def test_errors_are_recorded_past_a_note():
    """Every code but -10 (entries were ignored, the results stand) goes through the one function that lets it take -10's place."""
    seen = 0
    for name in sorted(os.listdir(CSRC)):
        for call in re.findall(r"atomicCAS\(([^;]*?),\s*(?:0|-10),\s*([^;)]*)\)", _code(name)):
            seen += 1
            assert call[1].strip() == "-10" or (name == "sm100_prims.cuh" and call[1].strip() == "code"), (name, call)
    assert seen >= 4
