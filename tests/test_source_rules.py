"""Rules that the device code keeps by its text, checked without a GPU."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_09905_amd", "csrc")


def _sources():
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        if path.endswith((".hip", ".h", ".cpp")):
            with open(path) as f:
                yield os.path.basename(path), f.read()


def test_loads_to_lds_wait_for_m0():
    # the hardware wants one wait state between an instruction that writes M0
    # and a load to LDS, which takes its address from there; the compiler puts
    # it between instructions of its own, not into inline assembly
    writes = 0
    for name, text in _sources():
        for m in re.finditer(r"s_\w+ m0,[^\"]*?\\n\\t(\w+)( \d+)?", text):
            writes += 1
            assert m.group(1) == "s_nop", (name, m.group(0))
        # none whose next instruction is out of this test's sight
        assert len(re.findall(r"s_\w+ m0,", text)) == len(re.findall(r"s_\w+ m0,[^\"]*?\\n\\ts_nop 0", text)), name
    assert writes > 0
