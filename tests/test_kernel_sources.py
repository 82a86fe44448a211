"""What the kernels' sources must not hold, looked up in their text."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_23635_gb300", "csrc")


def instructions(text):
    """The instructions of a source's inline PTX (neighbouring string literals joined)."""
    text = re.sub(r'"\s*"', "", text)
    for literal in re.findall(r'"((?:[^"\\\n]|\\.)*)"', text):
        for one in literal.replace("\\n", ";").replace("\\t", " ").split(";"):
            yield one.strip(" {}")


def test_copies_go_to_one_cta():
    """The library serves programs of one GPU and of several from the same sources, on whatever memory a
    caller hands it: each block's bulk copies are for that block alone."""
    files = glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))
    copies = [(os.path.basename(f), i) for f in files for i in instructions(open(f).read())
              if i.startswith("cp.async.bulk")]
    assert len(copies) > 5
    assert not [c for c in copies if "multicast" in c[1]]
