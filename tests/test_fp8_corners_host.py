"""What of the 8-bit float operators can be checked without a device: sources, decisions of the host, refusals."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2104_04731_b200", "csrc")


def test_results_of_waits_are_voted():
    """The rule of the convolution's kernels (test_bounded_waits): lanes of a warp act on a wait's result together, or some could be at a
    warp-wide instruction, or store a result, without the others."""
    waits = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "fp8_*.cu"))):
        for n, line in enumerate(open(path).read().split("\n")):
            call = re.search(r"\bmbar_wait(_\w+)?\(", line)
            if not call or "__device__" in line or line.lstrip().startswith("//"):
                continue
            waits += 1
            assert line[:call.start()].strip().endswith("__all_sync(0xffffffffu,"), (os.path.basename(path), n + 1, line)
    assert waits >= 10
