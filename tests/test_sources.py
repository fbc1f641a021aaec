"""What the device sources must not hold.  The library is built once and runs
as one replica a GPU (bench.py --gpus N), over pointers that the caller gives,
so no copy in it may be one that is only sound within a single GPU's own
memory."""
import glob
import os

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_28870_gb300", "csrc")


def test_no_copy_writes_to_several_ctas():
    files = [f for f in glob.glob(os.path.join(CSRC, "*")) if os.path.isfile(f)]
    assert files
    for f in files:
        for i, line in enumerate(open(f), 1):
            assert "multicast" not in line, f"{os.path.basename(f)}:{i}: {line.strip()}"
