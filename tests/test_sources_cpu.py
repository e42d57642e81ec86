"""What the CUDA sources may not hold, whoever calls them: every rank of a job on several GPUs loads the
one library."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_20438_gb300", "csrc")


def _asm_statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        with open(path) as f:
            text = f.read()
        for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\((.*?)\);", text, re.S):
            yield os.path.basename(path), "".join(re.findall(r'"([^"]*)"', m.group(1)))


def test_no_copy_is_a_cluster_multicast():
    """A bulk or tensor copy writes its own CTA's shared memory alone (the arrival that ends a tensor-core
    product may go to both CTAs of a pair)."""
    copies = [(f, a) for f, a in _asm_statements() if "cp.async.bulk" in a]
    assert len(copies) > 3
    assert not [f for f, a in copies if "multicast" in a]
