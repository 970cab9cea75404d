"""The token operators on devices that place smaller clusters than a GB300 does, or none: DBL_MAX_CLUSTER (read once per
process) as the answer of such a device.  The tests of the sizes that take clusters run again in a process of their own:
wide rows by single blocks that read them again, long sequences part after part, rows of logits from memory."""
import os
import re
import subprocess
import sys

import pytest

from gpu_common import need_gpu

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
WIDE = ["8192", "8208", "9001", "10447", "16000", "16384", "20000", "32768", "33333", "65536", "70001"]  # columns
LONG = ["t1500", "t3001", "t4097", "t5000", "t9000", "t2100"]
LARGE = ["20001", "32000", "45001", "50008", "65537", "131071", "120001", "260000", "700001", "1500007", "90001"]  # classes


@pytest.mark.parametrize("largest", [1, 4])
def test_wide_and_long_sizes_with_smaller_clusters(largest):
    need_gpu()
    files = ["test_gpu_layer_norm.py", "test_gpu_gated_scan.py", "test_gpu_gated_scan_ends.py", "test_gpu_distill.py",
             "test_gpu_distill_clusters.py"]
    cmd = [sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", "-k", " or ".join(WIDE + LONG + LARGE)]
    r = subprocess.run(cmd + [os.path.join(HERE, f) for f in files], capture_output=True, text=True, timeout=900,
                       cwd=os.path.dirname(HERE), env=dict(os.environ, DBL_MAX_CLUSTER=str(largest)))
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert int(re.search(r"(\d+) passed", r.stdout).group(1)) > 200
