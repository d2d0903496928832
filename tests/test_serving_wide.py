"""4-bit products of nearly as many rows of w as there can be, on a host without a device: the call comes to its launches."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2506_17615_amd import binding as eq
from paper_2506_17615_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALL = """
from paper_2506_17615_amd import binding as eq
p = [(i + 1) << 42 for i in range(5)]
print(eq.load().equarx_mx4_product(*p[:4], {M}, {N}, {K}, p[4], {N}, None, 0, None))
"""


@pytest.mark.skipif(torch.cuda.is_available(), reason="its addresses are no memory: nothing may be launched")
@pytest.mark.parametrize("M,N,K", ((100, (1 << 31) - 1, 400), (100, (1 << 31) - 128, 512), (65, (1 << 31) - 1, 512), (128, 1 << 30, 1000)))
def test_a_call_ends(M, N, K):
    """Where N alone has as many tiles as a launch holds threads for, a launch has fewer of them."""
    if build.is_stale():
        build.build()
    run = subprocess.run([sys.executable, "-c", CALL.format(M=M, N=N, K=K)], cwd=ROOT, capture_output=True, text=True, timeout=60,
                         env=dict(os.environ, PYTHONPATH=ROOT, HIP_VISIBLE_DEVICES="-1"))
    assert run.returncode == 0 and run.stdout.split() == [str(eq.STATUS_DEVICE_ERROR)], run.stdout + run.stderr
