"""The adapters' tcgen05 kernel when a wait runs out, in every role and with slices of K that fit in its stages: it lets its
copies and MMAs end, says so, and the calls after it are right."""
import os
import subprocess
import sys

import pytest
import torch

from tests.kv_reference import i32
from tests.test_gpu_adapters import make

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# rows, inputs, rank, first rows of the sequences: one step of 64 and two to a slice, as many as there are stages, more of
# them; clusters of one and of several; adapters that take several turns of a tile
CASES = [(2000, 64, 16, [0, 900, 2000]), (2000, 128, 32, [0, 900, 2000]), (20000, 256, 16, [0, 9000, 20000]),
         (20000, 192, 64, [0, 9000, 20000]), (300, 2048, 48, [0, 300]), (1500, 4096, 64, list(range(0, 1501, 20))),
         (40000, 1024, 64, list(range(0, 40001, 25)))]


def check_waits(cases=CASES, rounds=10):
    from paper_2608_30877_gb300 import w4a16 as W
    for M, K, rank, starts in cases:
        given = make(M, 256, K, rank, 7)
        lists = dict(adapters=i32([i % 7 for i in range(len(starts) - 1)]), seq_start=i32(starts))
        want = W.add_adapters(**given, **lists)
        assert W.get_device_error() == W.OK
        for _ in range(rounds):
            W.set_wait_limit(1)
            try:
                W.add_adapters(**given, **lists)
                assert W.get_device_error() == W.ERR_TIMEOUT
            finally:
                W.set_wait_limit(0)
            assert torch.equal(W.add_adapters(**given, **lists), want)
            assert W.get_device_error() == W.OK


def test_waits_that_run_out():
    check_waits()


_CHILD = r"""
import sys
sys.path.insert(0, {root!r})
from paper_2608_30877_gb300 import w4a16 as W
from tests.test_gpu_adapter_waits import check_waits
assert W.LIB_PATH.endswith("libw4a16_debug.so"), W.LIB_PATH
check_waits()
print("ok")
"""


def test_any_role_may_give_up_first():
    """In the debug build every role polls without suspending, so that it is not the producer alone that gives up."""
    from paper_2608_30877_gb300 import build as B
    B.build(debug=True)
    r = subprocess.run([sys.executable, "-c", _CHILD.format(root=ROOT)], env=dict(os.environ, W4A16_DEBUG="1"),
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "ok" in r.stdout, r.stdout[-3000:] + r.stderr[-3000:]
