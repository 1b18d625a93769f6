"""Decode attention's bounded waits and index checks: with a lowered wait limit the kernel
gives up, reports a timeout and leaves the context and the cache usable; the debug build's
checks of every copy pass on ragged batches, and there any role may give up first."""
import pytest
import torch

from tests.gpu_helpers import run_in_child

pytestmark = pytest.mark.gpu

CASES = [(16, 16, 16, 64, [500] * 40), (16, 24, 2, 16, [3000, 1, 700, 5000]), (16, 40, 1, 32, [9000, 20]),
         (8, 8, 8, 16, [900] * 60), (8, 32, 4, 128, [4000, 64, 6000]), (8, 12, 1, 64, [20000, 3])]


def check_timeouts():
    from paper_2608_30877_gb300 import w4a16 as W
    from tests.test_gpu_attention_decode import Case
    for i, (bits, H, Hkv, T, lengths) in enumerate(CASES):
        case = Case(bits, H, Hkv, T, lengths, 40 + i, layers=1, layer=0)
        want = W.attention_decode(case.cache, 0, case.qkv, case.slots, H)
        assert W.get_device_error() == W.OK
        # (a first copy from the L2 cache may be there before its producer looks)
        torch.zeros(1 << 28, dtype=torch.float32, device="cuda")
        W.set_wait_limit(1)
        try:
            W.attention_decode(case.cache, 0, case.qkv, case.slots, H, workspace=case.cache.new_workspace(H))
            assert W.get_device_error() == W.ERR_TIMEOUT, (bits, H, Hkv)
        finally:
            W.set_wait_limit(0)
        # (a workspace that a timed-out call has used is zeroed before its next use)
        again = W.attention_decode(case.cache, 0, case.qkv, case.slots, H)
        assert W.get_device_error() == W.OK
        assert torch.equal(again, want)
        for row in range(len(lengths)):
            case.check_row(again, row, 32768)


def check_debug_build():
    from paper_2608_30877_gb300 import w4a16 as W
    from tests import test_gpu_attention_decode as T
    assert W.LIB_PATH.endswith("libw4a16_debug.so"), W.LIB_PATH
    for bits in (16, 8):
        for page in (16, 64, 128):
            T._run(T.Case(bits, 4, 4, page, T.EDGES, page + bits))
        T._run(T.Case(bits, 24, 2, 32, [1, 40, 129, 3000], 5))
        T._run(T.Case(bits, 70, 1, 16, [300, 17], 6))
        T._run(T.Case(bits, 6, 3, 16, [1, 64, 100, 129, 300], 7), 65)
    check_timeouts()


def test_timeout_is_reported_and_the_cache_stays_usable():
    check_timeouts()


def test_debug_build():
    from paper_2608_30877_gb300 import build as B
    B.build(debug=True)
    run_in_child({"W4A16_DEBUG": "1"}, "test_gpu_decode_failure", "check_debug_build")
