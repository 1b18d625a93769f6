"""The version names the operators that a library has (no GPU needed)."""
import os
import re

from paper_2608_30877_gb300 import build as B
from paper_2608_30877_gb300 import w4a16 as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_version_with_the_layer_operators():
    B.build()
    for name in ("residual_norm", "rotary_table", "rotary", "kv_rotary", "log_probs", "add_adapters"):
        assert hasattr(W.lib(), "w4a16_" + name)
    assert W.version() >= 300


def test_benchmark_traffic_is_of_the_present_dispatch():
    """A version is not part of what decides a launch's traffic."""
    import bench
    for files in bench.KERNEL_FILES.values():
        for name in files:
            with open(os.path.join(ROOT, "paper_2608_30877_gb300", "csrc", name)) as f:
                assert not re.search(r"\bw4a16_version\b", f.read()), name
