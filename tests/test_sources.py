"""What the kernels' sources have to keep to (CPU)."""
import os

import pytest

from paper_2608_13076_gb300 import _build


@pytest.mark.parametrize("name", ["attn_common.cuh", "int4.cuh", "kv4_attention_tc.cu", "kv4_cache.cu", "linear_w4.cu",
                                  "verify_attention_tc.cu"])
def test_early_launched_kernels_read_by_plain_loads(name):
    """Launched while the kernel before still runs, they read the caller's tensors without a read-only load's promise
    that nothing writes those for as long as the kernel lives (see launch.h)."""
    with open(os.path.join(_build.CSRC, name)) as f:
        source = f.read()
    for load in ("__ldg", "ld.global.nc", "__restrict__"):
        assert load not in source
