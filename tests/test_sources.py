"""What the kernels' sources have to keep to (CPU)."""
import os
import re

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


def test_rounds_of_histograms_take_turns():
    """A thread late in reading where a round's boundary lies must not meet what the next round's first threads store
    there, as no barrier stands between the two: every access within the rounds is to the round's own slot."""
    with open(os.path.join(_build.CSRC, "sample.cu")) as f:
        source = f.read()
    rounds = source[source.index("auto boundary = ["):source.index("// ---- draw in ascending order")]
    shared = [w for name in ("cut", "above") for w in re.findall(r"\bs\." + name + r"\w*(?:\[\w+\])?", rounds)]
    assert len(shared) >= 5 and all(w.endswith("[turn]") for w in shared), shared
    assert "turn ^= 1" in rounds


def test_the_start_of_the_values_waits_for_a_barrier_that_completes_once():
    """A wait by parity has to look before the barrier's next phase ends.  Nothing holds the queries' barrier back for the
    warp that copies values, which is no user of them: it waits for one that is arrived at once."""
    with open(os.path.join(_build.CSRC, "tree_attention.cu")) as f:
        source = f.read()
    waits = re.findall(r"if \(is_v && it == 0\) ok = wait_short\(&bars\[(\w+)\], 0, s_abort\);", source)
    assert waits == ["kBarStart"]
    assert re.findall(r"if \((.*)\) mbar_arrive\(&bars\[kBarStart\]\);", source) == ["seg == 0 && lane == 0"]
    assert len(re.findall("kBarStart", source)) == 5  # its number twice, its initialisation, the wait, the arrival
