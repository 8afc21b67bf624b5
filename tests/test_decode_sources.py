"""What the decode entry points' host code has to do in a certain order, read off the sources: it takes two devices to see it at run time."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_00198_b200", "csrc")


def _entry_points():
    """(name, body) of every exported function that makes its context's device current."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        src = open(path).read()
        for m in re.finditer(r'extern "C" int (str_\w+)\([^{;]*\) \{(.*?)\n\}', src, re.S):
            if "StrDeviceScope" in m.group(2):
                yield m.group(1), m.group(2)


ENTRIES = dict(_entry_points())


def test_all_decode_calls_make_their_device_current():
    assert {"str_kv4_append", "str_kv4_read", "str_kv4_attn", "str_kv4_evict", "str_mamba2_step"} <= set(ENTRIES)


@pytest.mark.parametrize("name", sorted(ENTRIES))
def test_the_device_is_current_before_anything_is_made_or_enqueued_on_it(name):
    """Timing events are created on the current device and recorded on a stream of the context's; the same goes for all else."""
    body = ENTRIES[name]
    at = body.index("StrDeviceScope")
    for call in ("StrProfScope", "<<<", "cudaMemsetAsync", "cudaLaunchKernelEx", "launch_type", "str_topk_select("):
        if call in body:
            assert at < body.index(call), call
