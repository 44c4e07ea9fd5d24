"""What the compiler made of the kernels of changed scores and of new tokens, read from the code objects of the built library."""
import os
import re
import subprocess

import pytest

from paper_2410_18038_amd import pod
from tests.test_kernel_resources import READELF, code_objects


def scratch_bytes(tmp_path, pattern):
    with open(pod.LIB_PATH, "rb") as f:
        blob = f.read()
    found = {}
    for i, obj in enumerate(code_objects(blob)):
        path = tmp_path / f"{i}.elf"
        path.write_bytes(obj)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True).stdout
        for name, size in re.findall(r"\.name:\s+(\S+).*?\.private_segment_fixed_size:\s+(\d+)", notes, re.S):
            if re.search(pattern, name):
                found[name] = int(size)
    return found


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_kernels_of_one_operation_have_no_scratch_memory(tmp_path):
    """The loops of both operations have no room to wait for reloads.  The kernels that hold both operations keep a few
    values of their set-up in scratch memory, read again between items and units, not in the loops."""
    alone = scratch_bytes(tmp_path, r"(prefill|decode)_scored")
    # 2 types x 3 head_dims x 2 operations x 4 layouts x (masks and slopes, caps), and decodes whose units merge up to 128 channels
    assert len(alone) == 2 * 3 * 2 * 4 * 2 + 2 * 2 * 4 * 2
    assert {k: v for k, v in alone.items() if v} == {}
    both = scratch_bytes(tmp_path, r"fused_(cta_)?scored")
    assert len(both) == 2 * 3 * 2 * 4 * 2 + 2 * 2 * 4 * 2
    assert max(both.values()) <= 160                 # 40 values


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_kernels_of_new_tokens_have_no_scratch_memory(tmp_path):
    found = scratch_bytes(tmp_path, r"append_tokens|token_tables")
    # 2 types x 3 head_dims x 2 rope layouts x one or two groups of heads, and the tables
    assert len(found) == 2 * 3 * 2 * 2 + 1
    assert {k: v for k, v in found.items() if v} == {}
