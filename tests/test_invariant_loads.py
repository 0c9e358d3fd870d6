"""The kernels of a step of serving start before the launches that write what they read have ended, and wait for them.  An invariant
load (``__ldg``, a ``const __restrict__`` pointer, ``ld.global.nc``) at an address that is known at the launch need not stay behind
that wait.  Read from the sources: no GPU."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_01305_b200", "csrc")
FILES = ["attention.cu", "attention.cuh", "attention_tc.cu", "kvcache.cu", "linear8.cu", "linear8.cuh", "linear8_tc.cu", "mx4.cu", "mx4.cuh", "mx4_tc.cu",
         "plan.cu", "tree.cu", "tree.cuh", "tensorcore.cuh"]
# at an address that hangs on lengths or positions, which plain loads bring
DEPENDENT = {"attention.cuh": ["__ldg(a.own_len + b)", "OWN ? __ldg(pages)"], "kvcache.cu": ["ldg_f4(cs + rd / 2)"]}


@pytest.mark.parametrize("name", FILES)
def test_no_invariant_load_at_an_address_known_at_the_launch(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    for known in DEPENDENT.get(name, []):
        assert known in text
        text = text.replace(known, "")
    found = re.findall(r"__ldg\([^;]*|\bldg_\w+\([^;]*|const [\w ]+\*\s*__restrict__ \w+|ld\.global\.nc[^;]*", text)
    assert not found
