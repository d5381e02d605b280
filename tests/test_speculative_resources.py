"""CPU: what the kernels of a speculative step spill, from the compiler's report and assembly for gfx950. Nothing goes to
memory, and no vector register is spilled; scalar ones are, into lanes of vector registers: pointers and
lengths that are set once and used again after a loop. In tree attention none is read back in a loop over keys. In
verification's last launch, one workgroup a sequence, they are: about 30 of the 1500 instructions that a wave
takes for 1024 elements, under the pass's loads. Draft trees and compaction spill none."""
import os
import re
import subprocess

import pytest

from test_kernel_resources import CSRC, FLAGS, HIPCC, _resources

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")

# scalar registers in lanes, at most: what the kernels hold now
MOST = {"draft.hip": 0, "tree.hip": 0, "tree_rows.hip": 18, "verify.hip": 45}


@pytest.mark.parametrize("src", list(MOST))
def test_spills(src):
    for name, r in _resources(src).items():
        assert r["VGPRs Spill"] == 0 and r["ScratchSize"] == 0, (name, r)
        most = 1 if "verify_round" in name else MOST[src]
        assert r["SGPRs Spill"] <= most, (name, r)


def _inner_loops(src):
    """(kernel, lines) of the loops that hold no other loop."""
    out = subprocess.run([HIPCC, *FLAGS, "--cuda-device-only", "-S", os.path.join(CSRC, src), "-o", "-"],
                         capture_output=True, text=True, check=True).stdout
    for f in re.finditer(r"^(_ZN\S+):", out, re.M):
        body = out[f.start():out.index(".Lfunc_end", f.start())].split("\n")
        labels = {m.group(1): i for i, x in enumerate(body) if (m := re.match(r"^(\.LBB\d+_\d+):", x))}
        spans = []
        for i, x in enumerate(body):
            m = re.search(r"s_c?branch\w*\s+(\.LBB\d+_\d+)\s*$", x)
            if m and labels.get(m.group(1), i) < i:
                spans.append((labels[m.group(1)], i))
        for a, b in spans:
            if not any(a <= c and d <= b and (a, b) != (c, d) for c, d in spans):
                yield f.group(1), body[a:b + 1]


def test_tree_attention_reads_no_spilled_register_in_its_key_loops():
    pairs = set()
    for name, body in _inner_loops("tree_rows.hip"):
        m = re.search(r"cross_rows_kernelILi(\d+)ELi(\d+)ELi(\d)ELi(\d)E", name)
        mfma = sum("v_mfma" in x for x in body)
        if not m or not mfma:
            continue
        assert not any(re.search(r"v_readlane|v_writelane|scratch_", x) for x in body), name
        d, tiles = int(m.group(1)), int(m.group(4))
        if mfma == 2 * tiles * (2 * (d // 32) + d // 16):     # two steps of 32 keys
            pairs.add(m.groups())
    assert len(pairs) == 24                                     # found in every form
