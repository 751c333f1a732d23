"""Where the paged attention kernels keep values in scratch memory (CPU only): few of them, and none beside a matrix instruction of a loop over keys.

paged_tile_kernel<128, e4m3>, paged_tile_kernel<64, bf16> and paged_rows_kernel<128, bf16, 32 rows> have more values than registers.  What they keep in scratch
they read back in a row tile's set-up and in the parts of a loop that most tiles jump over: masks, descriptors of tiles that are not seen as a whole, the
second pass."""
import os
import re
import shutil

import pytest

from tests import asm_checks

pytestmark = pytest.mark.skipif(shutil.which(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")) is None, reason="hipcc not found")

SPILLS = {"paged_rows_kernelILi128ELb0ELi2E": 8, "paged_tile_kernelILi64ELb0E": 29, "paged_tile_kernelILi128ELb1E": 39}


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    d = tmp_path_factory.mktemp("asm")
    return [asm_checks.compile_to_asm(f + ".hip", str(d / (f + ".s"))) for f in ("attn_paged", "attn_paged_tile")]


def _blocks(asm):
    """(kernel, depth of the loop that it is in, instructions) of every basic block."""
    name, depth, ins = None, 0, []
    for line in asm.split("\n"):
        m = re.match(r"^(_Z\w+):", line)
        if m or line.startswith(".Lfunc_end") or re.match(r"^(\.LBB\d+_\d+|; %bb\.\d+):", line):
            if name is not None and ins:
                yield name, depth, ins
            ins, depth = [], 0
            if m:
                name = m.group(1)
            elif line.startswith(".Lfunc_end"):
                name = None
        if name is None:
            continue
        depth = max([depth] + [int(x) for x in re.findall(r"Depth[= ](\d+)", line)])
        text = line.split(";")[0].strip()
        if text and not text.startswith(".") and not text.endswith(":"):
            ins.append(text)


def test_spills_are_as_few_as_they_are(asm):
    seen = 0
    for text in asm:
        for name, spills, _ in asm_checks.spill_report(text):
            seen += 1
            assert spills <= next((n for part, n in SPILLS.items() if part in name), 0), (name, spills)
    assert seen == 18


def test_no_scratch_beside_the_products_of_a_loop(asm):
    loops = 0
    for text in asm:
        for name, depth, ins in _blocks(text):
            products, scratch = sum(s.startswith("v_mfma") for s in ins), [s for s in ins if s.startswith("scratch_")]
            if depth >= 2:                                       # (depth 1 is the loop over row tiles)
                loops += products > 0
                assert not any(s.startswith("scratch_store") for s in scratch), name
                assert products == 0 or not scratch, (name, scratch)
    assert loops >= 30
