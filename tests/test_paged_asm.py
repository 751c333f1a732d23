"""The generated code of the paged attention kernels: LDS reads and matrix instructions in assembly keep their waits, the direct loads have their
descriptors, bases and offsets in scalar registers and m0 to themselves, and nothing spills in a loop over keys (CPU only)."""
import os
import re
import shutil

import pytest

from tests import asm_checks
from tests.test_run_kernel import result_hazards, unbounded_offsets

pytestmark = pytest.mark.skipif(shutil.which(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")) is None, reason="hipcc not found")

LOAD = re.compile(r"global_load_lds_dword(x4)? v\d+, s\[\d+:\d+\]|buffer_load_dwordx4 v\d+, s\[\d+:\d+\], s\d+ offen( nt)? lds|global_load_lds_dword v\[\d+:\d+\], off")


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    d = tmp_path_factory.mktemp("asm")
    return {f: asm_checks.compile_to_asm(f + ".hip", str(d / (f + ".s"))) for f in ("attn_paged", "attn_paged_tile")}


def _kernels(asm):
    return {n: i for text in asm.values() for n, i in asm_checks.kernels(text).items() if "paged_rows_kernel" in n or "paged_tile_kernel" in n}


def test_direct_loads(asm):
    ks = _kernels(asm)
    assert len(ks) == 12
    for name, ins in ks.items():
        ins = [s for _, s in ins if not s.endswith(":")]
        loads = [k for k, s in enumerate(ins) if s.endswith(" lds") or s.startswith("global_load_lds")]
        # (the tile kernels of e4m3 pages load into registers)
        assert len(loads) >= 8 or "paged_tile_kernelILi64ELb1E" in name or "paged_tile_kernelILi128ELb1E" in name, (name, len(loads))
        for k in loads:
            assert LOAD.fullmatch(ins[k]), (name, ins[k])
            assert ins[k - 1] == "s_nop 0" and re.match(r"s_mov_b32 m0, (s\d+|vcc_(lo|hi))$|s_add_u32 m0, s\d+, ", ins[k - 2]), (name, ins[k - 2 : k + 1])
        assert sum("m0" in s for s in ins) == len(loads), name


def test_assembly_reads_and_products_have_their_waits(asm):
    for name, ins in _kernels(asm).items():
        if "paged_tile_kernel" in name:
            assert asm_checks.in_flight_violations(ins) == [], name
            assert result_hazards(ins) == [], name


def test_offsets_stop_at_the_records(asm):
    """The range check of a descriptor takes records less the scalar offset: that is a minimum with the records, or 0."""
    for name, ins in _kernels(asm).items():
        bad = [b for b in unbounded_offsets([i for i in ins if not i[1].startswith("buffer_load_dwordx4") or i[1].endswith("lds")]) if not re.fullmatch(r"s_mov_b32 s\d+, 0", b[2])]
        assert bad == [], (name, bad[:3])


def test_no_spills_where_they_would_count(asm):
    """Nothing is kept in scratch by the kernels of the listed forms; the others (d = 64 with three workgroups to a compute unit, e4m3 with d = 128 in
    tiles of 128 rows, 32 rows of bf16 with d = 128) have a few values there."""
    for f, text in asm.items():
        for name, spills, _ in asm_checks.spill_report(text):
            if "combine" in name:
                continue
            few = "paged_tile_kernelILi64ELb0E" in name or "paged_tile_kernelILi128ELb1E" in name or "paged_rows_kernelILi128ELb0ELi2E" in name
            assert spills <= (64 if few else 0), (name, spills)
