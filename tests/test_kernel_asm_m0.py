"""The compiled gfx950 kernels leave an instruction between a scalar write of M0 and a load to
LDS, which takes its LDS address from M0 (CPU only: the device assembly is read, nothing runs).

On this family of GPUs such a load that directly follows the write may still see the old M0
and put its data at another place of LDS. The compiler keeps the two apart where it writes
both, but not inside of inline asm."""
import glob
import os
import re

import pytest

from test_kernel_asm import ROOT, device_asm

SOURCES = sorted(os.path.basename(p) for p in glob.glob(os.path.join(ROOT, "paper_2601_20595_amd", "csrc", "*.hip")))

_WRITE = re.compile(r"s_\w+\s+m0\s*,")
_READ = re.compile(r"buffer_load_\w+\s.*\blds\b|global_load_lds_\w+\s")


def loads_behind_m0(asm: str):
    """Loads to LDS whose last instruction before them writes M0."""
    bad, last = [], ""
    for line in asm.split("\n"):
        inst = line.split(";")[0].strip()
        if not inst or inst.startswith(".") or inst.endswith(":"):
            continue
        if _READ.match(inst) and _WRITE.match(last):
            bad.append(inst)
        last = inst
    return bad


def test_the_search_finds_a_load_right_behind_the_write():
    load = "buffer_load_dwordx4 v2, s[4:7], 0 offen lds"
    assert loads_behind_m0("\ts_mov_b32 m0, s2\n\t%s\n" % load) == [load]
    assert loads_behind_m0("\ts_add_i32 m0, s2, s3 ; note\n.LBB0_1:  ; loop\n\t;;#ASMSTART\n\tglobal_load_lds_dword v[0:1], off\n") != []
    assert loads_behind_m0("\ts_mov_b32 m0, s2\n\ts_nop 0\n\t%s\n" % load) == []
    assert loads_behind_m0("\ts_mov_b32 m0, s2\n\tv_add_u32 v2, s3, v1\n\t%s\n" % load) == []
    assert loads_behind_m0("\ts_mov_b32 m0, s2\n\tbuffer_load_dwordx4 v[0:3], v2, s[4:7], 0 offen\n") == []
    assert loads_behind_m0("\ts_mov_b32 s3, m0\n\t%s\n" % load) == []


@pytest.mark.parametrize("source", SOURCES)
def test_no_load_to_lds_right_behind_a_write_of_m0(source):
    asm = device_asm(os.path.join(ROOT, "paper_2601_20595_amd", "csrc", source))
    if "attn" in source or "gemm" in source:
        assert re.search(r"^\s*buffer_load_\w+ .*\blds\b", asm, re.M), "the pattern finds no load to LDS"
    assert loads_behind_m0(asm) == []
