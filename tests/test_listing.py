"""The checks that build() makes on the compiler's listings: planted mistakes in listings are found, the library's own sources have none."""
import glob
import os

import pytest

from paper_2602_21760_amd import build, listing

SOURCES = [s for s in sorted(glob.glob(os.path.join(build.CSRC, "*.hip"))) if build.has_asm(s)]


def _kernel(*lines):
    """asm statements are written as `asm: ...`."""
    text = ["_Z6kernelv:"]
    for line in lines:
        text += [";;#ASMSTART", "\t" + line[5:], ";;#ASMEND"] if line.startswith("asm: ") else [line if line.startswith(".") else "\t" + line]
    return "\n".join(text + ["\ts_endpgm", ".Lfunc_end0:"])


READ = "asm: ds_read_b128 v[4:7], v1 offset:0"
WAIT = "asm: s_waitcnt lgkmcnt(0)"


@pytest.mark.parametrize("code,wrong", [
    ((READ, "v_add_u32_e32 v8, v9, v10", WAIT, "v_mov_b32_e32 v8, v4"), False),
    ((READ, "v_mov_b32_e32 v8, v4", WAIT), True),                                            # a copy of what has not arrived
    ((READ, "v_mov_b32_e32 v7, 0", WAIT), True),                                             # another value in the same register
    ((READ, "scratch_store_dwordx2 off, v[6:7], off", WAIT), True),                          # a spill
    ((READ, "asm: ds_read_b128 v[12:15], v1 offset:16", "asm: s_waitcnt lgkmcnt(1)", "v_mov_b32_e32 v8, v4", WAIT), False),      # the older one has arrived
    ((READ, "asm: ds_read_b128 v[12:15], v1 offset:16", "asm: s_waitcnt lgkmcnt(1)", "v_mov_b32_e32 v8, v12", WAIT), True),      # the younger one has not
    ((READ, "asm: s_waitcnt lgkmcnt(1)", "v_mov_b32_e32 v8, v4", WAIT), True),               # a wait that waits for nothing
    ((READ, "s_waitcnt vmcnt(0)", "v_mov_b32_e32 v8, v4"), True),
    ((READ, "s_cbranch_scc0 .LBB0_2", WAIT, ".LBB0_2:", "v_mov_b32_e32 v8, v4"), True),      # on one path only
    ((READ, "s_cbranch_scc0 .LBB0_2", WAIT, "s_branch .LBB0_3", ".LBB0_2:", "s_waitcnt lgkmcnt(0)", ".LBB0_3:", "v_mov_b32_e32 v8, v4"), False),
    ((READ,), True),                                                                         # the kernel ends before it
    (("ds_read_b128 v[4:7], v1 offset:0", "s_waitcnt lgkmcnt(0)", "v_mov_b32_e32 v8, v4"), False)])
def test_reads_in_flight(code, wrong):
    assert bool(listing.faults(_kernel(*code))) == wrong


MFMA = "v_mfma_f32_16x16x32_bf16 v[4:7], v[8:11], v[12:15], v[4:7]"
MAX = "asm: v_max3_f32 v0, v1, v2, v7"


@pytest.mark.parametrize("code,wrong", [
    ((MFMA, MAX), True), ((MFMA, "s_nop 6", MAX), True), ((MFMA, "s_nop 7", MAX), False), ((MFMA, "asm: s_nop 7", MAX), False), ((MFMA, "s_nop 3", "s_setprio 0", "v_mov_b32_e32 v20, 0", "s_nop 1", MAX), False),
    ((MFMA, "asm: v_max3_f32 v0, v1, v2, v3", "asm: v_mov_b32 v4, 0"), True),                # written over
    ((MFMA, "s_cbranch_scc0 .LBB0_2", "s_nop 7", ".LBB0_2:", MAX), True),                    # on one path
    ((MFMA, "s_nop 0", "v_max3_f32 v0, v1, v2, v7"), False),                                 # the compiler's own
    (("v_mfma_f32_16x16x4_f32 v[4:7], v8, v9, v[4:7]", "s_nop 7", MAX), True), (("v_mfma_f32_16x16x4_f32 v[4:7], v8, v9, v[4:7]", "s_nop 11", MAX), False)])
def test_mfma_results(code, wrong):
    assert bool(listing.faults(_kernel(*code))) == wrong


def test_sources_with_asm_are_found():
    names = {os.path.basename(s) for s in SOURCES}
    assert {"packed_attention_mfma.hip", "packed_attention_few.hip", "attention_mfma.hip", "gemm_f32_mfma.hip"} <= names


@pytest.mark.parametrize("src", SOURCES, ids=[os.path.basename(s) for s in SOURCES])
def test_own_sources(src):
    text = build.listing_of(src)
    reads, found = listing.reads_in_flight(text)
    assert reads > 0 and found == []
    assert listing.faults(text) == []


def test_build_refuses_unsafe_code(monkeypatch):
    monkeypatch.setattr(build, "listing_of", lambda src: _kernel(READ, "v_mov_b32_e32 v8, v4", WAIT))
    with pytest.raises(RuntimeError, match="v_mov_b32_e32 v8, v4"):
        build._check_listing("kernel.hip")
