"""What the compiler reported about the kernels when the library was built: no kernel may keep
registers in scratch memory (a spill turns every use into memory traffic inside the hot loops;
it has cost single instantiations up to 28 % without failing any parity test)."""
import os
import re
import subprocess

import pytest

import __graft_entry__ as entry

REPORT = os.path.join(entry.PKG, "_build", "kernel_resources.txt")

SAMPLE = """\
a.hip:5:1: remark: Function Name: _Z5alphav [-Rpass-analysis=kernel-resource-usage]
    5 | __global__ void alpha() {
      | ^
a.hip:5:1: remark:     TotalSGPRs: 16 [-Rpass-analysis=kernel-resource-usage]
a.hip:5:1: remark:     VGPRs: 74 [-Rpass-analysis=kernel-resource-usage]
a.hip:5:1: remark:     AGPRs: 0 [-Rpass-analysis=kernel-resource-usage]
a.hip:5:1: remark:     ScratchSize [bytes/lane]: 0 [-Rpass-analysis=kernel-resource-usage]
a.hip:5:1: remark:     Dynamic Stack: False [-Rpass-analysis=kernel-resource-usage]
a.hip:5:1: remark:     Occupancy [waves/SIMD]: 6 [-Rpass-analysis=kernel-resource-usage]
a.hip:5:1: remark:     SGPRs Spill: 0 [-Rpass-analysis=kernel-resource-usage]
a.hip:9:1: remark: Function Name: _Z4betav [-Rpass-analysis=kernel-resource-usage]
a.hip:9:1: remark:     VGPRs: 128 [-Rpass-analysis=kernel-resource-usage]
a.hip:9:1: remark:     ScratchSize [bytes/lane]: 68 [-Rpass-analysis=kernel-resource-usage]
a.hip:9:1: remark:     Occupancy [waves/SIMD]: 4 [-Rpass-analysis=kernel-resource-usage]
a.hip:1:1: warning: something else
"""


def test_resource_remarks_are_parsed():
    assert entry.kernel_resources(SAMPLE) == {"_Z5alphav": (74, 0, 6), "_Z4betav": (128, 68, 4)}
    assert entry.kernel_resources("") == {}


def test_no_kernel_spills_registers():
    if not os.path.exists(REPORT):
        pytest.skip("the library in the tree was not built by build() of this version: no resource report")
    rows = [l.split() for l in open(REPORT) if l.strip() and not l.startswith("#")]
    assert len(rows) >= 100, "the report lists fewer kernels than the library has"
    spilled = [(r[0], int(r[2])) for r in rows if int(r[2]) != 0]
    assert not spilled, spilled


def unguarded_moves(listing):
    """Moves between lanes (DPP) of a compiler's listing whose source one of the two wait states in front of them wrote inside an
    inline assembly block: the hardware does not wait there, and the compiler does not see it.  A wait state is an instruction, or
    one of an s_nop's."""
    regs = lambda text: {int(n) for a, b, c in re.findall(r"\bv(?:(\d+)\b|\[(\d+):(\d+)\])", text)   # noqa: E731
                         for n in ([a] if a else range(int(b), int(c) + 1))}
    found, inside, recent, at = [], False, {}, 0   # recent: register -> wait state of its last write, in a block
    for number, line in enumerate(listing.splitlines(), 1):
        if "#ASMSTART" in line or "#ASMEND" in line:
            inside = "#ASMSTART" in line
            continue
        for text in line.split(";")[0].split("\n"):
            m = re.match(r"\s+([a-z]\w+)\s*(.*)", text)
            if not m:
                continue
            op, operands = m.group(1), [x.strip() for x in m.group(2).split(",")]
            if op == "s_nop":
                at += 1 + int(operands[0], 0)
                continue
            if re.search(r"\b(quad_perm|row_\w+|wave_\w+):", text) or op.endswith("_dpp"):
                found += [(number, text.strip()) for r in regs(operands[1]) if r in recent and at - recent[r] < 2]
            at += 1
            if op.startswith("v_"):
                for r in regs(operands[0]):
                    recent.pop(r, None)
                    if inside:
                        recent[r] = at
    return found


def test_unguarded_moves_are_found():
    text = """
\tv_min_f32_e32 v1, v2, v3
\tv_mov_b32_dpp v4, v1 row_newbcast:2 row_mask:0xf bank_mask:0xf
\t;;#ASMSTART
\tv_min_f32 v5, v2, v3
\t;;#ASMEND
{}\tv_mov_b32_dpp v4, v5 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf
"""
    assert len(unguarded_moves(text.format(""))) == 1
    assert len(unguarded_moves(text.format("\tv_add_u32_e32 v9, v8, v8\n"))) == 1
    assert len(unguarded_moves(text.format("\ts_nop 0\n"))) == 1
    assert unguarded_moves(text.format("\t;;#ASMSTART\n\ts_nop 1\n\t;;#ASMEND\n")) == []
    assert unguarded_moves(text.format("\tv_add_u32_e32 v9, v8, v8\n\tv_add_u32_e32 v10, v8, v8\n")) == []
    assert unguarded_moves(text.format("\tv_add_u32_e32 v5, v8, v8\n")) == []


def test_moves_between_lanes_wait_for_inline_assembly(tmp_path):
    out = tmp_path / "store.s"
    subprocess.check_call(["hipcc", *entry.HIPCC_FLAGS, "-I" + os.path.join(entry.ROOT, "include"), "-I" + entry.CSRC, "--cuda-device-only", "-S",
                           os.path.join(entry.CSRC, "thk_paged_store.hip"), "-o", str(out)], stderr=subprocess.DEVNULL)
    listing = out.read_text()
    assert listing.count("v_mov_b32_dpp") > 100 and "#ASMSTART" in listing
    assert unguarded_moves(listing) == []
