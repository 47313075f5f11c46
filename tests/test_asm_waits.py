"""Inline assembly that reads memory at a scalar address waits for that address.

On this architecture a vector-memory instruction may use a scalar register that a vector instruction wrote (v_readfirstlane and the
like) five wait states later at the earliest.  Nothing in the machine checks that, and the compiler, which keeps such distances for its own
instructions, does not look into inline assembly.  The sources that hold such assembly are compiled to a listing with the library's own
flags, and every load in it is followed back to the last vector instruction that wrote its address.
"""
import os
import re
import shutil
import subprocess

import pytest

from paper_1811_03617_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
WAIT_STATES = 5
WRITES = re.compile(r"v_read(?:first)?lane_b32 s(\d+)\b|v_\w+ s\[(\d+):(\d+)\]|v_\w+ v\S+, s\[(\d+):(\d+)\],")


def _written(instruction):
    """Scalar registers that a vector instruction writes."""
    m = WRITES.match(instruction)
    if not m:
        return set()
    if m.group(1):
        return {int(m.group(1))}
    a, b = (m.group(2), m.group(3)) if m.group(2) else (m.group(4), m.group(5))
    return set(range(int(a), int(b) + 1))


def _states(instruction):
    m = re.match(r"s_nop (\d+)", instruction)
    return int(m.group(1)) + 1 if m else 1


def too_early(listing):
    """(loads in inline assembly that have a scalar address, those of them that come too early)."""
    before, loads, early, inside = [], 0, [], False
    for line in listing.splitlines():
        text = line.strip()
        if text.startswith(";;#ASMSTART"):
            inside = True
        elif text.startswith(";;#ASMEND"):
            inside = False
        if not line.startswith("\t") or text.startswith((".", ";")):
            continue
        text = text.split(";")[0].strip()
        address = re.search(r"s\[(\d+):(\d+)\]", text) if inside and re.match(r"(global|flat|scratch|buffer)_", text) else None
        if address:
            loads += 1
            need, passed = set(range(int(address.group(1)), int(address.group(2)) + 1)), 0
            for earlier in reversed(before):
                if passed >= WAIT_STATES:
                    break
                if _written(earlier) & need:
                    early.append((earlier, text, passed))
                    break
                passed += _states(earlier)
        before = (before + [text])[-WAIT_STATES - 1:]
    return loads, early


def test_the_reader_of_listings():
    """On listings of its own: too early, just late enough, another register, a compare's result."""
    block = "\t;;#ASMSTART\n\ts_mov_b32 m0, s4\n\ts_nop {}\n\tglobal_load_lds_dwordx4 v1, s[8:9]\n\t;;#ASMEND\n"
    for first, nop, want in (("v_readfirstlane_b32 s8, v6", 0, 1), ("v_readfirstlane_b32 s9, v6", 2, 1), ("v_readfirstlane_b32 s9, v6", 3, 0),
                             ("v_readfirstlane_b32 s10, v6", 0, 0), ("v_cmp_gt_f32_e64 s[8:9], 0, v5", 0, 1), ("s_add_u32 s8, s2, s3", 0, 0),
                             ("v_mad_u64_u32 v[10:11], s[8:9], v10, s6, v[188:189]", 0, 1)):
        loads, early = too_early("\t" + first + "\n" + block.format(nop))
        assert loads == 1 and len(early) == want, (first, nop)


@pytest.mark.parametrize("source", ["gvq_muon.hip", "gvq_mx_product.hip", "gvq_codec_ws.hip"])
def test_scalar_addresses_of_inline_assembly(tmp_path, source):
    if shutil.which(HIPCC) is None:
        pytest.skip("no hipcc")
    out = tmp_path / "listing.s"
    subprocess.run([HIPCC, *build.FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-S", "-o", str(out),
                    os.path.join(build.CSRC, source)], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    loads, early = too_early(out.read_text())
    assert loads > 0 or source == "gvq_codec_ws.hip"   # (whose addresses are in vector registers)
    assert not early, f"{len(early)} of {loads}, the first: {early[0]}"
