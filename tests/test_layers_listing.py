"""What the 8-bit kernels' inline assembly and LDS assume, read from the compiler's listings: scalar addresses of copies into LDS are waited for,
words of 16 bytes stand at multiples of 16."""
import os
import re
import shutil
import subprocess

import pytest

from paper_1811_03617_amd import build
from test_asm_waits import too_early

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def _compile(tmp_path, source, *more):
    if shutil.which(HIPCC) is None:
        pytest.skip("no hipcc")
    out = tmp_path / "listing"
    subprocess.run([HIPCC, *build.FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", *more, "-S", "-o", str(out),
                    os.path.join(build.CSRC, source)], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    return out.read_text()


def test_copies_wait_for_their_addresses_and_nothing_spills(tmp_path):
    listing = _compile(tmp_path, "gvq_i8_product.hip")
    loads, early = too_early(listing)
    assert loads > 0 and not early, f"{len(early)} of {loads}, the first: {early[:1]}"
    # the sums of a 256 x 256 tile leave 128 registers for everything else: one too many would go to scratch memory
    assert listing.count("scratch_store") == 0


@pytest.mark.parametrize("source,names", [("gvq_i8_product.hip", {"lds"}), ("gvq_i8.hip", {"turn"}), ("gvq_i8_few.hip", {"lds", "sums"}),
                                          ("gvq_distill.hip", {"lds"})])
def test_words_of_16_bytes_are_aligned(tmp_path, source, names):
    seen = set()
    code = _compile(tmp_path, source, "-emit-llvm", "-Xclang", "-disable-llvm-passes")
    for name, align in re.findall(r"^@(\S+) = .*addrspace\(3\) global \[.*align (\d+)$", code, re.M):
        short = next((n for n in names if name == n or re.search(rf"E\d+{n}(_\d+)?$", name)), None)
        if short and not ("lds" == short and name != "lds"):
            seen.add(short)
            assert int(align) >= 16, name
    assert seen == names
