"""What the kernels assume of their LDS is said to the compiler: words of 16 bytes stand at multiples of 16, and a copy into LDS goes where
the array that it fills lies.  Both are read from the compiler's own intermediate code."""
import os
import re
import shutil
import subprocess

import pytest

from paper_1811_03617_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def _code(tmp_path, source, *more):
    if shutil.which(HIPCC) is None:
        pytest.skip("no hipcc")
    out = tmp_path / "code.ll"
    subprocess.run([HIPCC, *build.FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-emit-llvm", *more, "-S",
                    "-o", str(out), os.path.join(build.CSRC, source)], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    return out.read_text()


@pytest.mark.parametrize("source,names", [("gvq_muon.hip", {"lds", "tile"}), ("gvq_muon_small.hip", {"lds"}), ("gvq_mx_product.hip", {"lds"}),
                                          ("gvq_mx.hip", {"tile", "dust"}), ("gvq_mx_few.hip", {"sums"})])
def test_words_of_16_bytes_are_aligned(tmp_path, source, names):
    seen = set()
    for name, align in re.findall(r"^@(\S+) = .*addrspace\(3\) global \[.*align (\d+)$", _code(tmp_path, source, "-Xclang", "-disable-llvm-passes"), re.M):
        short = next((n for n in names if name == n or re.search(rf"E\d+{n}(_\d+)?$", name)), None)
        # (the few numbers of a sum over a work-group are read one by one)
        if short and not ("lds" == short and name != "lds"):
            seen.add(short)
            assert int(align) >= 16, name
    assert seen == names


def test_copies_go_where_their_array_lies(tmp_path):
    code = _code(tmp_path, "gvq_mx_product.hip")
    assert "global_load_lds_dwordx4" in code
    assert re.search(r"ptrtoint \(ptr addrspace\(3\) @lds to i\d+\)", code)
