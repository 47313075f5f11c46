"""Which way a 4-bit product takes (csrc/gvq_mx_plan.h), checked on the CPU: the header is plain C++."""
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_1811_03617_amd", "csrc")


def _run(tmp_path, body):
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text('#include <cstdio>\n#include <cmath>\n#include "gvq_mx_plan.h"\n' + body)
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout[-4000:]
    return out.stdout


def test_the_time_is_that_of_the_way_that_is_taken(tmp_path):
    """Sums of fewer than four steps have one shape of tiles, and it is its time that is compared with the other ways; longer ones have the rest."""
    _run(tmp_path, r"""
int main()
{
    for (int64_t steps = 0; steps < 40; ++steps)
        for (double m = 1; m < 40000; m *= 1.7)
            for (double n = 1; n < 40000; n *= 1.7) {
                const MxWay t = mx_tiles((int64_t)m, (int64_t)n, steps), w = mx_way((int64_t)m, (int64_t)n, steps);
                if ((t.shape == MX_NARROW) != (steps < 4) || t.us != mx_tile_time(mx_shapes[t.shape], (int64_t)m, (int64_t)n, steps)) return 1;
                const double us = w.few ? mx_few_time((int64_t)m, (int64_t)n, steps, w.few) : t.us;
                if (w.us != us || (!w.few && w.shape != t.shape)) return 2;
                for (int k = 0; k < 5; ++k)
                    if ((k == MX_NARROW) == (steps < 4) && mx_tile_time(mx_shapes[k], (int64_t)m, (int64_t)n, steps) < w.us) return 3;
                if (mx_few_time((int64_t)m, (int64_t)n, steps, 1) < w.us || mx_few_time((int64_t)m, (int64_t)n, steps, 2) < w.us) return 4;
            }
    return 0;
}
""")


# measured, us, with tiles and with 16 and 32 rows a work-group: m, n, k
SHORT = [((64, 64, 250), (3.44, 2.94, 3.03)), ((64, 512, 384), (3.90, 3.09, 3.16)), ((17, 1000, 250), (3.45, 3.07, 3.13)), ((200, 1000, 384), (4.04, 4.86, 3.71)),
         ((64, 4096, 100), (3.40, 5.08, 3.69)), ((200, 4096, 384), (4.37, 12.48, 8.51)), ((4096, 4096, 250), (16.76, 203.52, 116.76)),
         ((4096, 25088, 384), (100.53, 1197.18, 718.40)), ((4, 25088, 100), (3.36, 6.88, 7.29)), ((9000, 3, 384), (3.98, 4.33, 3.58))]


def test_short_sums_take_what_is_fast(tmp_path):
    """At most 6 % behind the fastest."""
    sizes = ", ".join("{%d, %d, %d}" % s for s, _ in SHORT)
    out = _run(tmp_path, "int main()\n{\n    const int sizes[][3] = {" + sizes + r"""};
    for (auto& s : sizes) printf("%d\n", mx_way(s[0], s[1], (s[2] + 127) / 128).few);
}
""")
    for (size, us), few in zip(SHORT, out.split()):
        assert us[int(few)] <= 1.06 * min(us), size


def test_the_sizes_that_are_run_take_every_way(tmp_path):
    text = open(os.path.join(HERE, "test_gpu_mx_ways.py")).read()
    sizes = re.findall(r"\((\d+), (\d+), (\d+)\)", text[text.index("SIZES = ["):text.index("]\n")])
    out = _run(tmp_path, "int main()\n{\n    const int sizes[][3] = {" + ", ".join("{%s, %s, %s}" % s for s in sizes) + r"""};
    for (auto& s : sizes) {
        const MxWay w = mx_way(s[0], s[1], (s[2] + 127) / 128);
        printf("%d%d ", w.few, w.few ? 0 : w.shape);
    }
}
""")
    assert set(out.split()) == {"10", "20", "00", "01", "02", "03", "04"}
