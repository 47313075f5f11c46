"""Which way an 8-bit product takes (csrc/gvq_i8_plan.h), checked on the CPU: the header is plain C++."""
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_1811_03617_amd", "csrc")


def _run(tmp_path, body):
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text('#include <cstdio>\n#include <cmath>\n#include "gvq_i8_plan.h"\n' + body)
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout[-4000:]
    return out.stdout


def test_the_way_that_is_picked_is_the_least(tmp_path):
    """For one product and for two; sums over nothing take tiles."""
    _run(tmp_path, r"""
int main()
{
    for (int64_t steps = 0; steps < 1000; steps = steps * 3 / 2 + 1)
        for (double m = 1; m < 100000; m *= 2.3)
            for (double n = 1; n < 100000; n *= 2.3)
                for (int sums = 1; sums <= 2; ++sums) {
                    const int w = i8_pick((int64_t)m, (int64_t)n, sums, steps);
                    if (w < 0 || w >= I8_WAYS || (steps == 0 && w <= I8_FEW_32)) return 1;
                    const double us = i8_way_time(i8_ways[w], (int64_t)m, (int64_t)n, sums, steps);
                    for (int k = steps == 0 ? I8_TILE_64 : 0; k < I8_WAYS; ++k)
                        if (i8_way_time(i8_ways[k], (int64_t)m, (int64_t)n, sums, steps) < us) return 2;
                    const int64_t m1 = (int64_t)n, n1 = (int64_t)m, s1 = steps / 2;
                    const int p = i8_pick_pair((int64_t)m, (int64_t)n, steps, m1, n1, s1);
                    if (p != -1 && p < I8_TILE_64) return 3;
                }
    return 0;
}
""")


# measured, us, 16 and 32 rows straight from memory, tiles of 64 with two stages and four, of 128 and 256: m, n, k
MEASURED = [((17, 256, 384), (3.82, 3.86, 4.53, 4.52, 6.84, 11.05)), ((17, 4096, 4096), (10.36, 7.37, 12.41, 12.66, 22.94, 40.16)),
            ((64, 4096, 16384), (59.91, 45.35, 60.57, 40.36, 77.39, 132.5)), ((100, 4096, 384), (8.59, 6.6, 4.65, 4.68, 7.13, 11.43)),
            ((256, 25088, 384), (86.25, 53.05, 10.73, 14.37, 10.4, 13.21)), ((1000, 8192, 4096), (1e9, 1e9, 55.0, 63.2, 37.34, 45.95)),
            ((2048, 25088, 4096), (1e9, 1e9, 303.18, 339.12, 220.94, 192.83)), ((4096, 8192, 16384), (1e9, 1e9, 750.85, 790.5, 495.09, 371.31)),
            ((2048, 256, 1000), (1e9, 1e9, 6.05, 6.12, 9.96, 16.58)), ((500, 1000, 16384), (1e9, 1e9, 60.54, 39.18, 79.2, 134.63))]


def test_what_is_picked_is_fast(tmp_path):
    sizes = ", ".join("{%d, %d, %d}" % s for s, _ in MEASURED)
    out = _run(tmp_path, "int main()\n{\n    const int sizes[][3] = {" + sizes + r"""};
    for (auto& s : sizes) printf("%d\n", i8_pick(s[0], s[1], 1, (s[2] + 127) / 128));
}
""")
    for (size, us), way in zip(MEASURED, out.split()):
        assert us[int(way)] <= 1.1 * min(us), size


def test_the_sizes_that_are_run_take_every_way(tmp_path):
    text = open(os.path.join(HERE, "test_gpu_i8_ways.py")).read()
    for name, sums in (("PLAIN", 1), ("GATED", 2)):
        block = text[text.index(name + " = ["):]
        sizes = re.findall(r"\((\d+), (\d+), (\d+)\)", block[:block.index("]\n")])
        out = _run(tmp_path, "int main()\n{\n    const int sizes[][3] = {" + ", ".join("{%s, %s, %s}" % s for s in sizes) + r"""};
    for (auto& s : sizes) printf("%d ", i8_pick(s[0], s[1], """ + str(sums) + r""", (s[2] + 127) / 128));
}
""")
        assert set(out.split()) == set("012345"), (name, out)
    block = text[text.index("PAIRS = ["):]
    sizes = re.findall(r"\((\d+), (\d+), (\d+)\)", block[:block.index("]\n")])
    out = _run(tmp_path, "int main()\n{\n    const int sizes[][3] = {" + ", ".join("{%s, %s, %s}" % s for s in sizes) + r"""};
    // rows, n_in, n_out of a layer: dx sums n_out, dw sums rows
    for (auto& s : sizes) printf("%d ", i8_pick_pair(s[0], s[1], (s[2] + 127) / 128, s[2], s[1], (s[0] + 127) / 128));
}
""")
    assert set(out.split()) == {"-1", "2", "3", "4", "5"}, out
