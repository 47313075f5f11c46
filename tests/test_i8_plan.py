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


# measured, us, 16 and 32 rows straight from memory, tiles of 64 with one team, two and four, of 128 and 256: m, n, k
MEASURED = [
    ((17, 256, 384), (4.37, 4.26, 5.38, 4.92, 5.69, 7.08, 11.35)),
    ((17, 4096, 4096), (10.48, 7.36, 13.13, 11.18, 10.13, 23.43, 40.11)),
    ((64, 4096, 16384), (58.55, 45.44, 59.87, 41.09, 33.61, 78.73, 132.78)),
    ((100, 4096, 384), (8.63, 6.59, 4.82, 5.13, 5.89, 7.3, 11.61)),
    ((256, 25088, 384), (84.51, 52.8, 11.27, 16.01, 29.8, 10.67, 13.42)),
    ((1000, 8192, 4096), (1e9, 1e9, 52.15, 57.14, 83.23, 36.77, 42.64)),
    ((2048, 25088, 4096), (1e9, 1e9, 316.94, 338.27, 495.69, 224.32, 191.12)),
    ((4096, 8192, 16384), (1e9, 1e9, 753.2, 756.51, 928.33, 492.53, 364.65)),
    ((2048, 256, 1000), (1e9, 1e9, 6.26, 6.17, 6.64, 10.03, 16.61)),
    ((500, 1000, 16384), (1e9, 1e9, 60.39, 40.72, 33.08, 79.69, 133.59)),
    ((160, 1000, 4096), (14.28, 13.8, 13.79, 11.23, 10.19, 24.01, 41.21)),
    ((333, 4096, 4096), (78.85, 63.95, 19.38, 15.57, 22.44, 23.59, 40.28)),
]


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
        assert set(out.split()) == set("0123456"), (name, out)
    block = text[text.index("PAIRS = ["):]
    sizes = re.findall(r"\((\d+), (\d+), (\d+)\)", block[:block.index("]\n")])
    out = _run(tmp_path, "int main()\n{\n    const int sizes[][3] = {" + ", ".join("{%s, %s, %s}" % s for s in sizes) + r"""};
    // rows, n_in, n_out of a layer: dx sums n_out, dw sums rows
    for (auto& s : sizes) printf("%d ", i8_pick_pair(s[0], s[1], (s[2] + 127) / 128, s[2], s[1], (s[0] + 127) / 128));
}
""")
    assert set(out.split()) == {"-1", "2", "3", "4", "5", "6"}, out
