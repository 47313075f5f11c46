"""The units of the Newton-Schulz steps (csrc/gvq_muon_plan.h), checked on the CPU: the header is plain C++."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1811_03617_amd", "csrc")


def _run(tmp_path, body):
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include "gvq_muon_plan.h"\n' + body)
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout[-4000:]
    return out.stdout


RANDOM = r"""
static unsigned seed = 1;
static double rnd() { return seed = seed * 1664525u + 1013904223u, (seed >> 8) / 16777216.0; }
[[maybe_unused]] static double coefficient() { return rnd() < 0.2 ? 0.0 : (rnd() - 0.5) * std::exp(6.0 * rnd()); }
"""


def test_bounds_hold_and_are_met(tmp_path):
    """Against 2000 points of [0, S]: never below any of them, and no more above the largest than two neighbouring points differ."""
    _run(tmp_path, RANDOM + r"""
int main()
{
    for (int n = 0; n < 3000; ++n) {
        const double a = coefficient(), b = coefficient(), c = coefficient(), S = std::exp(12.0 * (rnd() - 0.6));
        const double step = ns_step_bound(a, b, c, S), poly = ns_poly_bound(b, c, S);
        double s1 = 0, p1 = 0, ds = 0, dp = 0, sl = 0, pl = 0;
        for (int i = 0; i <= 2000; ++i) {
            const double s = S * i / 2000, x = s * s, f = std::fabs(s * (a + x * (b + x * c))), p = std::fabs(x * (b + x * c));
            s1 = f > s1 ? f : s1;
            p1 = p > p1 ? p : p1;
            if (i) { ds = std::fabs(f - sl) > ds ? std::fabs(f - sl) : ds; dp = std::fabs(p - pl) > dp ? std::fabs(p - pl) : dp; }
            sl = f; pl = p;
        }
        const double e = 1e-12;
        if (step < s1 * (1 - e) || step > s1 * (1 + e) + ds || poly < p1 * (1 - e) || poly > p1 * (1 + e) + dp) {
            printf("%g %g %g to %g: %g for %g, %g for %g\n", a, b, c, S, step, s1, poly, p1);
            return 1;
        }
    }
    return 0;
}
""")


def test_everything_that_is_kept_fits(tmp_path):
    """Numbers at their bounds are at least as many units as ordinary ones, and at most 65504 where singular values stay below 3.9 and the polynomial
    below 63, in every step of random polynomials; the factors do what the formula says (of results that fp32 holds)."""
    _run(tmp_path, RANDOM + r"""
int main()
{
    for (int n = 0; n < 3000; ++n) {
        float coef[8][3];
        for (auto& t : coef)
            for (float& v : t) v = (float)coefficient();
        const double S0 = n % 3 == 0 ? 1.0 : std::exp(60.0 * (rnd() - 1.0));
        NsFactors f[8];
        ns_factors(coef[0], 8, S0, f);
        double S = S0;
        for (int t = 0; t < 8 && S > 1e-30 && S < 1e30; ++t) {
            const double a = coef[t][0], b = coef[t][1], c = coef[t][2];
            const int k = ns_unit_x(S);
            const double x = std::ldexp(S, 12 + k), A = std::ldexp(S * S, 12 + 2 * k), B = ns_poly_bound(b, c, S);
            const int j = ns_unit_p(B);
            const double P = std::ldexp(B, 10 + j);
            if (k < 0 || j < 0 || (S < 3.9 && (x > 65504 || A > 65504)) || (B < 63 && P > 65504) || x < 2048 || (B > 0 && P < 64)) { printf("%d %d: S %g k %d x %g A %g P %g\n", n, t, S, k, x, A, P); return 1; }
            // what the kernels make of one number s = S: from its units into theirs
            const double s = S, want = B == 0 ? 0 : s * s * (b + s * s * c), next = ns_step_bound(a, b, c, S);
            const int kn = t < 7 ? ns_unit_x(next) : k;
            const double p = f[t].pa * A + f[t].pc * A * A, y = f[t].sa * x + f[t].ss * p * x, up = std::ldexp(1.0, 10 + j), ux = std::ldexp(1.0, 12 + kn);
            if (std::fabs(p - want * up) > 1e-9 * B * up || (next < 1e30 && std::fabs(y - s * (a + want) * ux) > (1e-9 * s * (std::fabs(a) + B) + 1e-38) * ux) || (t == 7 && f[t].out * ux != 1)) {
                printf("%d %d: p %g for %g, y %g for %g\n", n, t, p, want * up, y, s * (a + want) * ux);
                return 1;
            }
            S = next;
        }
    }
    return 0;
}
""")


def test_ordinary_matrices_keep_their_units(tmp_path):
    """The default polynomial of a matrix whose norm is far above eps: 2^-12 and 2^-10 in every step; and what a norm of none, or none that is a number, gets."""
    _run(tmp_path, r"""
int main()
{
    const float a = 3.4445f, b = -4.7750f, c = 2.0315f;
    float coef[64][3];
    for (auto& t : coef) { t[0] = a; t[1] = b; t[2] = c; }
    NsFactors f[64];
    ns_factors(coef[0], 64, 1.0, f);
    for (auto& t : f)
        if (t.pa != b / 4 || t.pc != c / 16384 || t.sa != a || t.ss != 1.f / 1024 || t.out != 1.f / 4096) return 1;
    if (!ns_is_whole(1.0) || !ns_is_whole(0.51) || ns_is_whole(0.5) || ns_is_whole(1e-30) || !ns_is_whole(0.0) || !ns_is_whole(NAN)) return 2;
    return ns_unit_x(NAN) || ns_unit_x(INFINITY) || ns_unit_x(0.0) || ns_unit_p(NAN) || ns_unit_p(INFINITY) ? 3 : 0;
}
""")


def test_the_sizes_that_are_run_take_every_way(tmp_path):
    """Each size of _muon_ways.py is computed as it says there, and together they reach everything that the rule can pick: over many sizes it picks
    nothing else."""
    from _muon_ways import PICKED, WAYS
    out = _run(tmp_path, "#include <initializer_list>\nstatic const int sizes[][3] = {" + ", ".join("{%d, %d, %d}" % k for k in WAYS) + "};\n" + RANDOM + r"""
static void tell(int64_t b, int64_t m, int64_t n)
{
    const NsWays w = ns_ways(b, m, n);
    for (const NsChoice& c : {w.gram, w.poly, w.step}) printf("%d %d ", ns_shapes[c.shape].size, c.splits > 1);
    printf("\n");
}
int main()
{
    for (auto& s : sizes) tell(s[0], s[1], s[2]);
    for (int i = 0; i < 20000; ++i) {
        const int64_t m = 65 + (int64_t)std::exp(8.5 * rnd()), n = m + (int64_t)std::exp(10.5 * rnd()), b = rnd() < 0.5 ? 1 : 1 + (int64_t)std::exp(4.0 * rnd());
        tell(b, m, n);
    }
}
""")
    ways = [tuple((int(v[i]), v[i + 1] == "1") for i in (0, 2, 4)) for v in (line.split() for line in out.splitlines())]
    assert dict(zip(WAYS, ways)) == WAYS
    for kind in range(3):
        assert {w[kind] for w in WAYS.values()} == PICKED[kind]
        assert {w[kind] for w in ways} <= PICKED[kind]
