"""The power table of the draws' pass over the logits, on the host: whatever the scale and
the base, every logit that is added without moving the base has its weight in a cell
of the table, and that cell is its weight's."""
import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cfloat>
#include <cstdio>

#include "cpes_powers.hpp"

using namespace cpes;

int main()
{
    long seen = 0, outside = 0, far = 0, infinite = 0;
    for (int s = -160; s <= 151; ++s)
        for (int b = -400; b <= 507; ++b)
            for (int sign = -1; sign <= 1; sign += 2) {
                const float scale = (float)pow(10.0, s / 4.0), base = sign * (float)pow(2.0, b / 4.0);
                if (!(scale > 0.f) || !(scale <= FLT_MAX / 2)) continue;
                const double c = (double)scale * M_LOG2E, cells = c * kCells, start = start_of(base, cells);
                const float last = last_above(base, c);
                infinite += !(last <= FLT_MAX) || last < base;
                auto look = [&](float x) {
                    if (!(x <= last)) return;
                    const double t = start_is_near(start) ? cells_near(x, cells, start) : cells_far(x, base, cells);
                    ++seen;
                    outside += !(t < kPowers);
                    // the octaves above the first cell, in doubles that hold the difference
                    const double octaves = ((double)x - (double)base) * c - kLow;
                    far += octaves >= 0 && fabs(t / kCells - octaves) > 1e-9 * fmax(1.0, fabs(octaves));
                };
                float x = base;
                for (int ulps = 0; ulps < 12; ++ulps, x = nextafterf(x, INFINITY)) look(x);
                x = last;
                for (int ulps = 0; ulps < 4; ++ulps, x = nextafterf(x, -INFINITY)) look(x);
            }
    printf("%ld %ld %ld %ld\n", seen, outside, far, infinite);
}
"""


def test_every_weight_lies_in_the_table(tmp_path):
    gxx = shutil.which("g++")
    assert gxx is not None
    (tmp_path / "p.cpp").write_text(PROGRAM)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run([gxx, "-std=c++17", "-O1", "-ffp-contract=off", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-I",
                    os.path.join(ROOT, "paper_2608_02391_amd", "csrc"), "-o", str(tmp_path / "p"), str(tmp_path / "p.cpp")], check=True)
    out = subprocess.run([str(tmp_path / "p")], capture_output=True, text=True, check=True).stdout.split()
    seen, outside, far, infinite = map(int, out)
    assert seen > 1000000
    assert (outside, far, infinite) == (0, 0, 0)
