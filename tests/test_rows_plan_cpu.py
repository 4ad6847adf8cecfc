"""How rows are dealt to threads (rows_plan.h): every unit has a thread, work-groups fit, the backward pass's work-groups have every row and fit the CUs at once."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2006_06762_amd", "csrc")


def test_plans(tmp_path):
    (tmp_path / "plan.cpp").write_text("""
#include <cstdio>
#include <initializer_list>
#include "rows_plan.h"
using namespace anr::rows;
#define CHECK(c) do { if (!(c)) { printf("%s: V %d C %d T %ld\\n", #c, V, C, (long)T); return 1; } } while (0)
int main()
{
    const int64_t rows[] = {1, 2, 3, 63, 64, 65, 100, 1023, 1024, 1025, 5003, 1 << 20, ((int64_t)1 << 31) - 1};
    for (int V : {1, 4, 8})
        for (int C = V == 1 ? 1 : V; C <= (V == 1 ? 7 : kHeldBy1024); C += C < 3000 ? 1 : 37)
            for (int64_t T : rows) {
                const int most = kHeld / V;
                const int64_t units = (C + V - 1) / V;
                auto fits = [&](const Plan& p) {
                    const bool power = (p.units & (p.units - 1)) == 0, lanes = p.threads == 8 || p.threads == 16 || p.threads == 32 || p.threads % 64 == 0;
                    return power && p.units >= 1 && p.units <= most && lanes && p.rows >= 1 && p.threads * p.rows <= kMostThreads && p.threads * p.rows % 64 == 0 &&
                           (int64_t)p.threads * p.units >= units;
                };
                const Plan f = plan_of(units, most, T);
                CHECK(fits(f));
                // (a row's number is then a scalar of its waves)
                CHECK(f.units <= 2 || f.threads % 64 == 0);
                const BackwardPlan b = backward_plan_of(units, most, T);
                CHECK(fits(b.rows));
                CHECK(b.rows.units == 1 || b.rows.threads % 64 == 0);
                // (a thread that keeps more than 16 sums has them in LDS, 128 KB, for one row at a time; rows of a work-group are joined in LDS)
                CHECK(b.rows.units * V <= 16 || b.rows.rows == 1);
                CHECK(b.rows.rows == 1 || (int64_t)b.rows.rows * C * 4 <= 65536);
                CHECK(b.lines >= 1 && b.lines <= (T + b.rows.rows - 1) / b.rows.rows);
                CHECK(b.lines * b.rows.threads * b.rows.rows <= 256 * 2048);
            }
    return 0;
}
""")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-I", CSRC, str(tmp_path / "plan.cpp"), "-o", str(tmp_path / "plan")], check=True)
    ran = subprocess.run([str(tmp_path / "plan")], capture_output=True, text=True)
    assert ran.returncode == 0, ran.stdout
