"""Plans of packed products (csrc/da_planes_plan.h) on the host: within the limits that the calls state, no launch has 2^32 threads or more
along an axis, and a tile's parts cover the inner axis once."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2202_08556_amd", "csrc")

PROGRAM = r"""
#include "da_planes_plan.h"
#include <cmath>
#include <cstdio>
#include <random>
static int units = 256;
namespace daspmm { int compute_units() noexcept { return units; } }
using namespace daspmm;

static int64_t pad(int64_t n) { return ceil_div(n, 64) * 64; }
static long checked = 0;

static bool good(int64_t Ma, int64_t Nb, int64_t steps, int64_t batches, bool symmetric, bool may_split, int halves) {
    const PlanePlan p = plane_plan(Ma, Nb, steps, batches, symmetric, may_split, halves);
    const int64_t side = p.shape == 0 ? 256 : p.shape == 1 ? 128 : 64, threads = p.shape == 0 ? 512 : 256;
    const int64_t m = ceil_div(Ma, side), n = ceil_div(Nb, side);
    ++checked;
    const bool ok = p.tiles == (symmetric ? m * (m + 1) / 2 : m * n) && p.tiles_m == m && p.tiles_n == n && p.tiles * threads < 1LL << 32 &&
                    p.splits >= 1 && p.splits <= 1024 && (p.splits == 1 || (may_split && p.tiles * batches <= kMostParted)) &&
                    (int64_t)p.splits * p.per >= steps && (int64_t)(p.splits - 1) * p.per < std::max<int64_t>(steps, 1);
    if (!ok)
        std::printf("%ld x %ld, %ld steps, %ld batches, symmetric %d, halves %d: shape %d, %ld tiles, %.3f of 2^32 threads, %d parts of %d\n", (long)Ma,
                    (long)Nb, (long)steps, (long)batches, symmetric, halves, p.shape, (long)p.tiles, (double)(p.tiles * threads) / 4294967296.0,
                    p.splits, p.per);
    return ok;
}

int main() {
    std::mt19937_64 rng(1);
    auto draw = [&](double lo, double hi) { return (int64_t)std::llround(std::exp(std::uniform_real_distribution<>(std::log(lo), std::log(hi))(rng))); };
    bool ok = true;
    for (int u : {256, 304, 80}) {
        units = u;
        for (long found = 0; found < 20000;) {               // the cross entropy's products
            const int64_t rows = draw(17, 1 << 26), d = draw(1, 1 << 22), V = draw(65, 1 << 22);
            const int64_t m = ceil_div(rows, 256), n = ceil_div(d, 256), v = ceil_div(V, 256);
            if (std::max({m * v, m * n, n * v}) >= 1 << 23) continue;
            ++found;
            for (int halves = 0; halves < 2; ++halves) {
                const int64_t step = halves ? 32 : 64, Ma = pad(rows), D = pad(d);
                const int64_t piece = std::min(V, std::max<int64_t>(1024, (512LL << 20) / (Ma * 2 * (halves + 1)) / 256 * 256));
                for (int64_t w : {V, piece}) {
                    ok = good(Ma, pad(w), D / step, 1, false, false, halves) && ok;
                    ok = good(Ma, D, pad(w) / step, 1, false, true, halves) && ok;
                    ok = good(D, pad(w), Ma / step, 1, false, true, halves) && ok;
                }
                if (!ok) return 1;
            }
        }
        for (long found = 0; found < 5000;) {                // the orthogonalised updates'
            const int64_t a = draw(1, 1 << 17), b = draw(1, 1 << 17), batch = draw(1, 65535);
            if (batch * ceil_div(a, 64) * ceil_div(b, 64) >= 1LL << 30) continue;
            ++found;
            const int64_t m = pad(std::min(a, b)), n = pad(std::max(a, b));
            ok = good(m, m, n / 32, batch, true, true, 1) && good(m, m, m / 32, batch, true, true, 1) && good(m, n, m / 32, batch, false, true, 1) && ok;
            if (!ok) return 1;
        }
    }
    std::printf("%ld plans\n", checked);
    return 0;
}
"""


def test_every_launch_is_one_that_the_device_takes(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    source, program = tmp_path / "plan.cpp", tmp_path / "plan"
    source.write_text(PROGRAM)
    subprocess.run([gxx, "-O2", "-std=c++17", "-Wall", "-Werror", "-I" + CSRC, str(source), "-o", str(program)], check=True)
    res = subprocess.run([str(program)], stdout=subprocess.PIPE, text=True)
    assert res.returncode == 0, res.stdout
