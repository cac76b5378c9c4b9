"""The gated block's plans (csrc/da_gated_plan.h) on the host: every product that a backward pass may launch has room for
its parts in the workspace that the call reports, whichever gradients are asked for."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2202_08556_amd", "csrc")

PROGRAM = r"""
#include "da_gated_plan.h"
#include <cstdio>
#include <vector>
static int units = 256;
namespace daspmm { int compute_units() noexcept { return units; } }
using namespace daspmm;

// bytes of the parts that a launch of a product writes, by either kernel
static size_t written(const Product& g, int splits) {
    return splits > 1 ? (size_t)g.batches * splits * g.M * g.N * (g.epi == kGate ? 2 : 1) * 4 : 0;
}
static size_t needs(const Product& g, int size) {
    if (g.M == 0 || g.N == 0) return 0;
    size_t most = written(g, gemm_plan(g, size).splits);
    if (size == 2) {
        const WidePlan w = wide_plan(g);
        if (w.rows) {
            const int64_t step = w.rows == 256 ? 64 : 32, inner = ceil_div(g.K, step) * g.segments;
            const int64_t per = std::max<int64_t>(1, ceil_div(inner, w.splits));
            most = std::max(most, written(g, (int)std::max<int64_t>(1, ceil_div(inner, per))));
        }
    }
    return most;
}

int main() {
    const std::vector<int64_t> rows = {1, 5, 9, 16, 17, 40, 64, 79, 128, 129, 300, 1000, 1531, 4096, 8192, 20003, 100003, 1000000},
                               widths = {1, 7, 16, 41, 64, 100, 128, 216, 257, 602, 768, 1024, 1187, 2048, 4096, 9560, 12288},
                               outs = {1, 7, 64, 216, 1024, 4096};
    long checked = 0;
    for (int u : {256, 304, 80, 1}) {
        units = u;
        for (int size : {4, 2}) for (int64_t r : rows) for (int64_t d : widths) for (int64_t h : widths) for (int64_t o : outs) {
            const GatedShape s{r, d, h, o};
            const size_t room = backward_part_bytes(s, size);
            const Product launched[] = {hidden_grad_product(s), input_grad_product(s), up_grad_product(s, 1), up_grad_product(s, 2),
                                        down_grad_product(s)};
            for (const Product& g : launched) {
                ++checked;
                if (needs(g, size) > room) {
                    std::printf("units %d size %d rows %ld d %ld h %ld dout %ld: product %ld x %ld x %ld, %d at once, writes %zu of %zu bytes\n",
                                u, size, (long)r, (long)d, (long)h, (long)o, (long)g.M, (long)g.N, (long)g.K, g.batches, needs(g, size), room);
                    return 1;
                }
            }
            if (std::max(needs(gate_product(s), size), needs(down_product(s), size)) >
                std::max(part_bytes(gate_product(s), size), part_bytes(down_product(s), size)))
                return std::printf("forward\n"), 1;
        }
    }
    std::printf("%ld products\n", checked);
    return 0;
}
"""


def test_every_launch_fits_its_workspace(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    source, program = tmp_path / "plan.cpp", tmp_path / "plan"
    source.write_text(PROGRAM)
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-I" + CSRC, str(source), "-o", str(program)], check=True)
    res = subprocess.run([str(program)], stdout=subprocess.PIPE, text=True)
    assert res.returncode == 0, res.stdout


# rows, d, h, d_out and the parts of the gradient of one of w_gate and w_up: the product d x h takes 256 tiles, one for each unit,
# and its sum over the rows is cut in two
@pytest.mark.parametrize("dtype", [0, 1])
def test_workspace_of_one_weights_gradient(dtype):
    lib = ctypes.CDLL(os.path.join(ROOT, "paper_2202_08556_amd", "libdaspmm.so"))
    forward, backward = ctypes.c_size_t(), ctypes.c_size_t()
    rows, d, h, dout = 8192, 1024, 4096, 7
    assert lib.da_gated_workspace(dtype, *map(ctypes.c_int64, (rows, d, h, dout)), ctypes.byref(forward), ctypes.byref(backward)) == 0
    hidden = 2 * rows * h * (4 if dtype == 0 else 2)
    assert backward.value - hidden >= 2 * d * h * 4


THREADS = r"""
#include "da_gated_plan.h"
#include <cstdio>
#include <cstdlib>
namespace daspmm { int compute_units() noexcept { return 256; } }
using namespace daspmm;

static int64_t threads(const Product& g, int size) {
    if (g.M == 0 || g.N == 0) return 0;
    const int64_t width = g.epi == kGate ? 2 * g.N : g.N;
    const GemmPlan p = gemm_plan(g, size);
    int64_t most = ceil_div(g.M, p.BM) * ceil_div(width, p.BN) * (p.BM == 128 && p.BN == 128 ? 512 : 256);
    const WidePlan w = wide_plan(g);
    if (size == 2 && w.rows) most = std::max(most, ceil_div(g.M, w.rows) * ceil_div(width, kWideColumns) * 2 * w.rows);
    return most;
}

int main(int argc, char** argv) {
    for (int i = 1; i + 3 < argc; i += 4) {
        const GatedShape s{std::atoll(argv[i]), std::atoll(argv[i + 1]), std::atoll(argv[i + 2]), std::atoll(argv[i + 3])};
        for (int size : {4, 2})
            for (const Product& g : {gate_product(s), down_product(s), hidden_grad_product(s), input_grad_product(s), up_grad_product(s, 1),
                                     up_grad_product(s, 2), down_grad_product(s)})
                if (threads(g, size) >= 1LL << 32) {
                    std::printf("rows %ld d %ld h %ld dout %ld: %ld threads side by side\n", (long)s.rows, (long)s.d, (long)s.h, (long)s.dout,
                                (long)threads(g, size));
                    return 1;
                }
    }
    return 0;
}
"""


def test_accepted_sizes_are_no_more_threads_than_a_launch_counts(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    source, program = tmp_path / "threads.cpp", tmp_path / "threads"
    source.write_text(THREADS)
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-I" + CSRC, str(source), "-o", str(program)], check=True)
    lib = ctypes.CDLL(os.path.join(ROOT, "paper_2202_08556_amd", "libdaspmm.so"))
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    sizes = (1, 9, 32, 33, 64, 65, 129, 2 ** 20, 2 ** 24, 2 ** 29, 2 ** 29 + 1, 2 ** 30 - 128, 2 ** 30 - 63, 2 ** 30)
    accepted = [s for s in ((r, d, h, o) for r in sizes for d in sizes for h in sizes for o in sizes)
                if lib.da_gated_workspace(0, *map(ctypes.c_int64, s), ctypes.byref(a), ctypes.byref(b)) == 0]
    assert (2 ** 30 - 128, 1, 1, 1) in accepted and len(accepted) > 1000
    for i in range(0, len(accepted), 2000):
        res = subprocess.run([str(program), *(str(n) for s in accepted[i:i + 2000] for n in s)], stdout=subprocess.PIPE, text=True)
        assert res.returncode == 0, res.stdout
