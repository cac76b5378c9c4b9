"""Host side of the training step's operators, without a GPU: what the built library holds."""
import os
import re
import subprocess

from paper_2202_08556_amd import binding as da

PKG = os.path.dirname(os.path.abspath(da.__file__))


def test_every_kernel_has_a_flag_of_its_own():
    """Dynamic LDS beyond 64 KB is allowed kernel by kernel: one kernel's flag must not stand for another of the same signature."""
    names = [line.split()[-1] for line in subprocess.run(["nm", os.path.join(PKG, "libdaspmm.so")], capture_output=True, text=True, check=True).stdout.splitlines()]
    flags = [n for n in names if n.startswith("_ZZN6daspmm") and n.endswith("7allowed")]
    for kernel in ("16ce_narrow_kernel", "12plane_kernel", "17orth_small_kernel"):
        kernels = {n for n in names if re.match(r"_ZN6daspmm(12_GLOBAL__N_1)?" + kernel, n)}
        assert len(kernels) >= 2
        mine = [n for n in flags if "allow_lds" in n and kernel in n]
        assert len(mine) == len(kernels), (kernel, len(mine), len(kernels))
