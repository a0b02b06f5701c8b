"""The rule that chooses a kernel for the 8-bit products (host-only C++) under the sanitizers, and that the sizes of the GPU tests reach
every kernel that it can choose.  No GPU, no HIP."""
import os
import subprocess

from tests.test_e4m3_shapes import FEW, GATED, K, PLAIN
from tests.test_sanitizers import ENV, HERE, SAN


def test_sizes_of_the_tests_reach_every_kernel(tmp_path):
    exe = str(tmp_path / "driver")
    subprocess.check_call(["g++", "-std=c++17"] + SAN + [os.path.join(HERE, "sanitize", "e4m3_plan_driver.cpp"), "-o", exe])

    def kernels(word, *args):
        proc = subprocess.run([exe, *map(str, args)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=ENV, timeout=600)
        lines = proc.stdout.strip().splitlines()
        assert proc.returncode == 0 and lines[-1] == "ok", proc.stdout[-4000:]
        return {l[len(word) + 1:] for l in lines if l.startswith(word + " ")}
    can = kernels("can")
    takes = kernels("takes", *(v for gated, sizes in ((0, PLAIN + FEW), (1, GATED + FEW)) for M, N in sizes for v in (gated, M, N)))
    assert takes == can, (sorted(can - takes), sorted(takes - can))
    assert len(can) >= 30 and not any("exact 256x128" in k for k in can)
    assert K % 128 and K // 128 >= 9                       # several turns of four steps, the last one a part
