"""What the prefix kernel's hand-over of registers rests on: the compiler gives a kernel with setmaxnreg the most registers that its launch bounds allow, even if
it needs fewer (the library refuses to launch one that has fewer)."""
import os
import re
import subprocess

import pytest

from paper_2407_20143_b200 import build

KERNEL = """
__global__ void __launch_bounds__(THREADS, 1) split(int* p) {
  if (threadIdx.x < 512) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %d;");
    p[threadIdx.x] = 1;
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
  }
}
"""


def used(tmp_path, threads, more):
    source = tmp_path / "split.cu"
    source.write_text((KERNEL % more).replace("THREADS", str(threads)))
    r = subprocess.run([build.nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-Xptxas", "-v", "-c", str(source), "-o", str(tmp_path / "split.o")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return int(re.search(r"Used (\d+) registers", r.stdout + r.stderr).group(1))


def test_the_numbers_are_those_of_the_kernel():
    with open(os.path.join(build.CSRC, "kv_prefix.cu")) as f:
        source = f.read()
    assert "REGS = quant ? 72 : 80, REGS_ROWS = quant ? 80 : 88" in source and "LOADERS = quant && STREAMS == 2 ? 8 : 4" in source


@pytest.mark.parametrize("threads,at_launch,more", [(768, 80, 88), (896, 72, 80)])  # 16-bit caches, 8-bit caches
def test_a_kernel_that_hands_on_registers_has_the_most_of_its_launch_bounds(tmp_path, threads, at_launch, more):
    assert used(tmp_path, threads, more) == at_launch == 65536 // threads // 8 * 8
