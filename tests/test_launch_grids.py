"""Launch grids of the operators on sequences: every workgroup is there, and no dimension has 2^32 threads or more, which a launch refuses (host-only: the
header's function, compiled without device code)."""
import os
import subprocess

import pytest

from paper_1912_05234_amd import build

CSRC = os.path.join(build.PKG, "csrc")
MOST_THREADS = 1024  # of a workgroup
COUNTS = [1, 2, 1000, (1 << 21) - 1, 1 << 21, (1 << 21) + 1, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, 4259840, (1 << 31) + 5, 1 << 36]

PROGRAM = """
#include "cnn_types.h"
#include <stdio.h>
int main() {
  long long n;
  while (scanf("%lld", &n) == 1) {
    const dim3 g = cnn::grid_of(n);
    printf("%u %u %u\\n", g.x, g.y, g.z);
  }
}
"""


@pytest.fixture(scope="module")
def grids(tmp_path_factory):
    source, program = (str(tmp_path_factory.mktemp("grids") / n) for n in ("grids.hip", "grids"))
    open(source, "w").write(PROGRAM)
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-host-only", "-std=c++17", "-I", os.path.join(build.ROOT, "include"), "-I", CSRC, source, "-o", program],
                   check=True, capture_output=True, text=True)
    out = subprocess.run([program], input="\n".join(map(str, COUNTS)), check=True, capture_output=True, text=True).stdout
    return dict(zip(COUNTS, (tuple(map(int, line.split())) for line in out.splitlines())))


@pytest.mark.parametrize("n", COUNTS)
def test_grid(grids, n):
    x, y, z = grids[n]
    assert x * y >= n and z == 1 and (x * (y - 1) < n)
    assert x * MOST_THREADS < 1 << 32 and y < 1 << 16
