"""Host-callable parts of the paged kernels' headers, compiled into a small host program and run on the CPU."""
import os
import subprocess

from paper_2603_30033_b200 import build as Bu


def run_host_program(tmp_path, source):
    """Compiles `source` (a main that returns 0) against the kernels' headers and runs it; returns its output."""
    cu, exe = os.path.join(tmp_path, "prog.cu"), os.path.join(tmp_path, "prog")
    with open(cu, "w") as f:
        f.write(source)
    r = subprocess.run([Bu._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", Bu.INCLUDE, "-I", Bu.CSRC, cu, "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout


def test_a_note_of_the_streaming_kernel_that_was_never_written_is_no_index(tmp_path):
    """Whatever two words hold, the join reads partials of CTAs 0 .. grid - 1 only; every true note is taken as it is."""
    out = run_host_program(tmp_path, r"""
#include "ta_paged.cuh"
#include <climits>
#include <cstdio>
int main() {
  const int v[] = {INT_MIN, -1000000000, -2, -1, 0, 1, 2, 146, 147, 148, 149, 159, 160, 1000000, 0x3f800000, 0x7fc00000, INT_MAX};
  for (int grid : {1, 2, 148, 160})
    for (int first : v)
      for (int last : v) {
        const int n = ta::noted_parts(first, last, grid);
        const bool ok = first >= 0 && last >= first && last < grid;
        if (ok ? n != last - first + 1 : n != 0) { printf("%d %d %d: %d\n", first, last, grid, n); return 1; }
        if (n && (first < 0 || (long)first + n > grid)) return 2;
      }
  return 0;
}
""")
    assert out == ""
