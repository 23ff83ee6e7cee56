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


def test_a_block_of_the_append_never_stages_more_units_than_there_is_room_for(tmp_path):
    """Every division of a call that the plan can choose, over widths, d, T and numbers of SMs: the units that one CTA finishes."""
    out = run_host_program(tmp_path, r"""
#include "ta_append_umma.cuh"
#include <cstdio>
using namespace ta::append;
int main() {
  int most = 0;
  for (int sms : {1, 16, 132, 148, 160})
    for (int w0 = 32; w0 <= 256; w0 += 32)
      for (int w1 = 0; w1 <= 256; w1 += 32)
        for (int d : {64, 128, 768, 1024, 4096, 16384})
          for (int T = 1; T < 200000; T = T < 1000 ? T + 37 : T + T / 23) {
            const Plan q = append_plan(T, d, w0, w1, sms);
            for (int part = 0; part < (q.split_parts ? 2 : 1); ++part) {
              const int width = q.split_parts ? (part ? w1 : w0) : w0 + w1, units = q.MT * width / UC;
              for (int s = 0; s < q.S; ++s) {
                const int mine = units * (s + 1) / q.S - units * s / q.S;
                if (mine > MAX_UNITS || mine * STAGED_BYTES > RING_BYTES) { printf("T %d d %d %d/%d: %d units\n", T, d, w0, w1, mine); return 1; }
                most = mine > most ? mine : most;
              }
            }
          }
  return most == MAX_UNITS ? 0 : 2;
}
""")
    assert out == ""
