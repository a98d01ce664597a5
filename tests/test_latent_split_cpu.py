"""The work split at the sizes that latent attention admits (csrc/attn_sched.hpp, compiled for the host): lines of up to 2^30 granules, hundreds of thousands of units."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

PROGRAM = r"""
#include "attn_sched.hpp"
#include <limits.h>
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
using namespace sx;
static long checked = 0, bad = 0;
static void line(long gran, long B, long blocks, int wgrid) {
  const long bare = gran * blocks, T = bare + (bare > kAttnSpread ? 2 * B * blocks : 0);
  if (T >= 1l << 30) return;
  ++checked;
  const AttnLine l = attn_sched_line(gran, B, blocks, 2, INT_MAX, 0, wgrid);
  const long W = l.W, use = wgrid < kAttnSpread ? wgrid : kAttnSpread, most = (T + use - 1) / use;
  bool ok = l.T == T && W >= 1 && W <= wgrid && W <= T && l.q == T / W && l.r == T % W;
  // no share above what all workgroups would have
  if (bare > kAttnSpread && wgrid >= kAttnSpread) ok = ok && W <= kAttnSpread && (T + W - 1) / W == most;
  if (T >= 1l << 17) ok = ok && W == use;
  ok = ok && attn_sched_lo(l, 0) == 0 && attn_sched_lo(l, W) == T && attn_sched_lo(l, W / 2) == W / 2 * T / W;
  if (!ok && ++bad < 10) printf("%ld granules of %ld sequences, %ld blocks, grid %d: %ld workgroups of %ld granules, %d and %d\n", gran, B, blocks, wgrid, W, T, l.q, l.r);
}
static double uniform() { return (rand() % 100003 + 0.5) / 100003.0; }
static long spread(double lo, double hi) { return static_cast<long>(lo * exp(uniform() * log(hi / lo))); }

int main() {
  srand(3);
  line(512 * 600, 512, 64, 256);             // 512 sequences of 38400 entries, 8192 rows each
  line(256 * 2048, 256, 64, 256);            // 256 of 131072
  line(1024, 1024, 256, 256);
  for (int k = 0; k < 2000000; ++k) {
    const long B = spread(1, 1025), blocks = spread(1, 257), gran = spread(B, 2.0e9 / blocks);
    line(gran, B, blocks, k % 4 ? 256 : 304);
  }
  printf("%ld checks, %ld wrong\n", checked, bad);
  return bad != 0;
}
"""


@pytest.mark.skipif(not shutil.which(HIPCC), reason="no hipcc")
def test_lines_up_to_the_plans_limit(tmp_path):
    src = tmp_path / "line.hip"
    src.write_text(PROGRAM)
    exe = tmp_path / "line"
    subprocess.run([HIPCC, "-O2", "-std=c++17", "--offload-arch=gfx950", "--offload-host-only", "-I", os.path.join(ROOT, "paper_2509_24248_amd", "csrc"),
                    str(src), "-o", str(exe)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0, run.stdout
    assert int(run.stdout.split()[0]) > 1_000_000
