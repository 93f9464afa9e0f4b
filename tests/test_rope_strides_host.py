"""Head strides of rotary rows that take more than 31 bits in bytes: what the host hands to the kernels, compiled here with the library's own
source and looked at without a GPU."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_25385_amd", "csrc")
# (rope.hip needs two functions of other files to link; nothing here calls them)
DRIVER = r"""
#include <cstdio>
#include "rope.hip"
namespace glowq {
glowq_status hip_status(hipError_t) { return GLOWQ_OK; }
glowq_status kv_check_rows(const glowq_kv_cache*, const void*, int, const void*, int, const int32_t*, int) { return GLOWQ_OK; }
}
int main() {
  int bad = 0;
  for (int dtype : {GLOWQ_F16, GLOWQ_BF16, GLOWQ_F32}) {
    const long long size = dtype == GLOWQ_F32 ? 4 : 2;
    for (int lh : {128, (1 << 29) - 8, 1 << 29, (1 << 30) - 8, 1 << 30, 0x7fffffff - 255}) {
      const glowq_rope rope = {(const uint64_t*)64, 128, GLOWQ_ROPE_HALVES, 1.f};
      const glowq_rope_rows rows = {(const void*)64, (void*)4096, 2, lh + 128, lh, lh + 128, lh};
      if (glowq::check_rope_rows(&rows, 1, 128, dtype) != GLOWQ_OK) { printf("refused: dtype %d, %d apart\n", dtype, lh); bad = 1; continue; }
      long long threads;
      const glowq::RotateArgs a = glowq::make_rotate_args(rope, &rows, 1, 128, dtype, (const int32_t*)64, 3, &threads);
      const long long x = a.t[0].lhx, y = a.t[0].lhy;
      if (x != lh * size || y != lh * size) { printf("dtype %d, heads %d apart: %lld and %lld bytes, not %lld\n", dtype, lh, x, y, lh * size); bad = 1; }
      if (a.t[0].ldx != (lh + 128) * size || a.t[0].ldy != (lh + 128) * size) { printf("rows: %lld, %lld\n", a.t[0].ldx, a.t[0].ldy); bad = 1; }
    }
  }
  puts(bad ? "wrong" : "strides right");
  return bad;
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")
def test_head_strides_in_bytes(tmp_path):
    source, exe = tmp_path / "strides.hip", str(tmp_path / "strides")
    source.write_text(DRIVER)
    p = subprocess.run(["hipcc", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", CSRC,
                        str(source), "-o", exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout[-4000:]
    p = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0 and "strides right" in p.stdout, p.stdout
