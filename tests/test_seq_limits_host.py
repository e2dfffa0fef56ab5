"""The sizes that linattn.h allows for linattn_rotary and linattn_decay_*: the last of them is taken, the next refused; and grids that hold them."""
import os
import shutil
import subprocess

import pytest

from paper_2510_08318_amd import binding as L
from tests.test_seq_host import _decay, _rotary

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


# (a call without tensors is refused for them, once its sizes are taken)
@pytest.mark.parametrize("size,status", [
    (dict(B=2047, H=32, HK=32, n=1), "E_NULL"), (dict(B=2048, H=32, HK=32, n=1), "E_SHAPE"), (dict(B=1, H=65535, HK=1, n=1), "E_NULL"),
    (dict(B=1, H=65536, HK=1, n=1), "E_SHAPE"), (dict(B=1, H=1, HK=1, n=1 << 30), "E_NULL"), (dict(B=1, H=1, HK=1, n=(1 << 30) + 1), "E_SHAPE"),
    (dict(B=32, H=1, HK=1, n=1 << 30), "E_NULL"), (dict(B=33, H=1, HK=1, n=1 << 30), "E_SHAPE"), (dict(B=1, H=32, HK=1, n=1 << 30), "E_NULL"),
    (dict(B=1, H=33, HK=1, n=1 << 30), "E_SHAPE")])
def test_sizes_at_the_limits(size, status):
    assert L.linattn_rotary(_rotary(**size), None, None, None, None, check=False) == getattr(L, status)
    assert L.linattn_decay_fwd(_decay(**size), *[None] * 6, check=False) == getattr(L, status)
    assert L.linattn_decay_bwd(_decay(**size), *[None] * 10, check=False) == getattr(L, status)


def test_rotary_s_key_heads_have_the_same_limit():
    P = 1 << 40
    call = lambda HK: L.linattn_rotary(_rotary(B=1, H=1, HK=HK, n=1, dims=(32, 16, 0x7ffe)), P, P, P, P, check=False)
    assert call(65536) == L.E_SHAPE
    assert L.linattn_rotary(_rotary(B=1, H=1, HK=65535, n=1), None, P, None, P, check=False) == L.E_NULL
    assert L.linattn_rotary(_rotary(B=1, H=1, HK=65536, n=1), None, P, None, P, check=False) == L.E_SHAPE
    assert L.linattn_rotary(_rotary(B=1, H=1, HK=65536, n=1), None, None, None, None, check=False) == L.E_NULL


PROGRAM = r"""
#include "decay.h"
#include "rotary.h"
#include <cstdio>
using namespace linattn;
static long long bad = 0;
static void rotary_grid(long long blocks) {
  for (int groups : {1, 2, 1024}) {
    const dim3 g = rotary::grid_of(blocks, groups);
    const long long all = (long long)g.x * g.z;
    bad += (unsigned long long)g.x * 256 >= 1ull << 32 || g.y != (unsigned)groups || g.z > 65535 || g.x < 1 || all < blocks || all - blocks >= g.x;
  }
}
int main() {
  for (long long b = 1; b <= 1ll << 32; b *= 2)
    for (long long d = -1; d <= 1; ++d)
      if (b + d >= 1) rotary_grid(b + d);
  unsigned long long x = 12345;
  for (int b = 1; b < 2000; ++b) {
    x = x * 6364136223846793005ull + 1442695040888963407ull;
    rotary_grid((long long)((x >> 20) % (1ull << (1 + b % 32))) + 1);
  }
  // the decay kernels have a workgroup to a segment of a pass of a query head in grid.x, the states between them B * H in grid.y, 256 threads each
  const int heads[] = {1, 2, 3, 12, 40, 255, 256, 257, 511, 1000, 4096, 10000, 32768, 65535};
  const int tokens[] = {9, 17, 64, 65, 1000, 4133, 32760, 75600, 1 << 20, (1 << 25) + 1, 1 << 30};
  for (int h : heads)
    for (int n : tokens)
      for (int d : {64, 128})
        for (int back = 0; back < 2; ++back)
          for (int kind = 0; kind < 3; ++kind) {
            if ((long long)h * n > 1ll << 35) continue;
            const auto t = decay::chunk_times(kind == 1, kind == 2, d);
            const auto p = decay::plan_of(1, h, n, t, d, back ? 3 : 1, back ? 2 : 1);
            bad += p.segs < 1 || p.segs > 256 || p.tokens < 1 || p.tokens % t.chunk || (long long)p.segs * p.tokens < n || (long long)(p.segs - 1) * p.tokens >= n;
            bad += (unsigned long long)h * p.segs * (back ? 3 : 1) * 256 >= 1ull << 32;
            bad += (long long)(p.segs - 1) * p.tokens + 2ll * p.tokens > (p.segs > 1 ? 0x7fffffffll : 0x80000000ll);
          }
  printf("bad %lld\n", bad);
  return bad != 0;
}
"""


@pytest.mark.skipif(not shutil.which(os.path.join(ROCM, "bin", "hipcc")), reason="needs hipcc")
def test_grids(tmp_path):
    (tmp_path / "t.cpp").write_text(PROGRAM)
    subprocess.run([os.path.join(ROCM, "bin", "hipcc"), "-x", "hip", "--offload-arch=gfx950", "-O1", "-std=c++17", "-w", "-I", os.path.join(ROOT, "paper_2510_08318_amd", "csrc"),
                    str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    run = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout
