"""The grids of the paged cache's launches: every workgroup once, no x dimension of 2^32 threads (on the host)."""
import subprocess

import pytest

from paper_2608_15665_amd import _build

CHECK = r"""
#include "zo_kv.h"
#include <stdio.h>
void zo_set_error(const char*, ...) {}
int main() {
  const long long all[] = {1, 7, 511, 1 << 22, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, 18900000, (1 << 30) + 5, 0x7fffffffLL};
  for (long long n : all) {
    const dim3 g = kv_grid(n);
    const long long x = g.x, y = g.y, last = (x - 1) + ((y - 1) << 22);  // kv_block of the last workgroup
    if (x * 256 >= 1LL << 32 || y > 65535 || g.z != 1) return printf("%lld: %lld x %lld\n", n, x, y), 1;
    if (last < n - 1 || last > 0xffffffffLL || (y > 1 && x != 1 << 22)) return printf("%lld: last %lld\n", n, last), 1;
  }
  return 0;
}
"""


def test_grids(tmp_path):
    try:
        cc = _build.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    src, exe = tmp_path / "check.hip", str(tmp_path / "check")
    src.write_text(CHECK)
    p = subprocess.run([cc, "--offload-host-only", "-O1", "-std=c++17", f"-I{_build.INCLUDE}", f"-I{_build.CSRC}", str(src), "-o", exe],
                       capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-2000:]
    p = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert p.returncode == 0, p.stdout
