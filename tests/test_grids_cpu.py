"""Grids past one dimension, and the sizes that are refused before anything is enqueued."""
import os
import subprocess

from paper_2609_26425_amd import quantwm as qw
from test_streaming_abi_cpu import _cfg, _shared

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_26425_amd", "csrc")


def test_rows_of_workgroups_cover_every_one(tmp_path):
    """csrc/grid_rows.h, compiled with the host's compiler: every workgroup has its place, at
    most a row of them has none, and no dimension passes 2^32 threads (of 256) or 2^16 rows."""
    src = tmp_path / "grid.c"
    src.write_text(r"""
#include <stdio.h>
#include "grid_rows.h"
int main(void) {
  const int64_t most = INT64_C(0x7fff0000);
  for (int64_t n = 1; n <= most; n = n < 300000 ? n + 1 : n + n / 1000 + 1) {
    const uint64_t x = qwm_grid_x(n), y = qwm_grid_y(n);
    if (x * y < (uint64_t)n || x * (y - 1) >= (uint64_t)n || x * 256 >= (UINT64_C(1) << 32) || y > 65535) {
      printf("%lld: %llu x %llu\n", (long long)n, (unsigned long long)x, (unsigned long long)y);
      return 1;
    }
  }
  return qwm_grid_x(most) * (uint64_t)qwm_grid_y(most) < (uint64_t)most;
}
""")
    exe = tmp_path / "grid"
    subprocess.run(["gcc", "-O2", "-std=c11", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


def test_shared_refuses_more_rows_than_a_join_counts():
    pcfg, cfg = _cfg(heads=1 << 10), _cfg(heads=1 << 10, batch=3)
    n_q = 0x7fff0000 // 3 // 1024
    size = lambda n: qw.quantwm_attend_shared_workspace_bytes(pcfg, 500, cfg, 100, 0, n)  # noqa: E731
    assert size(n_q) > 0 and size(n_q + 1) == 0
    assert _shared(pcfg=pcfg, cfg=cfg, n_q=n_q + 1) == qw.ERR_UNSUPPORTED
    assert "Queries" in qw.quantwm_last_error()


def test_shared_refuses_batches_past_the_tiles_grid():
    """Rollouts and heads are grid dimensions of the tiled kernel (33 Queries and more): refused
    before the prefix pass is enqueued."""
    for pcfg, cfg in ((_cfg(heads=1), _cfg(heads=1, batch=70_000)), (_cfg(heads=70_000), _cfg(heads=70_000))):
        assert _shared(pcfg=pcfg, cfg=cfg, n_q=33, nb=1 << 50) == qw.ERR_UNSUPPORTED
        assert "65536" in qw.quantwm_last_error()
