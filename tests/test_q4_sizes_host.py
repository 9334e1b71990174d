"""Workspace sizes of calls over a 4-bit cache, without a GPU."""
import os
import subprocess
import sys

from ctypes import byref as by

import pytest

from paper_2604_10044_gb300 import lg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# in a process of its own: a size that divides by zero ends it
CHUNK = r"""
import sys
from ctypes import byref as by
from paper_2604_10044_gb300 import lg
F = 1 << 20
c = lg.LgCache(k=F, v=F, dtype=int(sys.argv[1]), L=2, H_kv=8, d=128, batch=2, S_total=64, seq_off=F, cap=F,
               len=F, sketch=F, dev_status=F)
L = lg.lib()
for H_q in (8, 24, 64):
    for T, max_len in ((0, 1), (0, 64), (7, 4096)):
        ch = lg.LgChunk(off=F, T=T, max_new=0)
        print(L.lg_chunk_workspace_size(by(c), by(ch), H_q, max_len),
              L.lg_chunk_attend(by(c), by(ch), 0, None, H_q, 0.1, 0, 0, None, max_len, None, 0, None))
"""


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_a_chunk_of_no_new_rows_has_a_size(dtype):
    """every sequence rests: a size as for any other step, and a call that does nothing"""
    r = subprocess.run([sys.executable, "-c", CHUNK, str(dtype)], cwd=ROOT, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, (r.returncode, r.stderr)
    got = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
    assert len(got) == 9
    assert all(size > 0 and size % 256 == 0 and status == 0 for size, status in got), got


@pytest.mark.parametrize("H_q", [8, 32, 64])
def test_a_decode_of_many_layers_fits_the_gpu_at_once(H_q):
    """single tokens: 152 SMs hold three CTAs each, whose shares are equal, so one more would be a wave of
    its own; the workspace has two tiles of eight rows and a record a CTA"""
    F, a_cta, resident = 1 << 20, 2 * 8 * (128 + 4) * 4 + 40, 3 * 152
    for L in list(range(1, 130)) + [151, 152, 153, 227, 228, 229, 455, 456]:
        c = lg.LgCache(k=F, v=F, dtype=lg.LG_Q4, L=L, H_kv=8, d=128, batch=64, S_total=64 * 16384, seq_off=F,
                       cap=F, len=F, dev_status=F)
        n = lg.lib().lg_workspace_size(by(c), H_q, L, 16384, 0) // a_cta
        assert resident // 2 <= n <= resident, (L, n)
        assert n % L == 0 and n + L > resident, (L, n)
