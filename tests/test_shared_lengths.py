"""Lengths of attention over shared prefixes that do not belong together are
refused before they are followed (CPU): a group of fewer than one row must not
let the groups before it read contexts that are not there.  Each call runs in a
process of its own, with the contexts directly in front of a page without access."""
import os
import subprocess
import sys

import pytest

from test_boundary_cpu import ppas  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_CALL = r"""
import ctypes, mmap, os, sys
import numpy as np
from paper_2608_15171_gb300 import ppas
rows = [int(x) for x in sys.argv[1].split(",")]
n_ctx, page = int(sys.argv[2]), mmap.PAGESIZE
m = mmap.mmap(-1, 2 * page)
base = ctypes.addressof(ctypes.c_char.from_buffer(m))
libc = ctypes.CDLL(None, use_errno=True)
assert libc.mprotect(ctypes.c_void_p(base + page), ctypes.c_size_t(page), 0) == 0
at = base + page - 4 * n_ctx
ctypes.cast(at, ctypes.POINTER(ctypes.c_int32 * n_ctx)).contents[:] = [40] * n_ctx
r, p = np.array(rows, np.int32), np.zeros(len(rows), np.int32)
lens = [len(rows), r.ctypes.data, p.ctypes.data, at, 16, 2]
assert ppas._lib.ppas_shared_attention_workspace_size(*lens) == 0
st = ppas._lib.ppas_shared_attention_step(16, 16, 16, 4, 16, 4, len(rows), r.ctypes.data, p.ctypes.data, at, 16, 2,
                                          128, 0.1, 16, 256, 1 << 40, None, None)
print("status", st)
sys.stdout.flush()
os._exit(0)
"""


@pytest.mark.parametrize("rows,n_ctx", [("5,-3", 2), ("2000000,-1999999", 1), ("3,0", 2), ("4,-2147483648", 1),
                                        ("2,2,-1", 3), ("2097151,2", 1)])
def test_refused_before_the_contexts_are_read(ppas, rows, n_ctx):  # noqa: F811
    out = subprocess.run([sys.executable, "-c", _CALL, rows, str(n_ctx)], cwd=ROOT, capture_output=True, text=True,
                         timeout=300)
    assert out.returncode == 0, (out.returncode, out.stderr[-500:])
    want = ppas.PPAS_ERR_UNSUPPORTED if rows == "2097151,2" else ppas.PPAS_ERR_INVALID_ARG
    assert out.stdout.split() == ["status", str(want)]


@pytest.mark.parametrize("rows,ctx", [([5, -3], [40, 33]), ([2000000, -1999999], [40]), ([3, -1, 1], [40] * 3)])
def test_refused_by_the_binding(ppas, rows, ctx):  # noqa: F811
    """Row counts whose sum is the number of contexts."""
    kw = dict(q=16, k_cache=16, v_cache=16, num_blocks=4, d_block_tables=16, max_blocks_per_seq=4, ctx_lens=ctx,
              group_rows=rows, prefix_lens=[0] * len(rows), n_q_heads=16, n_kv_heads=2, head_dim=128, scale=0.1, out=16,
              workspace=256, workspace_bytes=1 << 40, stream=0)
    with pytest.raises(ppas.PpasError) as e:
        ppas.ppas_shared_attention_step(**kw)
    assert e.value.status == ppas.PPAS_ERR_INVALID_ARG
    assert ppas.ppas_shared_attention_workspace_size(ctx, rows, [0] * len(rows), 16, 2) == 0
