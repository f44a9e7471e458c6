"""Attention over lists through the checked build of the library (-DPSA_DEBUG_CHECKS): no index, coordinate or slot that the
kernel computes from a list is out of range, and the results are those of the regular build, bit for bit -- with entries and rows
that are no valid lists, too, which both report.  In a child process each: a process can load only one of the two libraries."""
import os
import pickle
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_CHILD = r"""
import math, pickle, sys
import torch
sys.path.insert(0, sys.argv[1])
from paper_2609_37001_b200 import build, binding as B
B.LIB_PATH = build.build(checked=(sys.argv[2] == "checked"))
# grid, tile, heads, text, share of the blocks, and whether the lists are spoilt
CASES = [
    ((3, 13, 19), (1, 16, 16), 3, 0, 0.7, False),
    ((7, 17, 35), (3, 8, 16), 2, 0, 0.5, False),
    ((2, 64, 33), (2, 32, 4), 4, 70, 0.4, False),
    ((3, 45, 32), (1, 15, 16), 40, 0, 0.5, False),
    ((4, 32, 47), (1, 8, 16), 20, 0, 0.3, False),
    ((5, 32, 48), (1, 16, 16), 5, 0, 1.1, False),
    ((2, 16, 16), (1, 16, 16), 160, 0, 0.5, False),
    ((3, 16, 48), (1, 16, 16), 2, 0, 0.6, True),
    ((3, 16, 48), (1, 16, 16), 40, 9, 0.6, True),
]
res = []
for grid, tile, heads, text, share, spoilt in CASES:
    n = grid[0] * grid[1] * grid[2]
    nb = math.prod(-(-a // b) for a, b in zip(grid, tile))
    g = torch.Generator(device="cuda").manual_seed(n + text)
    q, k, v = (torch.randn((heads, n + text, 128), device="cuda", generator=g).bfloat16() for _ in range(3))
    mask = torch.rand((heads * nb, nb), device="cuda", generator=g) < share
    ptr = torch.zeros(heads * nb + 1, dtype=torch.int32, device="cuda")
    ptr[1:] = mask.sum(1).cumsum(0)
    col = mask.nonzero()[:, 1].to(torch.int32).contiguous()
    if spoilt:
        col[3::7] = torch.tensor([-1, nb, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda").repeat(len(col))[:len(col[3::7])]
        ptr[5] = 2 ** 31 - 1
        ptr[11] = -2 ** 31
    out, lse = B.psa_attn_fwd_lists(q, k, v, ptr, col, grid, tile, 1.0 / math.sqrt(128.0), n_text=text)
    res.append((spoilt, B.psa_last_device_status(), out.view(torch.int16).cpu(), lse.view(torch.int32).cpu()))
pickle.dump(res, open(sys.argv[3], "wb"))
"""


def test_lists_in_the_checked_build(tmp_path):
    import torch
    got = {}
    for kind in ("regular", "checked"):
        f = tmp_path / f"{kind}.pkl"
        r = subprocess.run([sys.executable, "-c", _CHILD, ROOT, kind, str(f)], capture_output=True, text=True, timeout=900)
        assert r.returncode == 0, r.stderr[-2000:]
        got[kind] = pickle.load(open(f, "rb"))
    for i, ((spoilt, st_r, o_r, l_r), (_, st_c, o_c, l_c)) in enumerate(zip(got["regular"], got["checked"])):
        if spoilt:   # (either of the two faults may be the first)
            assert all(st == -1 and detail in (0x600, 0x601) for st, detail in (st_r, st_c)), (i, st_r, st_c)
        else:
            assert st_r == (0, 0) and st_c == (0, 0), (i, st_r, st_c)
        assert torch.equal(o_r, o_c) and torch.equal(l_r, l_c), i
