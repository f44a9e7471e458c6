"""Long lists with entries that do not belong there, against the definition over what is left of them: an entry that is no block, or does
not come behind the entry in front of it (whatever that is), is left out, and a row that does not lie within the entries, or is longer
than there are blocks, is empty.  The kernel reads 32 entries at a time and may split a row between CTAs: faults lie at either border, at a row's
first entry and all over it."""
import math

import pytest
import torch

from paper_2609_37001_b200 import binding as B
from test_attn_lists import SCALE, check, pack, tensors
from test_select_blocks import blocks_of_tokens

pytestmark = pytest.mark.gpu


def left_of(row, nb):
    """The entries that count."""
    before, good = -1, []
    for j in row:
        if 0 <= j < nb and j > before:
            good.append(j)
        before = j
    return good


def run(grid, tile, heads, rows, text=0, bounds=None, mode=None):
    """rows: raw entries of every row, [heads][blocks]; bounds: row_ptr entries to replace."""
    nb = blocks_of_tokens(grid, tile)[1]
    q, k, v = tensors(heads, math.prod(grid) + text, 23)
    row_ptr, col_idx = pack(rows)
    lists = [[left_of(row, nb) for row in head] for head in rows]
    if bounds:
        col = col_idx.tolist()
        for r, x in bounds.items():
            row_ptr[r] = x
        ptr = row_ptr.tolist()
        for r in range(heads * nb):
            a, b = ptr[r], ptr[r + 1]
            lists[r // nb][r % nb] = left_of(col[a:b], nb) if 0 <= a <= b <= len(col) and b - a <= nb else []
    out, lse = B.psa_attn_fwd_lists(q, k, v, row_ptr, col_idx, grid, tile, SCALE, n_text=text)
    assert mode is None or B.psa_last_attn_launch()[1] == mode
    status, detail = B.psa_last_device_status()
    assert status == B.PSA_ERR_INVALID_ARG and detail in ((0x600, 0x601) if bounds else (0x601,))
    check(out, lse, q, k, v, lists, grid, tile, text)
    again = B.psa_attn_fwd_lists(q, k, v, row_ptr, col_idx, grid, tile, SCALE, n_text=text)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def spoil(row, kind, nb):
    row = list(row)
    if kind == "repeat":   # at the borders of 32 entries
        for p in (32, 64):
            row[p] = row[p - 1]
    elif kind == "descent":
        for p in (32, 64):
            row[p] = row[p - 3]
    elif kind == "beyond":   # the entry behind it comes from behind the border, and is left out with it
        row[31] = nb
        row[63] = 2 ** 31 - 1
    elif kind == "negative":
        row[0], row[31], row[32], row[64] = -1, -1, -2 ** 31, -7
    elif kind == "first":
        row[0] = nb + 5
    elif kind == "all":
        row = [(-1, nb, 2 ** 31 - 1, -2 ** 31)[i % 4] for i in range(len(row))]
    elif kind == "same":
        row = [row[5]] * len(row)
    elif kind == "falling":
        row = row[::-1]
    elif kind == "eighths":   # the borders of 2, 4 and 8 shares, and their neighbours
        for p in sorted({len(row) * i // 8 for i in range(1, 8)}):
            row[p] = row[p - 1]
    return row


FAULTS = ["repeat", "descent", "beyond", "negative", "first", "all", "same", "falling", "eighths"]
# grid, tile, heads, text, how items are handed out
LAUNCHES = [
    ((5, 32, 64), (1, 8, 16), 4, 0, "ticket"),
    ((5, 32, 64), (1, 8, 16), 4, 37, "ticket"),
    ((5, 31, 61), (1, 8, 16), 4, 0, "ticket"),
    ((3, 64, 96), (1, 16, 16), 1, 0, "shared_direct"),
    ((3, 63, 96), (1, 16, 16), 1, 5, "shared_direct"),
    ((3, 64, 96), (1, 16, 16), 2, 0, "direct"),
]


@pytest.mark.parametrize("launch", LAUNCHES, ids=lambda x: "%s-%d-%d" % (x[4], x[2], x[3]) if isinstance(x, tuple) else "")
@pytest.mark.parametrize("fault", FAULTS)
def test_long_rows(fault, launch):
    grid, tile, heads, text, mode = launch
    nb = blocks_of_tokens(grid, tile)[1]
    g = torch.Generator().manual_seed(29)
    rows = []
    for _ in range(heads):   # every third row as it should be
        good = [sorted(torch.randperm(nb, generator=g)[:67 + i % 5].tolist()) for i in range(nb)]
        rows.append([row if i % 3 == 2 else spoil(row, fault, nb) for i, row in enumerate(good)])
    run(grid, tile, heads, rows, text, mode=mode)


@pytest.mark.parametrize("heads,text", [(2, 0), (40, 9)])
def test_rows_that_do_not_lie_within_the_entries(heads, text):
    """With entries that are no blocks, in short rows."""
    grid, tile, nb = (3, 16, 48), (1, 16, 16), 9
    g = torch.Generator().manual_seed(31)
    rows = [[[j for j in range(nb) if torch.rand((), generator=g) < 0.6] for _ in range(nb)] for _ in range(heads)]
    n = 0
    for head in rows:
        for row in head:
            for i in range(len(row)):
                if n % 7 == 3:
                    row[i] = (-1, nb, 2 ** 31 - 1, -2 ** 31)[n // 7 % 4]
                n += 1
    run(grid, tile, heads, rows, text, bounds={5: 2 ** 31 - 1, 11: -2 ** 31})
