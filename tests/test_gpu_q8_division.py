"""sq_sparse_attn_decode_q8 in each of the ways in which it divides its work."""
import os
import re

import numpy as np
import pytest
import torch

from paper_2411_09688_amd import binding as sq
from test_gpu_q8_decode import Problem
from test_gpu_q8_rows import cu

pytestmark = pytest.mark.gpu


def bits(t):
    return t.view(torch.int16 if t.dtype is torch.float16 else torch.int32)


def run(p, rows=None):
    args = p.upload()
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    p.check(rows=rows)
    out, lse = p.out.clone(), p.lse.clone()
    p.ws.fill_(255)                                             # whatever the workspace holds: the same bits
    p.out.fill_(9.0), p.lse.fill_(9.0)
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    assert torch.equal(bits(p.out), bits(out)) and torch.equal(bits(p.lse), bits(lse))


# Without a cache a row that keeps no key has nothing at all: its output is 0, and no pool stands behind it to read from.
NO_KEYS = [  # B, H, Lq, L, C, keep, one_set
    (1, 1, 1, 64, 2, 0.0, False),                               # a single row, nothing kept
    (2, 3, 1, 500, 20, [0.0, 0.5], False),                      # workgroups for each row
    (2, 2, 4, 500, 20, [0.0, 0.5, 0.0], True),
    (1, 2, 16, 300, 30, 0.0, True),
    (50, 4, 4, 100, 9, [0.0, 0.5, 0.0], True),                  # shares of up to 256 rows
    (50, 4, 4, 100, 9, 0.0, True),
    (50, 4, 4, 100, 9, [0.0, 0.0, 0.5], False),                 # shares of more rows
    (4, 4, 4, 131072, 64, [0.0, 0.03, 0.0], True),              # shares of few, long rows
    (16, 1, 1, 140001, 900, [0.0, 0.01], False),                # the rows of a head together
    (16, 1, 1, 140001, 900, 0.0, False),
]


@pytest.mark.parametrize("B,H,Lq,L,C,keep,one_set", NO_KEYS)
def test_rows_that_keep_nothing_without_a_cache(B, H, Lq, L, C, keep, one_set):
    p = Problem(B + L, B, H, Lq, L, C, keep, None, 16, one_set)
    p.n_ranges[0], p.n_keys[0] = 0, 0
    p.ranges[0] = 0
    run(p)


def test_numbers_of_keys_outside_the_contract_without_a_cache():
    p = Problem(31, 2, 2, 1, 300, 12, 0.6, None, 16, False)
    p.n_keys[0], p.n_keys[1], p.n_ranges[2] = -5, -2 ** 31, -1
    run(p)


def constant(name):
    text = open(os.path.join(os.path.dirname(sq.__file__), "csrc", "sq_internal.hpp")).read()
    found = re.findall(rf"constexpr [a-z ]+\b{name} = ([0-9 *<]+);", text)
    assert len(found) == 1, name
    return eval(found[0])


def form(B, H, Lq, L, most_user, one_set):
    """How the launcher divides a call (L 0: no fixed context), from the constants that it uses."""
    per, g = (1, Lq) if one_set else (Lq, 1)
    if L and B * per >= 8 and 16 // g >= 8 and B * per * H * L >= constant("Q8_SHARED_MIN_KEYS"):
        return "union"
    rows, grid = B * H * per, constant("Q8_GRID")
    if rows <= grid // 4 and rows * ((L + most_user + 31) // 32 + 1) <= constant("Q8_ROW_TILES"):
        return "rows"
    return "wave" if rows <= constant("Q8_WAVE_ROWS") else "workgroup"


DIVIDED = [  # form, B, H, Lq, L, C, keep, lengths, page, one_set, spread
    ("rows", 2, 2, 4, 5000, 100, [0.0, 0.3, 0.05], [70, 0], 16, True, 2),
    ("wave", 129, 1, 1, None, 1, None, [i % 50 for i in range(129)], 16, False, 0),
    ("wave", 50, 4, 4, 100, 9, [0.0, 0.5, 1.0], [0, 40, 1, 16, 129] * 10, 16, True, 2),
    ("wave", 33, 5, 1, 300, 30, [0.0, 0.9, 0.2], [0, 0, 500] * 11, 32, False, 2),
    ("wave", 64, 4, 3, 260, 11, [0.4, 0.0, 1.0, 0.1], [33, 0] * 32, 16, True, 0),           # 256 rows
    ("wave", 64, 4, 3, 260, 11, 0.0, [0] * 64, 16, True, 0),                                # ... that have nothing
    ("wave", 4, 4, 4, 131072, 300, [0.0, 0.02, 0.0, 0.005, 0.3], [3000, 0, 17, 1], 64, True, 2),   # a row over many shares
    ("wave", 1, 4, 2, 200000, 16384, [0.02, 0.0, 0.3], [9000], 64, False, 0),               # more groups of ranges than a wave holds
    ("wave", 2, 1, 16, 600, 20, [1.0, 0.1], [20000, 9000], 64, True, 0),                    # a page table far larger than needed
    ("workgroup", 257, 1, 4, 260, 11, [0.4, 0.0, 1.0, 0.1], [33, 0, 7] * 85 + [1, 2], 16, True, 0),
    ("workgroup", 300, 1, 4, 20000, 40, [0.0] * 299 + [1.0], [i % 70 for i in range(300)], 32, True, 2),
    ("workgroup", 35, 4, 2, 400, 7, [0.0, 0.0, 0.9], [3000] + [0, 9] * 17, 16, False, 0),
]


@pytest.mark.parametrize("case", DIVIDED, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-{c[3]}-{c[4]}")
def test_each_way_of_dividing_the_work(case):
    want, B, H, Lq, L, C, keep, lengths, P, one_set, spread = case
    p = Problem(B + H, B, H, Lq, L or 1, C, keep, lengths, P, one_set, spread)
    if Lq == 16:
        p.table = np.pad(p.table, ((0, 0), (0, 600000 // P)), constant_values=-1)
        p.lengths[1] = 10 ** 6                                  # (tokens without a page are not there; of the others the last are NaN)
    assert form(B, H, Lq, L or 0, p.table.shape[1] * P, one_set) == want
    run(p, [0] if Lq == 16 else None)
    if Lq == 16:
        assert torch.isnan(p.out[1]).all() and torch.isnan(p.lse[1]).all()


@pytest.mark.parametrize("want,B,L", [("wave", 40, 0), ("wave", 40, 500), ("workgroup", 70, 0), ("workgroup", 70, 500)])
def test_pages_behind_32_bit_offsets(want, B, L):
    """A pool of more than 4 GB, of which the sequences have the last pages."""
    H, P, width = 4, 64, 2
    n = (1 << 32) // (H * P * 128) + B * width
    assert torch.cuda.mem_get_info()[0] > 3 * n * H * P * 128
    lengths = [(37 * b) % 129 for b in range(B)]
    p = Problem(B, B, H, 1, L or 1, 9, [0.0, 0.5, 0.9] if L else None, lengths, P, False, 2)
    assert form(B, H, 1, L, width * P, False) == want
    p.table = np.arange(B * width, dtype=np.int32)[::-1].reshape(B, width).copy()
    args = list(p.upload())
    pool = [torch.full((n, H, P, 128), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(n, H, device="cuda") for _ in range(2)]
    for i in range(2):
        c = p.cache[i]
        c[(c & 0x7f) == 0x7f] = 0x31
        for b in range(B):                                      # NaN behind the last token, by the table as it is now
            for t in range(lengths[b], width * P):
                c[p.table[b, t // P], :, t % P] = 0x7f
        pool[i][n - B * width:] = cu(c[:B * width])
        scales[i][n - B * width:] = cu(p.cache[2 + i][:B * width].astype(np.float32))
    args[10] = sq.make_cache(*(x.view(sq.F8) for x in pool), *scales, cu(p.table + (n - B * width)))
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    p.check()
