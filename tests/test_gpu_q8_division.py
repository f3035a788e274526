"""sq_sparse_attn_decode_q8 in each of the ways in which it divides its work: rows that have nothing to read."""
import pytest
import torch

from paper_2411_09688_amd import binding as sq
from test_gpu_q8_decode import Problem

pytestmark = pytest.mark.gpu


def run(p):
    args = p.upload()
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    p.check()
    out, lse = p.out.clone(), p.lse.clone()
    p.ws.fill_(255)                                             # whatever the workspace holds: the same bits
    p.out.fill_(9.0), p.lse.fill_(9.0)
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    assert torch.equal(p.out, out) and torch.equal(p.lse, lse)


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
