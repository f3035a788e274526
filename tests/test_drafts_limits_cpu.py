"""How large the attention of drafts may be: what is refused as too large, and what is not (the next check of the call refuses it here)."""
import ctypes as C

import pytest

from test_q8_boundary_cpu import at, cache, refused, sq  # noqa: F401


def attention(sq, B, H, L, G, T, max_pages=2, ranges=False, masked=False):  # noqa: F811
    """A call whose lse overlaps its queries, which is looked at behind the sizes."""
    shape = sq.make_shape(B, H, L, 5, G * T, 0, 0.1)
    fixed = [1 << 50, 1 << 51, 1 << 52, 1 << 53, 1 << 54, 1 << 55, 1 << 56] if ranges else [None] * 7
    far = [i << 57 for i in range(1, 5)]
    return sq.lib().sq_tree_attn_q8(C.byref(shape), T, at(1), *fixed, cache(sq, n_pages=1, max_pages=max_pages), at(2 ** 8), far[0], far[1], at(2 ** 9) if masked else None, None,
                                    far[2], at(1), None, 0, None)


MOST = 1 << 21


@pytest.mark.parametrize("B,H,L,G,T,max_pages,ranges", [(1, 1, 1, 1, MOST, 2, False), (1, 8, 1, 4, MOST // 4, MOST // 16, False), (64, 8, 1, 4, 2048, MOST // 16, False),
                                                        (16, 8, MOST, 4, 8192, MOST // 16, True), (1, 1023, MOST, 1, 1, MOST // 16, True), (4, 8, MOST, 64, 3, 2, True)])
def test_sizes_that_are_taken(sq, B, H, L, G, T, max_pages, ranges):  # noqa: F811
    refused(sq, attention(sq, B, H, L, G, T, max_pages, ranges), sq.SQ_ERR_INVALID_ARG, b"overlaps")


@pytest.mark.parametrize("B,H,L,G,T,max_pages,ranges,masked", [
    (1, 1, 1, 1, MOST + 1, 2, False, False),                    # drafts of a chain
    (1, 1, 1, 1, 32769, 2, False, True),                        # drafts with a mask
    (1, 1024, MOST, 1, 1, 2, True, False),                      # H * L
    (1 << 10, 1 << 10, 1, 1, 1 << 10, 2, False, False),         # B * H * Lq
    (1 << 12, 1 << 12, 1, 1, 1, 2, False, False),               # blocks
    (64, 64, 1, 64, 2048, MOST // 16, False, False),            # blocks times keys
])
def test_sizes_that_are_not(sq, B, H, L, G, T, max_pages, ranges, masked):  # noqa: F811
    refused(sq, attention(sq, B, H, L, G, T, max_pages, ranges, masked), sq.SQ_ERR_UNSUPPORTED, b"too large")
