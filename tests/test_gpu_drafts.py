"""Trees of drafts, what is accepted of them, and rows written to and read from the paged 8-bit cache, against plain implementations."""
import numpy as np
import pytest
import torch

import drafts_reference as plain
import q8_reference as ref
from paper_2411_09688_amd import binding as sq
from test_gpu_q8_rows import cu

pytestmark = pytest.mark.gpu
F16, F32, I32 = torch.float16, torch.float32, torch.int32


def forest(rng, B, T, kind):
    t = np.arange(T)
    if kind == "chain":
        p = np.broadcast_to(t - 1, (B, T)).copy()
    elif kind == "star":
        p = np.zeros((B, T), int)
    elif kind == "anything":                                    # roots among them, and parents that are none
        p = rng.integers(-3, T + 3, (B, T))
    else:
        p = (rng.random((B, T)) * t).astype(int)
    p[:, 0] = rng.integers(-2, T + 2, B)                         # not looked at
    return p.astype(np.int32)


@pytest.mark.parametrize("B,T,kind", [(1, 1, "tree"), (3, 2, "chain"), (2, 31, "tree"), (5, 32, "anything"), (2, 33, "chain"), (7, 64, "tree"),
                                      (3, 65, "anything"), (2, 200, "star"), (4, 256, "tree"), (1, 257, "tree"), (2, 1000, "anything"), (1, 1024, "chain")])
def test_prepare(B, T, kind):
    rng = np.random.default_rng(T)
    parents = forest(rng, B, T, kind)
    n = rng.integers(-1, T + 2, B)
    n[0] = T
    first = rng.integers(-50, 1 << 20, B)
    sh = sq.make_shape(B, 1, 1, 1, T, 0, 1.0)
    for counts, start in ((n, first), (None, None)):
        bits, positions = plain.prepare(parents, [T] * B if counts is None else counts, [0] * B if start is None else start)
        mask, pos = torch.full((B, T, -(-T // 32)), -7, dtype=I32, device="cuda"), torch.full((B, T), -7, dtype=I32, device="cuda")
        opt = lambda x: None if x is None else cu(x.astype(np.int32))  # noqa: E731
        sq.sq_tree_prepare(sh, cu(parents), opt(counts), opt(start), mask, pos)
        assert np.array_equal(mask.cpu().numpy(), plain.words(bits)) and np.array_equal(pos.cpu().numpy(), positions)
        only = torch.zeros_like(pos)
        sq.sq_tree_prepare(sh, cu(parents), opt(counts), opt(start), None, only)
        assert torch.equal(only, pos)
        only = torch.zeros_like(mask)
        sq.sq_tree_prepare(sh, cu(parents), opt(counts), opt(start), only, None)
        assert torch.equal(only, mask)


@pytest.mark.parametrize("B,T,kind,vocabulary", [(1, 1, "tree", 2), (4, 2, "chain", 1), (9, 63, "tree", 3), (9, 64, "chain", 1), (5, 65, "tree", 2), (3, 256, "anything", 2),
                                                 (3, 257, "tree", 2), (2, 1024, "chain", 1), (2, 1024, "star", 5), (300, 7, "tree", 2)])
def test_accept(B, T, kind, vocabulary):
    rng = np.random.default_rng(T + B)
    parents = forest(rng, B, T, kind)
    n = rng.integers(-1, T + 2, B)
    n[0] = T
    tokens, target = rng.integers(-1, vocabulary - 1, (2, B, T)).astype(np.int32)       # (-1 is a token like any other)
    held = rng.integers(0, 1 << 20, B).astype(np.int32)
    sh = sq.make_shape(B, 1, 1, 1, T, 0, 1.0)
    for counts in (n, None):
        found = plain.accept(parents, [T] * B if counts is None else counts, tokens, target)
        out = [torch.full(s, -7, dtype=I32, device="cuda") for s in ((B,), (B, T), (B,), (B,))]
        c = None if counts is None else cu(counts.astype(np.int32))
        sq.sq_tree_accept(sh, cu(parents), c, cu(tokens), cu(target), cu(held), *out)
        count, path, token, new = (x.cpu().numpy() for x in out)
        assert count.tolist() == [len(p) for p in found]
        assert path.tolist() == [p + [-1] * (T - len(p)) for p in found]
        assert token.tolist() == [int(target[b, p[-1]]) if p else -1 for b, p in enumerate(found)]
        assert new.tolist() == [int(held[b]) + len(p) for b, p in enumerate(found)]
        less = [torch.full_like(x, -7) for x in out[:2]]
        sq.sq_tree_accept(sh, cu(parents), c, cu(tokens), cu(target), None, *less, None, None)
        assert torch.equal(less[0], out[0]) and torch.equal(less[1], out[1])
    assert any(len(p) > 1 for p in found) or T == 1 or kind == "anything"


def pool(rng, B, H, page, width, spare=2):
    """Pages with the codes that 8-bit values leave, NaN among them, and scales; a table of pages that nobody else has."""
    n = B * width + spare
    codes = [rng.integers(0, 256, (n, H, page, 128)).astype(np.uint8) for _ in range(2)]
    scales = [2.0 ** rng.integers(-9, -4, (n, H)).astype(np.float64) for _ in range(2)]
    return codes, scales, rng.permutation(n)[:B * width].reshape(B, width).astype(np.int32)


def cache_of(codes, scales, table):
    return sq.make_cache(*(cu(c.copy()).view(sq.F8) for c in codes), *(cu(s.astype(np.float32)) for s in scales), cu(table))


def check_cache(cache, codes, scales):
    for i in range(2):
        assert ref.same_codes(cache.tensors[i].view(torch.uint8).cpu().numpy(), codes[i]).all()
        assert np.array_equal(cache.tensors[2 + i].cpu().numpy(), scales[i].astype(np.float32))


@pytest.mark.parametrize("B,H,T,page,rows,picked", [(1, 1, 1, 16, 1, True), (3, 2, 5, 16, 5, True), (2, 3, 64, 64, 6, True), (4, 2, 20, 32, 20, True), (2, 2, 100, 64, 70, True),
                                                    (3, 2, 1, 64, 1, False), (2, 3, 15, 32, 15, False), (2, 2, 16, 16, 16, False), (1, 2, 33, 32, 33, False),
                                                    (3, 1, 500, 64, 500, False), (2, 2, 130, 16, 130, False)])
def test_commit(B, H, T, page, rows, picked):
    rng = np.random.default_rng(T * 100 + page)
    width = -(-(70 + T) // page)
    codes, scales, table = pool(rng, B, H, page, width)
    scales[0][0] = 0.013                                        # a scale that is no power of two, if its page is appended to
    old = rng.integers(0, 70, B).astype(np.int32)
    old[0] = page * (width - 1) + page // 2                     # the end of the table: what is behind it is dropped
    if B > 2:
        table[1, old[1] // page] = -1                           # no page
        table[2, -1] = len(codes[0])
    n = rng.integers(0, rows + 1, B)
    n[0] = rows
    K, V = ((rng.standard_normal((B, H, T, 128)) * np.exp(rng.standard_normal((B, H, 1, 1)))).astype(np.float16) for _ in range(2))
    K[0, 0, 0, 3], V[0, 0, T // 2, 5:8] = np.inf, [np.nan, -np.inf, 65504]
    path = np.full((B, T), -1, np.int32)
    for b in range(B):
        path[b, :rows] = np.sort(rng.permutation(T)[:rows])
    path[0, 0] = -5                                             # read as row 0
    path[-1, rows - 1] = T + 3                                  # read as the last row
    sh = sq.make_shape(B, H, 1, 1, T, 0, 1.0)
    cache = cache_of(codes, scales, table)
    counts = None if not picked and rows == T and B == 1 else cu(n.astype(np.int32))
    for again in range(2):                                      # the same rows again change nothing
        sq.sq_cache_commit(sh, cache, cu(old), cu(path) if picked else None, counts, cu(K), cu(V))
    for i, X in enumerate((K, V)):
        X = X.astype(np.float64).transpose(0, 2, 1, 3)           # [B, T, H, 128]
        if picked:
            X = np.take_along_axis(X, np.clip(path, 0, T - 1)[:, :, None, None], 1)
        plain.commit(codes[i], scales[i], table, old.tolist(), [T] * B if counts is None else n.tolist(), X)
    check_cache(cache, codes, scales)


def test_commit_of_rows_that_were_appended_before():
    """The same f16 rows through sq_cache_append (no norm, no rotation) and through sq_cache_commit leave the same cache."""
    rng = np.random.default_rng(5)
    B, H, T, page = 3, 2, 40, 32
    codes, scales, table = pool(rng, B, H, page, 5)
    old = np.array([0, 31, 64], np.int32)
    K, V = (rng.standard_normal((B, T, H, 128)).astype(np.float16) for _ in range(2))
    a, b = cache_of(codes, scales, table), cache_of(codes, scales, table)
    sh = sq.make_shape(B, H, 1, 1, T, 0, 1.0)
    sq.sq_cache_append(sh, 1, sq.make_rotary(None), a, cu(old), None, None, cu(K.reshape(B * T, H, 128)), cu(V.reshape(B * T, H, 128)), None)
    rows = lambda x: cu(np.ascontiguousarray(x.transpose(0, 2, 1, 3)))  # noqa: E731
    sq.sq_cache_commit(sh, b, cu(old), None, None, rows(K), rows(V))
    for x, y in zip(a.tensors, b.tensors):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("B,H,U,page", [(1, 1, 1, 16), (2, 3, 63, 16), (3, 2, 64, 32), (2, 2, 65, 64), (4, 1, 700, 64), (3, 5, 200, 16)])
def test_read(B, H, U, page):
    rng = np.random.default_rng(U)
    width = -(-(U + 30) // page)
    codes, scales, table = pool(rng, B, H, page, width)
    scales[0][:, 0] = 2.0 ** rng.integers(-30, 12, len(scales[0]))      # past f16's range at both ends
    scales[1][:, -1] = 0.0123
    held = rng.integers(0, U + 31, B).astype(np.int32)
    first = rng.integers(-3, 30, B).astype(np.int32)
    held[0], first[0] = U + 29, 17
    if B > 2:
        held[1], held[2] = -4, 1 << 28                          # (the table's end is the sequence's)
        table[2, 0], table[2, -1] = -1, len(codes[0]) + 5
    cache = cache_of(codes, scales, table)
    sh = sq.make_shape(B, H, 1, 1, 1, U, 1.0)
    for start in (first, None):
        out = [torch.full((B, H, U, 128), 7.0, dtype=F16, device="cuda") for _ in range(2)]
        sq.sq_cache_read(sh, cache, None if start is None else cu(start), cu(held), *out)
        for i in range(2):
            want = np.full((B, H, U, 128), 7.0, np.float16)
            for b in range(B):
                f = 0 if start is None else max(start[b], 0)
                for u in range(max(min(U, min(held[b], width * page) - f), 0)):
                    page_id, slot = table[b, (f + u) // page], (f + u) % page
                    with np.errstate(over="ignore"):
                        want[b, :, u] = (ref.VALUES[codes[i][page_id, :, slot]] * scales[i][page_id].astype(np.float32)[:, None].astype(np.float64)
                                         if 0 <= page_id < len(codes[0]) else np.zeros((H, 128))).astype(np.float32).astype(np.float16)
            assert np.array_equal(out[i].cpu().numpy(), want, equal_nan=True)


def test_what_is_read_back_commits_to_the_same_cache():
    rng = np.random.default_rng(8)
    B, H, T, page = 2, 3, 150, 64
    codes, scales, table = pool(rng, B, H, page, 3, 3 * B)
    cache = cache_of(codes, scales, table)
    sh = sq.make_shape(B, H, 1, 1, T, T, 1.0)
    K, V = (cu(rng.standard_normal((B, H, T, 128)).astype(np.float16)) for _ in range(2))
    zero, full = torch.zeros(B, dtype=I32, device="cuda"), torch.full((B,), T, dtype=I32, device="cuda")
    sq.sq_cache_commit(sh, cache, zero, None, None, K, V)
    back = [torch.empty_like(K) for _ in range(2)]
    sq.sq_cache_read(sh, cache, None, full, *back)
    assert all(((x - y).abs() <= y.abs() * 2.0 ** -4 + 2.0 ** -10 * 2.0 ** -5).all() for x, y in zip(back, (K, V)))
    other = cache_of(codes, scales, (len(codes[0]) - 1 - np.arange(B * 3)).reshape(B, 3).astype(np.int32))
    sq.sq_cache_commit(sh, other, zero, None, None, *back)
    again = [torch.empty_like(K) for _ in range(2)]
    sq.sq_cache_read(sh, other, None, full, *again)
    assert all(torch.equal(x, y) for x, y in zip(back, again))


def test_calls_that_pass_the_caches():
    """From 256 MB on: rows written at once against the same rows written in two halves, and what is read back against torch."""
    B, H, T, page = 8, 8, 6000, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    K, V = (torch.randn(B, H, T, 128, generator=g, device="cuda").half() for _ in range(2))
    width = -(-(T + 50) // page)
    rng = np.random.default_rng(3)
    pages = rng.permutation(B * width).reshape(B, width).astype(np.int32)
    made = []
    for _ in range(2):
        codes = [torch.full((B * width, H, page, 128), 0x11, dtype=torch.uint8, device="cuda").view(sq.F8) for _ in range(2)]
        made.append(sq.make_cache(*codes, *(torch.full((B * width, H), 2.0 ** -9, device="cuda") for _ in range(2)), cu(pages)))
    old = cu(rng.integers(0, 50, B).astype(np.int32))
    sh = sq.make_shape(B, H, 1, 1, T, T + 50, 1.0)
    assert B * H * T * 128 * 6 >= 256 << 20
    sq.sq_cache_commit(sh, made[0], old, None, None, K, V)
    # (from whole pages on, so that no page's scale is decided in two calls)
    cut = ((old + T // 2) // page * page - old).int()
    for b in range(B):                                          # each sequence's halves end at its own page
        one = sq.make_shape(1, H, 1, 1, T, 0, 1.0)
        c = sq.make_cache(*made[1].tensors[:4], made[1].tensors[4][b:b + 1].clone())
        n = int(cut[b])
        start = old[b:b + 1].clone()
        sq.sq_cache_commit(one, c, start, None, torch.full((1,), n, dtype=I32, device="cuda"), K[b:b + 1].contiguous(), V[b:b + 1].contiguous())
        rest = [torch.cat([x[b:b + 1, :, n:], x[b:b + 1, :, :n]], 2).contiguous() for x in (K, V)]
        sq.sq_cache_commit(one, c, start + n, None, torch.full((1,), T - n, dtype=I32, device="cuda"), *rest)
    for x, y in zip(made[0].tensors[:4], made[1].tensors[:4]):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    out = [torch.full((B, H, T + 50, 128), 3.0, dtype=F16, device="cuda") for _ in range(2)]
    held = old + T
    sq.sq_cache_read(sh, made[0], None, held.int(), *out)
    t = torch.arange(T + 50, device="cuda")
    at = cu(pages).long()[:, (t // page).clamp(max=width - 1)]
    for i in range(2):
        codes = made[0].tensors[i].view(torch.uint8)[at, :, t % page].view(sq.F8).float() * made[0].tensors[2 + i][at][..., None]
        want = torch.where((t < held.view(-1, 1))[:, :, None, None], codes.half(), torch.tensor(3.0, dtype=F16, device="cuda"))
        assert torch.equal(out[i], want.transpose(1, 2))
