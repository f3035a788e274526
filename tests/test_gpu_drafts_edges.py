"""The calls around drafted tokens at their edges: codes read back with any scale, and the serving loop with trees of uneven size, its selection checked."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from oracle import literal
from paper_2411_09688_amd import binding as sq
from test_gpu_drafts_path import SCALE, Server
from test_gpu_q8_rows import cu

pytestmark = pytest.mark.gpu
F16, F32, I32 = torch.float16, torch.float32, torch.int32


def scales_that_round_twice(n):
    """Scales for which some code's product, rounded to fp32 first, falls onto a border of f16 and then to the other side."""
    rng = np.random.default_rng(1)
    found = []
    while len(found) < n:
        s = rng.uniform(2.0 ** -16, 2.0 ** -4, 400000).astype(np.float32)
        for m in range(9, 16):                                  # (a code's mantissa; 8 is a power of two)
            p = m * s.astype(np.float64)
            found += list(s[p.astype(np.float32).astype(np.float16) != p.astype(np.float16)])
    return np.array(found[:n], np.float32)


def test_what_is_read_back_is_rounded_once():
    """Every code times scales that are no powers of two, those among them where rounding twice shows: of both signs, into f16's subnormals and past its end."""
    rng = np.random.default_rng(2)
    picked = scales_that_round_twice(60)
    scales = np.concatenate([picked, -picked[:20], picked[:40] * 2.0 ** rng.integers(-20, 20, 40), [2.0 ** -126, 2.0 ** -127, 1.5 * 2.0 ** -127],
                             [0.0, 3e38, 0.0123, 2.0 ** -30, 2.0 ** 20]]).astype(np.float32)
    n = len(scales)
    codes = np.broadcast_to(np.arange(256, dtype=np.uint8).reshape(1, 1, 2, 128).repeat(8, 2), (n, 1, 16, 128)).copy()
    cache = sq.make_cache(*(cu(codes).view(sq.F8) for _ in range(2)), cu(scales.reshape(n, 1)), cu(-scales[::-1].reshape(n, 1)), cu(np.arange(n, dtype=np.int32).reshape(1, n)))
    sh = sq.make_shape(1, 1, 1, 1, 1, 16 * n, 1.0)
    out = [torch.zeros(1, 1, 16 * n, 128, dtype=F16, device="cuda") for _ in range(2)]
    sq.sq_cache_read(sh, cache, None, cu(np.array([16 * n], np.int32)), *out)
    twice = 0
    for x, s in zip(out, (scales, -scales[::-1])):
        with np.errstate(over="ignore", invalid="ignore"):
            p = ref.VALUES[codes[:, 0]] * s.astype(np.float64)[:, None, None]      # (4 times 24 bits: exact)
            want, other = p.astype(np.float16).reshape(16 * n, 128), p.astype(np.float32).astype(np.float16).reshape(16 * n, 128)
        assert np.array_equal(x[0, 0].cpu().numpy(), want, equal_nan=True)
        twice += ((want != other) & ~np.isnan(want)).sum()
    assert twice >= 100


def test_every_code_times_every_power_of_two_is_read_back():
    n = 254
    scales = np.ldexp(1.0, np.arange(-126, 128)).astype(np.float32)
    codes = np.broadcast_to(np.arange(256, dtype=np.uint8).reshape(1, 1, 2, 128).repeat(8, 2), (n, 1, 16, 128)).copy()
    cache = sq.make_cache(*(cu(codes).view(sq.F8) for _ in range(2)), cu(scales.reshape(n, 1)), cu(-scales.reshape(n, 1)), cu(np.arange(n, dtype=np.int32).reshape(1, n)))
    sh = sq.make_shape(1, 1, 1, 1, 1, 16 * n, 1.0)
    out = [torch.zeros(1, 1, 16 * n, 128, dtype=F16, device="cuda") for _ in range(2)]
    sq.sq_cache_read(sh, cache, None, cu(np.array([16 * n], np.int32)), *out)
    for x, s in zip(out, (scales, -scales)):
        with np.errstate(over="ignore"):
            want = (ref.VALUES[codes[:, 0]] * s.astype(np.float64)[:, None, None]).astype(np.float16).reshape(16 * n, 128)
        assert np.array_equal(x[0, 0].cpu().numpy(), want, equal_nan=True)


class Ragged(Server):
    """The serving loop with trees of uneven size: rows of drafts that there are not hold anything, and take their first draft's query before the
    sequence's kept set is chosen, which averages over all rows."""

    def __init__(self, seed, B, H, G, T, page):
        super().__init__(seed, B, H, G, T, page)
        self.t = torch.arange(T, device="cuda")

    def draw(self, rng):
        super().draw(rng)
        empty = (self.t >= self.n.view(-1, 1)) & (self.n.view(-1, 1) > 0)
        self.x[empty.flatten()] = float("nan")

    def step(self):
        H, G = self.H, self.G
        torch.add(self.held, self.L, out=self.first)
        sq.sq_tree_prepare(self.rows, self.parents, self.n, self.first, self.mask, self.positions)
        sq.sq_head_norm_rotate(self.rows, G, self.rot, self.positions, self.x[:, :H * G], self.x[:, H * G:H * G + H], self.x[:, H * G + H:], self.q, self.k, self.v)
        there = self.t < self.n.view(-1, 1)
        self.q.copy_(torch.where(there[:, None, :, None], self.q, self.q[:, :, :1]))
        sq.sq_centroid_score(self.sel, self.q, self.cent, self.sizes, self.logits, self.row_max, self.denom)
        sq.sq_select_mean(self.sel, self.logits, self.row_max, self.denom, self.thresh, self.sizes, self.offsets, self.keep, self.ranges, self.nr, self.nk, self.ws[0])
        sq.sq_tree_attn_q8(self.sel, self.T, self.q, *self.fixed, self.ranges, self.nr, self.nk, self.cache, self.held, self.k, self.v, self.mask, self.n, self.out,
                           self.lse, self.ws[1])
        sq.sq_tree_accept(self.rows, self.parents, self.n, self.tokens, self.target, self.held, self.count, self.path, self.token, self.new_len)
        sq.sq_cache_commit(self.rows, self.cache, self.held, self.path, self.count, self.k, self.v)
        self.held.copy_(self.new_len)

    def check_selection(self):
        """The kept sets from the drafts that there are: each query once, the first draft's for every row that is none."""
        q, n, cent, sizes, offsets = (x.cpu().numpy() for x in (self.q, self.n, self.cent, self.sizes, self.offsets))
        ranges, nr, nk, thresh = (x.cpu().numpy() for x in (self.ranges, self.nr, self.nk, self.thresh))
        decided = 0
        for b in range(self.B):
            if n[b] == 0:
                continue
            rows = np.minimum(np.arange(self.T), np.where(np.arange(self.T) < n[b], self.T, 0))
            for h in range(self.H):
                mine = q[b, h * self.G:h * self.G + self.G][:, rows].reshape(-1, 128)
                assert np.isfinite(mine).all()
                keep, mean = literal.select_mean(mine, cent[0, h], sizes[0, h], thresh[h], SCALE)
                got = np.zeros(self.C, bool)
                got[np.searchsorted(offsets[0, h, 1:], ranges[b, h, :nr[b, h], 0], side="right")] = True
                near = literal.near_threshold(mean, thresh[h])
                assert np.array_equal(got[~near], keep[~near]) and nr[b, h] == got.sum() and nk[b, h] == sizes[0, h][got].sum()
                ids = np.flatnonzero(got)
                assert np.array_equal(ranges[b, h, :nr[b, h]], np.stack([offsets[0, h][ids], sizes[0, h][ids]], 1))
                decided += (~near).sum()
        return decided


@pytest.mark.parametrize("B,H,G,T,page", [(2, 2, 3, 12, 16), (3, 1, 4, 33, 32), (2, 2, 1, 7, 64)])
def test_a_loop_with_trees_of_uneven_size(B, H, G, T, page):
    rng = np.random.default_rng(T + 7)
    s = Ragged(T, B, H, G, T, page)
    held, kept = [0] * B, []
    for _ in range(6):
        s.draw(rng)
        s.step()
        assert s.check_selection() > 0
        held = s.check(held)
        kept += s.nr.flatten().tolist()
    assert 0 < sum(kept) < len(kept) * s.C and len(set(kept)) > 1


def test_a_captured_loop_with_trees_of_uneven_size():
    made, eager = (Ragged(3, 3, 2, 4, 14, 16) for _ in range(2))
    made.draw(np.random.default_rng(0))
    made.step()
    for c, e in zip(made.cache.tensors, (0x7f, 0x7f, 1.0, 1.0)):
        (c.view(torch.uint8) if c.dtype == sq.F8 else c).fill_(e)
    for x in (made.held, made.out, made.lse, made.ranges):
        x.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made.step()
    held = [0] * 3
    for turn in range(4):
        for x in (made, eager):
            x.draw(np.random.default_rng(20 + turn))
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        for name in ("mask", "positions", "ranges", "nk", "out", "lse", "path", "count", "token", "held"):
            assert torch.equal(getattr(made, name), getattr(eager, name)), (turn, name)
        assert eager.check_selection() > 0
        held = eager.check(held)
