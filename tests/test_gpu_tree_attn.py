"""sq_tree_attn_q8 against a plain implementation in 64 bits: sizes, masks, sources, values that are not finite, input outside the contract."""
import numpy as np
import pytest
import torch

import drafts_reference as plain
import q8_reference as ref
from paper_2411_09688_amd import binding as sq
from test_gpu_drafts import forest
from test_gpu_q8_rows import cu

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))
F16, F32, I32 = torch.float16, torch.float32, torch.int32


class Problem:
    """Inputs of one call on the host, and what it has to give."""

    def __init__(self, seed, B, H, G, T, L=0, C=0, keep=0.3, user=0, page=16, mask="tree", ragged=False, drafts=True, scales=(-8, -4)):
        self.B, self.H, self.G, self.T, self.L, self.C, self.user, self.page = B, H, G, T, L, C, user, page
        rng = self.rng = np.random.default_rng(seed)
        codes = lambda *s: (rng.standard_normal(s) * 40).clip(-448, 448)  # noqa: E731
        code = lambda *s: ref.encode(codes(*s))  # noqa: E731
        power = lambda *s: 2.0 ** rng.integers(*scales, s).astype(np.float64)  # noqa: E731
        self.q = rng.standard_normal((B, H * G, T, 128)).astype(np.float16)
        self.bits = self.mask = None
        if drafts:
            self.Kd, self.Vd = (rng.standard_normal((B, H, T, 128)).astype(np.float16) for _ in range(2))
            if mask == "tree":
                self.bits = plain.prepare(forest(rng, B, T, "tree"), [T] * B, [0] * B)[0]
            elif mask == "any":
                self.bits = rng.random((B, T, T)) < 0.4
                self.bits[:, rng.integers(0, T)] = False
            if self.bits is not None:
                self.mask = plain.words(self.bits)
        else:
            self.Kd = self.Vd = None
        self.n = None
        if ragged:
            self.n = rng.integers(0, T + 1, B).astype(np.int32)
            self.n[0] = T
            self.n[-1] = 0 if B > 2 else self.n[-1]
        self.ranges = None
        if C:
            self.K8, self.V8 = code(H, L, 128), code(H, L, 128)
            self.ks, self.vs = power(H, -(-L // 64)), power(H, -(-L // 64))
            self.ranges, self.nr, self.nk = np.zeros((B, H, C, 2), np.int32), np.zeros((B, H), np.int32), np.zeros((B, H), np.int32)
            for h in range(H):
                cuts = np.sort(rng.integers(0, L + 1, C - 1))
                first, size = np.concatenate([[0], cuts]), np.diff(np.concatenate([[0], cuts, [L]]))
                for b in range(B):
                    ids = np.flatnonzero((rng.random(C) < keep) & (size > 0))
                    self.ranges[b, h, :len(ids)] = np.stack([first[ids], size[ids]], 1)
                    self.nr[b, h], self.nk[b, h] = len(ids), size[ids].sum()
        self.held = None
        if user:
            width = -(-user // page)
            self.cK, self.cV = code(B * width + 2, H, page, 128), code(B * width + 2, H, page, 128)
            self.cks, self.cvs = power(B * width + 2, H), power(B * width + 2, H)
            self.table = rng.permutation(B * width + 2)[:B * width].reshape(B, width).astype(np.int32)
            self.held = rng.integers(0, user + 1, B).astype(np.int32)
            self.held[0] = user

    def keys(self, b, h):
        """(k, v, seen by each row (t, g) or None, value's scale) of the context, the cache and the drafts."""
        found = [(np.zeros((0, 128)), np.zeros((0, 128)), None, np.ones(0))]
        if self.ranges is not None:
            ids = np.concatenate([np.arange(s, s + c) for s, c in self.ranges[b, h, :self.nr[b, h]]] + [np.zeros(0, int)]).astype(int)
            found.append((ref.VALUES[self.K8[h, ids]] * self.ks[h, ids // 64][:, None], ref.VALUES[self.V8[h, ids]] * self.vs[h, ids // 64][:, None], None,
                          self.vs[h, ids // 64]))
        if self.held is not None:
            t = np.arange(min(max(self.held[b], 0), self.table.shape[1] * self.page))
            page = self.table[b, t // self.page]
            t, page = t[(page >= 0) & (page < len(self.cK))], page[(page >= 0) & (page < len(self.cK))]
            at = (page, h, t % self.page)
            found.append((ref.VALUES[self.cK[at]] * self.cks[page, h][:, None], ref.VALUES[self.cV[at]] * self.cvs[page, h][:, None], None, self.cvs[page, h]))
        n = self.T if self.n is None else min(max(self.n[b], 0), self.T)
        if self.Kd is not None:
            seen = np.tril(np.ones((self.T, self.T), bool)) if self.bits is None else self.bits[b]
            seen = np.repeat(seen[:n, :n], self.G, 0)
            found.append((self.Kd[b, h, :n].astype(np.float64), self.Vd[b, h, :n].astype(np.float64), seen, np.ones(n)))
        return found, n

    def upload(self):
        opt = lambda x: None if x is None else cu(x)  # noqa: E731
        B, H, G, T = self.B, self.H, self.G, self.T
        self.shape = sq.make_shape(B, H, max(self.L, 1), max(self.C, 1), G * T, 0, SCALE)
        fixed = [None] * 7
        if self.ranges is not None:
            fixed = [cu(self.K8).view(sq.F8), cu(self.V8).view(sq.F8), cu(self.ks.astype(np.float32)), cu(self.vs.astype(np.float32)), cu(self.ranges),
                     cu(self.nr), cu(self.nk)]
        self.cache = None
        if self.held is not None:
            self.cache = sq.make_cache(cu(self.cK).view(sq.F8), cu(self.cV).view(sq.F8), cu(self.cks.astype(np.float32)), cu(self.cvs.astype(np.float32)), cu(self.table))
        self.out = torch.full((B, H * G, T, 128), 9.0, dtype=F16, device="cuda")
        self.lse = torch.full((B, H * G, T), 9.0, dtype=F32, device="cuda")
        self.ws = sq.workspace(self.shape, sq.SQ_CALL_TREE_ATTN_Q8, "cuda:0")
        self.args = [self.shape, T, cu(self.q), *fixed, self.cache, opt(self.held), opt(self.Kd), opt(self.Vd), opt(self.mask), opt(self.n)]
        return self

    def call(self, lse=True):
        sq.sq_tree_attn_q8(*self.args, self.out, self.lse if lse else None, self.ws)

    def check(self, skip=()):
        B, H, G, T = self.B, self.H, self.G, self.T
        out, lse = self.out.cpu().numpy().astype(np.float64), self.lse.cpu().numpy().astype(np.float64)
        for b in range(B):
            for h in range(H):
                if (b, h) in skip:
                    continue
                keys, n = self.keys(b, h)
                assert (out[b, h * G:h * G + G, n:] == 9).all() and (lse[b, h * G:h * G + G, n:] == 9).all()
                if n == 0:
                    continue
                rows = self.q[b, h * G:h * G + G, :n].transpose(1, 0, 2).reshape(n * G, 128).astype(np.float64)
                o, z, off, off_z = plain.attend(rows, keys, SCALE)
                back = lambda x: x.reshape(n, G, -1).transpose(1, 0, 2)  # noqa: E731
                got, got_z = out[b, h * G:h * G + G, :n], lse[b, h * G:h * G + G, :n, None]
                o, z, off, off_z = back(o), back(z), back(off), back(off_z)
                fine = np.isfinite(o) & (np.abs(o) < 65520)     # (past it f16 ends)
                border = np.abs(np.abs(o) - 65520) <= off
                assert (border | (fine == np.isfinite(got))).all(), (b, h, "not finite elsewhere")
                fine &= ~border
                with np.errstate(invalid="ignore"):
                    bad = np.argwhere(fine & (np.abs(got - o) > off))
                    assert not len(bad), (b, h, bad[:4], got[tuple(bad[0])], o[tuple(bad[0])], off[tuple(bad[0])])
                    assert np.array_equal(np.isneginf(z), np.isneginf(got_z))
                    ok = np.isfinite(z)
                    assert (np.abs(got_z - z)[ok] <= off_z[ok]).all(), (b, h, np.abs(got_z - z)[ok].max(), off_z[ok].max())

    def run(self):
        self.upload().call()
        self.check()


@pytest.mark.parametrize("B,H,G,T,L,C,user,page,mask,ragged", [
    (1, 1, 1, 1, 64, 2, 1, 16, "tree", False),                   # one of everything
    (1, 2, 1, 1, 300, 9, 40, 64, None, False),
    (2, 4, 1, 8, 1000, 30, 70, 16, "tree", False),               # 8 rows
    (3, 2, 3, 5, 777, 20, 33, 32, "any", True),                  # 15 rows, a row that sees no draft
    (2, 3, 4, 7, 2000, 50, 200, 64, "tree", True),               # 28
    (1, 2, 8, 4, 500, 12, 31, 16, "any", False),                 # 32
    (2, 2, 1, 33, 1500, 40, 64, 32, "any", True),                # 33, a mask of two words
    (2, 3, 4, 13, 3000, 90, 500, 16, "tree", True),              # 52
    (2, 2, 5, 13, 900, 25, 100, 64, "any", True),                # 65: rows of their own for two waves
    (1, 3, 5, 25, 1200, 33, 65, 32, "tree", False),              # 125
    (2, 1, 43, 3, 600, 11, 17, 16, None, True),                  # 129, heads of a draft in two waves
    (1, 2, 4, 64, 2500, 80, 300, 64, "tree", False),             # 256
    (2, 2, 3, 97, 700, 21, 90, 16, "any", True),                 # 291: two blocks
    (3, 1, 8, 67, 640, 10, 40, 32, None, True),                  # 536, a chain
    (1, 1, 4, 300, 1000, 30, 129, 64, None, False),              # 1200, a chain of ten tiles
    (2, 1, 2, 201, 300, 8, 20, 16, "any", True),
])
def test_sizes(B, H, G, T, L, C, user, page, mask, ragged):
    Problem(T * 31 + G, B, H, G, T, L, C, user=user, page=page, mask=mask, ragged=ragged).run()


@pytest.mark.parametrize("B,H,G,T,mask,ragged", [(1, 2, 4, 16, "tree", False), (2, 3, 4, 9, "any", True), (3, 2, 3, 25, None, True), (2, 1, 8, 30, "tree", True)])
def test_tables_of_many_pages(B, H, G, T, mask, ragged):
    """Room for 2M tokens a sequence, the most that there can be, few of them there: the most keys that there can be choose the size of a block, 48 or 64 rows here."""
    p = Problem(B * T, B, H, G, T, L=700, C=20, user=90, mask=mask, ragged=ragged)
    p.table = np.concatenate([p.table, np.full((B, (1 << 21) // 16 - p.table.shape[1]), -1, np.int32)], 1)
    p.run()
    p.held[-1] = 5000                                           # (pages that are none have no keys)
    p.run()


@pytest.mark.parametrize("mask", ["tree", None, "any"])
@pytest.mark.parametrize("sources", ["drafts", "context", "cache", "context+cache", "context+drafts", "cache+drafts"])
def test_sources(sources, mask):
    p = dict(L=400, C=12) if "context" in sources else {}
    p.update(dict(user=90, page=32) if "cache" in sources else {})
    Problem(3, 3, 2, 2, 11, mask=mask, drafts="drafts" in sources, ragged=True, **p).run()


def test_nothing_to_see():
    """Empty kept sets, empty caches, empty masks, no drafts: out 0 and lse -inf, or nothing written."""
    p = Problem(1, 4, 2, 2, 20, L=300, C=10, user=40, mask="any")
    p.bits[:] = False
    p.bits[1, 3, 5] = True
    p.mask = plain.words(p.bits)
    p.nr[:], p.nk[:], p.held[:] = 0, 0, 0
    p.held[2] = 7
    p.n = np.array([20, 6, 20, 0], np.int32)
    p.run()
    p = Problem(1, 2, 2, 2, 20, L=300, C=10, user=40, ragged=True)
    p.n[:] = [0, -3]                                            # no drafts at all
    p.run()
    p = Problem(2, 2, 2, 2, 20, L=300, C=10, user=40, ragged=True)
    p.n[:] = [100, 1 << 30]                                     # more than there are: all
    p.run()


def test_pages_that_are_none_and_lengths_past_the_table():
    p = Problem(5, 3, 2, 3, 9, L=200, C=6, user=150, page=16)
    p.table[0, 2], p.table[0, 7], p.table[1, 0] = -1, len(p.cK), 1 << 30
    p.held[:] = [150, 100000, -5]
    p.run()
    p = Problem(6, 2, 1, 2, 3, user=64, page=16, drafts=False)
    p.table[:] = -1                                             # no key at all
    p.held[:] = 64
    p.run()


@pytest.mark.parametrize("scales", [(-64, -50), (-64, 41), (0, 10)])
def test_scales(scales):
    p = Problem(7, 2, 2, 2, 17, L=700, C=20, user=100, page=32, scales=scales)
    if scales == (-64, 41):                                     # keys keep scores in reach; values as far apart as they get
        p.ks, p.cks = np.full_like(p.ks, 2.0 ** -6), np.full_like(p.cks, 2.0 ** -6)
        p.Vd[:] = 0                                             # (f16 drafts beside values of 2^40)
    p.run()


def test_scales_that_are_no_powers_of_two():
    p = Problem(8, 2, 2, 2, 17, L=700, C=20, user=100, page=32)
    for a in (p.ks, p.vs, p.cks, p.cvs):
        a[:] = (a * p.rng.uniform(0.5, 2, a.shape)).astype(np.float32)
    p.run()


def test_large_scores():
    """One key has nearly all of the weight, a different one for each row."""
    p = Problem(9, 2, 2, 4, 20, L=900, C=30, user=100, page=64)
    p.q *= np.float16(40)
    p.run()


@pytest.mark.parametrize("where", ["K", "V"])
@pytest.mark.parametrize("what", [np.nan, np.inf, -np.inf])
def test_drafts_that_are_not_finite(where, what):
    """They reach the rows that see them and no others, infinities of V those alone with their sign."""
    p = Problem(10, 2, 2, 3, 40, L=300, C=10, user=50, mask="any")
    x = p.Kd if where == "K" else p.Vd
    for j in (0, 17, 33, 39):
        x[:, :, j, j] = what
    p.upload().call()
    out = p.out.cpu().numpy()
    for b in range(2):
        hit = p.bits[b][:, [0, 17, 33, 39]]
        for h in range(2):
            got = out[b, h * 3:h * 3 + 3]
            if where == "K":
                assert np.array_equal(np.isfinite(got).all((0, 2)), ~hit.any(1)) or np.isinf(what)
            else:
                for i, j in enumerate((0, 17, 33, 39)):
                    assert not np.isfinite(got[:, hit[:, i], j]).any()
    clean = Problem(10, 2, 2, 3, 40, L=300, C=10, user=50, mask="any")
    (clean.Kd if where == "K" else clean.Vd)[:] = np.where(np.isfinite(x), x, 0)
    clean.upload().call()
    other = clean.out.cpu().numpy()
    for b in range(2):                                          # rows that see none of them: the same bits as beside zeros
        rows = ~p.bits[b][:, [0, 17, 33, 39]].any(1)
        assert rows.any() and np.array_equal(out[b][:, rows], other[b][:, rows])
    if where == "V":                                            # and the other dimensions of those that do
        dims = np.setdiff1d(np.arange(128), (0, 17, 33, 39))
        assert np.array_equal(out[..., dims], other[..., dims])


def test_codes_that_are_not_finite():
    """A NaN code reaches every row of its (sequence, head); codes behind the last key reach nobody."""
    p = Problem(11, 2, 2, 2, 9, L=300, C=10, user=50, page=16, mask="tree")
    p.held[:] = [50, 37]
    spare = np.setdiff1d(np.arange(len(p.cK)), p.table)
    p.cK[spare], p.cV[spare] = 0x7f, 0xff
    for b in range(2):
        last = p.table[b, p.held[b] // 16]
        p.cK[last, :, p.held[b] % 16:], p.cV[last, :, p.held[b] % 16:] = 0x7f, 0x7f
    unkept = np.ones((2, 300), bool)
    for b in range(2):
        for h in range(2):
            for s, c in p.ranges[b, h, :p.nr[b, h]]:
                unkept[h, s:s + c] = False
    p.K8[unkept], p.V8[unkept] = 0x7f, 0x7f
    p.run()
    p.cV[p.table[1, 0], 1, 3, 77] = 0x7f
    p.run()
    got = p.out.cpu().numpy()
    assert np.isnan(got[1, 2:, :, 77]).all() and np.isfinite(got[0]).all() and np.isfinite(got[1, :2]).all()


def test_queries_that_are_not_finite_reach_their_own_rows():
    p = Problem(12, 2, 2, 2, 30, L=300, C=10, user=50, mask="tree")
    p.upload().call()
    clean = p.out.cpu().numpy()
    p.q[1, 2, 7, 5], p.q[0, 0, 29, 100] = np.nan, np.inf
    p.upload().call()
    got = p.out.cpu().numpy()
    same = (got == clean).all(-1)
    assert not np.isfinite(got[1, 2, 7]).any() and same.sum() == same.size - 2 and not same[1, 2, 7] and not same[0, 0, 29]


@pytest.mark.parametrize("C,keep", [(300, 0.9), (2000, 0.5), (16384, 0.4), (16384, 1.0)])
def test_many_ranges(C, keep):
    """More than the four groups of 64 that fit registers elsewhere, up to the most there can be; empty ranges between them."""
    p = Problem(C, 1, 2, 2, 6, L=20000, C=C, keep=keep, user=40)
    p.run()
    p = Problem(C + 1, 1, 1, 1, 3, L=20000, C=C, keep=keep)
    p.ranges = np.ascontiguousarray(np.insert(p.ranges[:, :, :p.nr[0, 0]], slice(0, p.nr[0, 0], 3), 0, 2)[:, :, :C])
    p.nr[0, 0] = p.ranges.shape[2]
    pad = np.zeros((1, 1, C - p.nr[0, 0], 2), np.int32)
    p.ranges = np.concatenate([p.ranges, pad], 2)
    p.nk[0, 0] = p.ranges[0, 0, :, 1].sum()
    p.run()


@pytest.mark.parametrize("B,H,T", [(16, 32, 2), (40, 16, 1), (9, 60, 17), (33, 64, 1), (19, 111, 3)])
def test_many_sequences_and_heads(B, H, T):
    """Up to 2048 blocks in shares, more of them with a workgroup each."""
    Problem(B, B, H, 2, T, L=200, C=9, user=30, ragged=True).run()


def test_long_rows_with_a_workgroup_per_block():
    Problem(22, 2, 17, 16, 300, L=150, C=9, user=40, mask=None, ragged=True).run()   # 2 x 17 x 75 blocks


def test_more_blocks_than_threads():
    """Shares of up to 511 blocks: several a thread where they are divided."""
    Problem(20, 27, 17, 1, 5, L=300, C=9, user=100, ragged=True).run()
    Problem(21, 5, 2, 16, 130, L=100, C=5, user=10, mask=None, ragged=True).run()


def test_input_outside_the_contract_does_not_fault():
    """Wrong counts, ranges out of bounds or in disorder: nothing outside the tensors is read, other heads have their result."""
    p = Problem(13, 2, 2, 2, 9, L=500, C=16, user=50)
    good = [x.copy() for x in (p.ranges, p.nr, p.nk)]
    for bad in range(7):
        p.ranges, p.nr, p.nk = (x.copy() for x in good)
        if bad == 0:
            p.nk[0, 0] = 1 << 30
        elif bad == 1:
            p.nk[0, 0] = -4
        elif bad == 2:
            p.nr[0, 0] = 1 << 30
        elif bad == 3:
            p.nr[0, 0] = -1
        elif bad == 4:
            p.ranges[0, 0, :, 0] = np.iinfo(np.int32).max - 5
            p.nr[0, 0] = 16
        elif bad == 5:
            p.ranges[0, 0, :, 1] = np.iinfo(np.int32).max
            p.nr[0, 0], p.nk[0, 0] = 16, 500
        else:
            p.ranges[0, 0, :, 0], p.ranges[0, 0, :, 1] = -1000, 600
            p.nr[0, 0], p.nk[0, 0] = 16, 500
        p.upload().call()
        torch.cuda.synchronize()
        p.check(skip=[(0, 0)])


def test_without_lse_and_with_scratch_that_holds_anything():
    p = Problem(14, 2, 3, 4, 30, L=1000, C=30, user=100).upload()
    p.call()
    want, lse = p.out.clone(), p.lse.clone()
    p.ws.fill_(0xff)                                            # NaN wherever a float is read
    p.out.fill_(9)
    p.lse.fill_(9)
    p.call()
    assert torch.equal(p.out, want) and torch.equal(p.lse, lse)
    p.out.fill_(9)
    p.lse.fill_(9)
    p.call(lse=False)
    assert torch.equal(p.out, want) and (p.lse == 9).all()


def test_one_draft_agrees_with_the_decode_call():
    """T = 1 with the draft's key appended to the cache is a decode step with one kept set."""
    p = Problem(15, 3, 4, 4, 1, L=1000, C=40, user=64, page=32, mask=None, drafts=False).upload()
    p.call()
    sh = sq.make_shape(3, 4, 1000, 40, 4, 0, SCALE)
    out, lse = torch.empty(3, 16, 1, 128, dtype=F16, device="cuda"), torch.empty(3, 16, 1, device="cuda")
    sq.sq_sparse_attn_decode_q8(sh, True, *p.args[2:10], p.cache, p.args[11], out, lse, sq.workspace(sh, sq.SQ_CALL_ATTN_DECODE_Q8, "cuda:0"))
    assert ((out.view(3, 16, 1, 128).float() - p.out.float()).abs() <= 2.0 ** -10 * 4).all() and (lse.view(3, 16, 1) - p.lse).abs().max() < 1e-5


def test_two_streams_and_captured_graphs():
    """Two calls at once with workspaces of their own; a captured call replayed on new inputs, with other work between the replays."""
    a, b = (Problem(s, 2, 2, 4, 20, L=800, C=20, user=90).upload() for s in (16, 17))
    want = []
    for p in (a, b):
        p.ws = torch.empty_like(p.ws)
        p.call()
        want.append(p.out.clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for p, s in zip((a, b), streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                p.out.fill_(9)
                p.call()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.call()
    for turn in range(4):
        a.args[2].copy_(torch.randn(a.q.shape, generator=torch.Generator().manual_seed(turn)).half())
        a.args[11].copy_(cu(np.array([90 - turn, 11 * turn], np.int32)))
        a.out.fill_(9)
        graph.replay()
        b.call()
        torch.cuda.synchronize()
        got = a.out.clone()
        a.call()
        assert torch.equal(a.out, got) and torch.equal(b.out, want[1])


def test_the_binding_refuses_tensors_that_do_not_fit():
    p = Problem(18, 2, 3, 2, 6, L=100, C=5, user=20).upload()
    names = ["shape", "T", "q", "K8", "V8", "ks", "vs", "ranges", "nr", "nk", "cache", "held", "Kd", "Vd", "mask", "n"]
    good = dict(zip(names, p.args), out=p.out, lse=p.lse, ws=p.ws)
    call = lambda **kw: sq.sq_tree_attn_q8(*{**good, **kw}.values())  # noqa: E731
    call()
    t = lambda *s, dtype=F16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    for bad in (dict(q=t(2, 6, 5, 128)), dict(K8=t(3, 100, 128)), dict(Kd=t(2, 3, 6, 128, dtype=F32)), dict(Vd=t(2, 6, 3, 128).transpose(1, 2)),
                dict(mask=t(2, 6, 2, dtype=I32)), dict(n=torch.zeros(2, dtype=I32)), dict(n=t(3, dtype=I32)), dict(out=t(2, 6, 6, 128).transpose(1, 2)),
                dict(lse=t(2, 6, 6)), dict(ranges=t(6, 2, 5, 2, dtype=I32)), dict(held=t(2, dtype=torch.int64))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ValueError):
        call(T=5)                                               # (what the drafts' tensors then ought to hold)
    with pytest.raises(sq.SqError):
        call(T=5, Kd=None, Vd=None, mask=None)
    with pytest.raises(sq.SqError):
        call(ws=None)
    torch.cuda.synchronize()


@pytest.mark.parametrize("G,T", [(1, 8), (4, 7), (3, 15), (4, 40), (8, 100)])
def test_a_pool_of_more_than_4_gb(G, T):
    """Pages behind the reach of 32-bit offsets, for each size of a block of rows."""
    B, H, P = 9, 8, 64
    n = (1 << 32) // (H * P * 128) + 40
    p = Problem(G * T, B, H, G, T, L=400, C=9, user=150, page=P, ragged=True)
    used = B * p.table.shape[1]
    local = p.table.copy()
    p.upload()
    K8, V8 = (torch.zeros(n, H, P, 128, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.ones(n, H, device="cuda") for _ in range(2))
    far = (n - 1 - p.rng.permutation(used + 2)).astype(np.int32)                # page i of the small pool is page far[i] of the large one
    at = torch.from_numpy(far).cuda().long()
    for big, small in ((K8, p.cK), (V8, p.cV), (ks, p.cks.astype(np.float32)), (vs, p.cvs.astype(np.float32))):
        big[at] = cu(small)
    p.args[10] = sq.make_cache(K8.view(sq.F8), V8.view(sq.F8), ks, vs, cu(far[local]))
    p.call()
    p.check()


def test_a_long_chain():
    """5000 drafts of a prompt, 3 heads: checked at the rows where blocks, tiles and words end."""
    p = Problem(23, 1, 1, 3, 5000, L=600, C=20, user=200, page=32, mask=None).upload()
    p.call()
    keys, _ = p.keys(0, 0)
    q = p.q[0].transpose(1, 0, 2).reshape(15000, 128).astype(np.float64)
    out = p.out.cpu().numpy()[0].transpose(1, 0, 2).reshape(15000, 128).astype(np.float64)
    lse = p.lse.cpu().numpy()[0].T.reshape(15000)
    rows = np.unique(np.concatenate([[0, 1, 2, 3, 63, 64, 65, 95, 96, 97, 14997, 14998, 14999], p.rng.integers(0, 15000, 60)]))
    picked = [(k, v, None if seen is None else seen[rows], s) for k, v, seen, s in keys]
    o, z, off, off_z = plain.attend(q[rows], picked, SCALE)
    assert (np.abs(out[rows] - o) <= off).all() and (np.abs(lse[rows] - z) <= off_z).all()


def test_a_mask_of_many_words():
    """700 drafts in random order of sight: 22 words a row."""
    Problem(24, 1, 1, 2, 700, L=100, C=4, user=33, mask="any").run()


def test_masks_larger_than_their_offsets_reach_are_refused():
    p = Problem(25, 1, 1, 1, 4, user=16).upload()
    shape = sq.make_shape(1, 1, 1, 1, 32769, 0, SCALE)
    t = lambda *s, dtype=F16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    q, K, mask = t(1, 1, 32769, 128), t(1, 1, 32769, 128), t(1, 32769, 1025, dtype=I32)
    ws = sq.workspace(shape, sq.SQ_CALL_TREE_ATTN_Q8, "cuda:0")
    with pytest.raises(sq.SqError, match="too large"):
        sq.sq_tree_attn_q8(shape, 32769, q, *[None] * 7, p.cache, p.args[11], K, K, mask, None, t(1, 1, 32769, 128), None, ws)
