"""sq_sparse_attn_decode_q8 against a plain 64-bit implementation on the values that the codes stand for."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from paper_2411_09688_amd import binding as sq
from test_gpu_q8_rows import cu

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))


class Problem:
    def __init__(self, seed, B, H, Lq, L, C, keep, lengths, P, one_set, spread=0):
        """keep: share of the clusters that a row keeps (None: no fixed context); lengths: tokens per sequence (None: no cache);
        spread: the scales' exponents range over this much."""
        rng = self.rng = np.random.default_rng(seed)
        self.B, self.H, self.Lq, self.L, self.C, self.P, self.one_set = B, H, Lq, L, C, P, one_set
        self.q = (1.5 * rng.standard_normal((B, H * Lq, 128))).astype(np.float16)
        R = self.rows = B * H * (1 if one_set else Lq)
        scales = lambda *s: 2.0 ** (-7 + rng.integers(-spread, spread + 1, s)).astype(np.float64) * (1.1 if spread else 1.0)  # noqa: E731

        def codes(*s):
            if np.prod(s) < 1 << 22:
                return ref.encode((rng.standard_normal(s) * 64).clip(-448, 448))
            c = rng.integers(0, 256, s, np.uint8)               # (quicker: codes of any exponent)
            c[(c & 0x7f) == 0x7f] = 0x35
            return c

        self.fixed = self.cache = None
        if keep is not None:
            n = -(-L // 64)
            self.fixed = [codes(H, L, 128), codes(H, L, 128), 2.0 ** -7 * np.ones((H, n)), scales(H, n)]
            ends = np.sort(np.concatenate([rng.integers(0, L + 1, (H, C - 1)), np.full((H, 1), L)], 1), 1)
            first = np.concatenate([np.zeros((H, 1), int), ends[:, :-1]], 1)
            self.ranges, self.n_ranges = np.zeros((R, C, 2), np.int32), np.zeros(R, np.int32)
            for r in range(R):
                h = r // (1 if one_set else Lq) % H
                f = keep if np.isscalar(keep) else keep[r % len(keep)]
                kept = np.flatnonzero((rng.random(C) < f) & (ends[h] > first[h]))
                self.n_ranges[r] = len(kept)
                self.ranges[r, :len(kept), 0] = first[h, kept]
                self.ranges[r, :len(kept), 1] = (ends[h] - first[h])[kept]
            self.n_keys = self.ranges[:, :, 1].sum(1).astype(np.int32)
        if lengths is not None:
            width = max(1, -(-max(lengths) // P))
            n = B * width + 1
            self.lengths = np.asarray(lengths, np.int32)
            self.table = rng.permutation(n)[:B * width].reshape(B, width).astype(np.int32)
            self.cache = [codes(n, H, P, 128), codes(n, H, P, 128), 2.0 ** -7 * np.ones((n, H)), scales(n, H)]
            for b in range(B):                                  # what lies behind a sequence's last token is not read: NaN
                for t in range(lengths[b], width * P):
                    for c in self.cache[:2]:
                        c[self.table[b, t // P], :, t % P] = 0x7f

    def keys(self, r):
        """The keys and values that a row sees, and the pieces its values came in."""
        h, b = r // (1 if self.one_set else self.Lq) % self.H, r // (self.rows // self.B)
        k, v = [np.zeros((0, 128))], [np.zeros((0, 128))]
        if self.fixed is not None:
            ids = []
            for s, c in self.ranges[r, :min(max(self.n_ranges[r], 0), self.C)]:
                ids += [i for i in range(int(s), int(s) + max(0, int(c)))]
            ids = np.clip(np.asarray(ids[:min(max(int(self.n_keys[r]), 0), self.L)], int), 0, self.L - 1)
            K, V, ks, vs = self.fixed
            k.append(ref.VALUES[K[h, ids]] * ks[h, ids // 64][:, None].astype(np.float32))
            v.append(ref.VALUES[V[h, ids]] * vs[h, ids // 64][:, None].astype(np.float32))
        if self.cache is not None:
            K, V, ks, vs = self.cache
            for t in range(min(max(int(self.lengths[b]), 0), self.table.shape[1] * self.P)):
                page = self.table[b, t // self.P]
                if 0 <= page < len(K):
                    k.append(ref.VALUES[K[page, h, t % self.P]][None] * np.float32(ks[page, h]))
                    v.append(ref.VALUES[V[page, h, t % self.P]][None] * np.float32(vs[page, h]))
        return np.concatenate(k), np.concatenate(v)

    def upload(self):
        f8 = lambda c: cu(c).view(sq.F8)  # noqa: E731
        f32 = lambda s: cu(s.astype(np.float32))  # noqa: E731
        self.sh = sq.make_shape(self.B, self.H, self.L, self.C, self.Lq, 0, SCALE)
        fixed = [None] * 7
        if self.fixed is not None:
            K, V, ks, vs = self.fixed
            fixed = [f8(K), f8(V), f32(ks), f32(vs), cu(self.ranges), cu(self.n_ranges), cu(self.n_keys)]
        cache = seq = None
        if self.cache is not None:
            K, V, ks, vs = self.cache
            cache, seq = sq.make_cache(f8(K), f8(V), f32(ks), f32(vs), cu(self.table)), cu(self.lengths)
        self.out = torch.full((self.B, self.H * self.Lq, 1, 128), 9.0, dtype=torch.float16, device="cuda")
        self.lse = torch.full((self.B, self.H * self.Lq, 1), 9.0, device="cuda")
        self.ws = sq.workspace(self.sh, sq.SQ_CALL_ATTN_DECODE_Q8, "cuda:0")
        return (self.sh, self.one_set, cu(self.q), *fixed, cache, seq)

    def check(self, out=None, lse=None, rows=None):
        out = (self.out if out is None else out).cpu().numpy().astype(np.float64).reshape(-1, 128)
        lse = (self.lse if lse is None else lse).cpu().numpy().reshape(-1)
        g = self.Lq if self.one_set else 1
        q = self.q.reshape(-1, 128).astype(np.float64)
        for r in range(self.rows) if rows is None else rows:
            k, v = self.keys(r)
            at = slice(r * g, r * g + g)
            o, z, moved = ref.attend(q[at], k, v, SCALE)
            if len(k) == 0:
                assert (out[at] == 0).all() and (lse[at] == -np.inf).all(), r
                continue
            # one rounding to f16, and what fp32 may have moved
            off = np.abs(out[at] - o) - np.abs(o) * 2.0 ** -11 - 2.0 ** -25
            assert (off <= moved[:, :1]).all(), (r, off.max(), moved)
            assert (np.abs(lse[at] - z) <= moved[:, 1] + np.abs(z) * 2.0 ** -22).all(), (r, lse[at], z)


CASES = [  # B, H, Lq, L, C, keep, lengths, page, one_set, spread
    (1, 1, 1, 1, 1, 1.0, None, 16, False, 0),                              # one key
    (1, 1, 1, 64, 2, None, [1], 16, False, 0),                             # one token, nothing else
    (1, 4, 1, 4096, 64, 0.25, [128], 64, False, 0),
    (2, 3, 1, 1000, 31, [0.0, 0.3, 1.0], [0, 37], 16, False, 3),           # rows that keep nothing and see nobody
    (3, 2, 4, 777, 25, [0.2, 0.9, 0.0], [5, 0, 300], 32, False, 0),        # a kept set per query head
    (3, 2, 4, 777, 25, [0.2, 0.9, 0.0], [5, 0, 300], 32, True, 2),         # ... per K/V head
    (1, 2, 16, 300, 300, 0.5, [65], 64, True, 0),                          # clusters of one key; 16 query heads
    (2, 1, 13, 50, 3, None, [31, 33], 16, True, 0),
    (5, 1, 7, 129, 4, 1.0, None, 16, True, 20),                            # everything kept; scales 2^40 apart
    (1, 1, 1, 70001, 1, 1.0, [33], 16, False, 0),                          # one cluster of everything over many workgroups
    (1, 2, 2, 40000, 9000, [0.4, 0.02], [3000], 64, False, 0),             # more than one batch of ranges
    (300, 2, 2, 100, 5, [0.5, 0.0], [i % 40 for i in range(300)], 16, False, 0),   # more rows than workgroups
    (7, 5, 3, 64, 4, 0.6, [100] * 7, 32, True, 0),
    # eight rows or more of a head with two million keys to select from between them: keys that several rows keep are read once
    (16, 1, 1, 140001, 4000, [0.02, 0.0, 0.005], [0, 1, 64, 65, 200, 7, 31, 130] * 2, 32, False, 3),   # a last window of 225 keys
    (17, 1, 1, 131073, 16384, [0.01, 0.03], None, 16, False, 0),           # a group of one row behind one of 16; a window of one key
    (2, 2, 8, 70000, 500, [0.02, 0.0, 0.04], [90, 0], 16, False, 0),
    (9, 2, 2, 131072, 3000, [0.01, 0.03], [3] * 9, 64, True, 2),           # two query heads to a set, eight rows to a group
    (40, 8, 1, 131072, 4096, [0.004, 0.01], [40] * 40, 16, False, 0),      # more windows than are marked at a time
    (8, 8, 1, 131072, 2048, [0.01, 0.0, 0.03], [40, 0] * 4, 16, False, 2),  # a context of 268 MB, and one group: past the caches
    (11, 1, 3, 65536, 16, [0.0] * 30 + [1.0], [3000] + [0] * 10, 16, False, 0),   # one sequence's own; one row of everything
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:6]) if c[0] < 300 else "many rows")
def test_decode(case):
    p = Problem(sum(case[:5]), *case)
    args = p.upload()
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    few = None if p.rows <= 64 and p.L < 60000 else list(range(0, p.rows, 37 if p.rows > 64 else 5)) + [p.rows - 1]
    p.check(rows=few)
    out, lse = p.out.clone(), p.lse.clone()
    p.ws.fill_(255)                                             # whatever the workspace holds; without lse; the same bits
    p.out.fill_(9.0)
    sq.sq_sparse_attn_decode_q8(*args, p.out, None, p.ws)
    assert torch.equal(p.out, out) and torch.equal(p.lse, lse)


def test_scales_of_any_size():
    """Values whose scales are far outside f16's range, and no powers of two."""
    p = Problem(11, 1, 2, 2, 500, 10, 0.5, [70], 16, True)
    p.fixed[3][:] = 1e-9 * (1 + p.rng.random(p.fixed[3].shape))
    p.cache[3][:] = 3e-9
    args = p.upload()
    out, lse = p.out, p.lse
    sq.sq_sparse_attn_decode_q8(*args, out, lse, p.ws)
    big = Problem(11, 1, 2, 2, 500, 10, 0.5, [70], 16, True)
    big.fixed[3][:], big.cache[3][:] = p.fixed[3] * 2.0 ** 30, p.cache[3] * 2.0 ** 30
    args = big.upload()
    sq.sq_sparse_attn_decode_q8(*args, big.out, big.lse, big.ws)
    big.check()
    p.check()                                                   # (these outputs are subnormal in f16)


def test_nan_reaches_the_queries_that_see_it_only():
    p = Problem(12, 2, 2, 2, 256, 4, 1.0, [40, 20], 16, False)
    p.ranges[:] = 0
    for r in range(p.rows):                                     # rows keep the first or the second half
        p.ranges[r, 0] = (0, 128) if r % 2 else (128, 128)
    p.n_ranges[:], p.n_keys[:] = 1, 128
    args = p.upload()
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    p.check()
    clean = p.out.clone().reshape(p.rows, 128)
    p.fixed[0][0, 5, 3] = 0x7f                                  # a key of head 0 that the odd rows see
    p.fixed[1][1, 200, 9] = 0xff                                # a value of head 1 that the even rows see
    args = p.upload()
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    got = p.out.reshape(p.rows, 128)
    for r in range(p.rows):
        h = r // 2 % 2
        if h == 0 and r % 2:
            assert torch.isnan(got[r]).all()
        elif h == 1 and r % 2 == 0:
            assert torch.isnan(got[r, 9]) and torch.equal(got[r, 10:], clean[r, 10:]) and torch.equal(got[r, :9], clean[r, :9])
        else:
            assert torch.equal(got[r], clean[r])


def test_nan_reaches_the_rows_of_a_group_that_see_it_only():
    """Twelve rows share a head, and each other's tiles: a NaN in a value that some of them keep, and in a user's own value."""
    p = Problem(22, 6, 1, 2, 180000, 64, [0.05, 0.03], [70, 5, 40, 0, 64, 9], 16, False)
    args = p.upload()
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    p.check()
    clean, lse = p.out.clone().reshape(p.rows, 128), p.lse.clone()
    key = int(next(p.ranges[r, 0, 0] for r in range(p.rows) if p.n_ranges[r]))
    sees = [any(s <= key < s + c for s, c in p.ranges[r, :p.n_ranges[r]]) for r in range(p.rows)]
    assert 1 <= sum(sees) <= 10
    p.fixed[1][0, key, 77] = 0x7f
    p.cache[1][p.table[2, 1], 0, 3, 5] = 0xff                   # token 19 of sequence 2: rows 4 and 5
    args = p.upload()
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    got = p.out.reshape(p.rows, 128)
    for r in range(p.rows):
        want = clean[r].clone()
        if sees[r]:
            want[77] = float("nan")
        if r in (4, 5):
            want[5] = float("nan")
        assert torch.equal(torch.isnan(got[r]), torch.isnan(want)), r
        ok = ~torch.isnan(want)
        assert (got[r][ok].float() - want[ok].float()).abs().max() <= 2.0 ** -9 * want[ok].float().abs().max(), r
    assert torch.isfinite(p.lse).all()


def test_input_outside_the_contract_stays_inside_the_tensors():
    p = Problem(13, 2, 2, 1, 300, 12, 0.6, [50, 90], 16, False)
    p.table[0, 1], p.table[1, 0], p.table[1, 5] = -1, 10 ** 8, -2 ** 31   # no pages: their tokens are not there
    p.ranges[0, 0] = (-4, 9)                                    # rows outside: the nearest
    p.ranges[1, 0] = (296, 20)
    p.ranges[2, 1, 1] = -5                                      # skipped
    for r in range(3):
        p.n_keys[r] = p.ranges[r, :p.n_ranges[r], 1].clip(0).sum()
    p.n_keys[3] -= 7                                            # fewer than listed: the first of them
    args = p.upload()
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    p.check()
    p.n_keys[3] += 50                                           # more than listed: those there are
    p.n_keys[0], p.n_ranges[1], p.n_ranges[2] = -3, 1000, -1
    p.n_keys[1] = p.ranges[1, :, 1].clip(0).sum()
    p.lengths[:] = (-8, 10 ** 6)
    args = p.upload()
    for c in args[10].tensors[:2]:
        c.view(torch.uint8)[(c.view(torch.uint8) & 0x7f) == 0x7f] = 0x11
    for i in range(2):
        p.cache[i][(p.cache[i] & 0x7f) == 0x7f] = 0x11
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    p.check()


def test_two_graphs_share_a_workspace_and_a_side_stream():
    p = Problem(14, 4, 2, 4, 3000, 100, 0.3, [100, 7, 0, 333], 16, True)
    args = p.upload()
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    want = p.out.clone()
    p.check()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    p.out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(p.out, want)
    o = Problem(15, 1, 3, 2, 900, 30, 0.5, [64], 64, False)
    oargs = o.upload()
    ws = torch.empty(max(p.ws.numel(), o.ws.numel()), dtype=torch.uint8, device="cuda")
    graphs = []
    for a, x in ((args, p), (oargs, o)):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sq.sq_sparse_attn_decode_q8(*a, x.out, x.lse, ws)
        graphs.append(g)
    for _ in range(3):
        p.out.zero_(), o.out.zero_()
        graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        assert torch.equal(p.out, want)
        o.check()


def test_a_group_of_rows_with_input_outside_the_contract():
    """Rows whose ranges lie outside the context, overlap or are too many; the group's other rows are as they would be."""
    p = Problem(16, 16, 1, 1, 140001, 900, 0.01, [70] * 16, 16, False)
    p.ranges[1, :3] = ((-5, 40), (140000, 50), (2 ** 31 - 1, 2 ** 31 - 1))
    p.ranges[2, :2] = ((-2 ** 31, 2 ** 31 - 1), (100, -3))
    p.ranges[3, :4] = ((7, 100), (50, 100), (7, 100), (0, 1))
    p.n_ranges[4], p.n_ranges[5] = 10 ** 9, -4
    p.n_keys[6], p.n_keys[7] = -1, 10 ** 9
    p.table[8, 1] = -1
    args = p.upload()
    p.lengths[9] = 80                                           # (all of the pages there are, for the reference)
    args[11][9] = 10 ** 9
    for c in args[10].tensors[:2]:                              # (behind the last token: what a reused page holds)
        c.view(torch.uint8)[(c.view(torch.uint8) & 0x7f) == 0x7f] = 0x11
    for i in range(2):
        p.cache[i][(p.cache[i] & 0x7f) == 0x7f] = 0x11
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    torch.cuda.synchronize()
    p.check(rows=[0] + list(range(8, 16)))
    assert torch.isfinite(p.out).all() and torch.isfinite(p.lse).all()


def test_two_calls_at_once_and_a_captured_group():
    """A group of rows captured and replayed for rows that change, while another call runs on a stream and workspace of its own."""
    p = Problem(17, 16, 1, 1, 140001, 900, 0.01, [20, 0, 65, 300] * 4, 16, False)
    args = p.upload()
    o = Problem(18, 1, 3, 2, 9000, 300, 0.5, [64], 64, False)
    oargs = o.upload()
    sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
    side = torch.cuda.Stream()
    lengths = p.lengths.copy()
    for i in range(4):
        p.lengths = (lengths * (i + 1) // 4).astype(np.int32)
        p.n_ranges[i], p.n_keys[i] = 0, 0
        for t, x in ((args[11], p.lengths), (args[8], p.n_ranges), (args[9], p.n_keys)):
            t.copy_(cu(x).view(t.shape))
        p.out.fill_(9.0), o.out.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        sq.sq_sparse_attn_decode_q8(*oargs, o.out, o.lse, o.ws, stream=side)
        torch.cuda.synchronize()
        p.check(rows=[i, 5, 11, 15])
        o.check()
        again = p.out.clone()
        sq.sq_sparse_attn_decode_q8(*args, p.out, p.lse, p.ws)
        torch.cuda.synchronize()
        assert torch.equal(p.out, again)
