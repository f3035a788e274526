"""The calls on drafted tokens as a serving program makes them: a clustered context in 8 bits, then steps of trees -- masks and positions,
rotation, selection, attention, acceptance, writing what was accepted -- eagerly and as a captured graph; and a finished conversation that
becomes part of a context."""
import numpy as np
import pytest
import torch

import drafts_reference as plain
import q8_reference as ref
from paper_2411_09688_amd import binding as sq
from test_gpu_drafts import forest
from test_gpu_q8_rows import cu, table

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))
F16, F32, I32 = torch.float16, torch.float32, torch.int32


def empty(*s, dtype=F16):
    return torch.zeros(*s, dtype=dtype, device="cuda")


class Server:
    """The buffers of a serving loop with drafts, and one step of it."""

    def __init__(self, seed, B, H, G, T, page, L=700, C=24, capacity=400):
        self.B, self.H, self.G, self.T, self.page, self.L, self.C = B, H, G, T, page, L, C
        rng = np.random.default_rng(seed)
        # the context: clustered, sorted, in 8 bits
        K = cu((rng.standard_normal((1, H, L, 128)) + 2 * rng.standard_normal((1, H, C, 128))[:, :, rng.integers(0, C, L)]).astype(np.float16))
        V = cu(rng.standard_normal((1, H, L, 128)).astype(np.float16))
        flat = sq.make_shape(1, H, L, C, 1, 0, 1.0)
        X = empty(1, H, L, 128)
        sq.sq_kmeans_normalize(flat, K, X)
        centers = X[:, :, :C].contiguous()
        assign, perm = empty(1, H, L, dtype=I32), empty(1, H, L, dtype=I32)
        self.sizes, self.offsets, self.cent = empty(1, H, C, dtype=I32), empty(1, H, C + 1, dtype=I32), empty(1, H, C, 128)
        ws = sq.workspace(flat, sq.SQ_CALL_KMEANS_STEP, "cuda:0")
        for _ in range(2):
            sq.sq_kmeans_step(flat, X, centers, centers, assign, self.sizes, self.offsets, perm, ws)
        Ks, Vs = empty(1, H, L, 128), empty(1, H, L, 128)
        sq.sq_cluster_layout(flat, K, V, perm, self.sizes, self.offsets, Ks, Vs, self.cent)
        n = -(-L // 64)
        self.fixed = [empty(1, H, L, 128, dtype=sq.F8), empty(1, H, L, 128, dtype=sq.F8), empty(1, H, n, dtype=F32), empty(1, H, n, dtype=F32)]
        sq.sq_kv_quantize(flat, K, V, perm, *self.fixed)
        self.value = [ref.VALUES[c.view(torch.uint8).cpu().numpy()[0]] * s.cpu().numpy()[0].repeat(64, 1)[:, :L, None] for c, s in
                      ((self.fixed[0], self.fixed[2]), (self.fixed[1], self.fixed[3]))]
        self.scale_v = self.fixed[3].cpu().numpy()[0].repeat(64, 1)[:, :L].astype(np.float64)
        # the cache
        width = -(-capacity // page)
        self.table = rng.permutation(B * width + 1)[:B * width].reshape(B, width).astype(np.int32)
        self.codes = [np.full((B * width + 1, H, page, 128), 0x7f, np.uint8) for _ in range(2)]
        self.scales = [np.ones((B * width + 1, H)) for _ in range(2)]
        self.cache = sq.make_cache(*(cu(c).view(sq.F8) for c in self.codes), *(cu(s.astype(np.float32)) for s in self.scales), cu(self.table))
        # the step
        self.rot = sq.make_rotary(cu(table(L + capacity + T, 128)))
        self.rows, self.sel = sq.make_shape(B, H, L, C, T, 0, SCALE), sq.make_shape(B, H, L, C, G * T, 0, SCALE)
        self.x = empty(B * T, H * G + 2 * H, 128)
        self.parents, self.tokens, self.target = (empty(B, T, dtype=I32) for _ in range(3))
        self.n, self.held, self.first = (empty(B, dtype=I32) for _ in range(3))
        self.mask, self.positions, self.path = empty(B, T, -(-T // 32), dtype=I32), empty(B, T, dtype=I32), empty(B, T, dtype=I32)
        self.q, self.k, self.v = empty(B, H * G, T, 128), empty(B, H, T, 128), empty(B, H, T, 128)
        self.logits, self.row_max, self.denom = empty(B, H, G * T, C, dtype=F32), empty(B, H, G * T, dtype=F32), empty(B, H, G * T, dtype=F32)
        self.thresh = torch.full((H,), 1.0 / L, device="cuda")
        self.keep, self.ranges, self.nr, self.nk = empty(B, H, -(-C // 32), dtype=I32), empty(B, H, C, 2, dtype=I32), empty(B, H, dtype=I32), empty(B, H, dtype=I32)
        self.out, self.lse = empty(B, H * G, T, 128), empty(B, H * G, T, dtype=F32)
        self.count, self.token, self.new_len = (empty(B, dtype=I32) for _ in range(3))
        # (workspaces of its own: two servers' graphs must not share one)
        self.ws = [torch.empty(max(sq.workspace_bytes(self.sel, w), 256), dtype=torch.uint8, device="cuda") for w in (sq.SQ_CALL_SELECT_MEAN, sq.SQ_CALL_TREE_ATTN_Q8)]

    def draw(self, rng):
        B, T = self.B, self.T
        self.x.copy_(cu(rng.standard_normal(self.x.shape).astype(np.float16)))
        self.parents.copy_(cu(forest(rng, B, T, "tree")))
        self.tokens.copy_(cu(rng.integers(0, 2, (B, T)).astype(np.int32)))
        self.target.copy_(cu(rng.integers(0, 2, (B, T)).astype(np.int32)))
        n = rng.integers(max(1, T // 2), T + 1, B).astype(np.int32)
        n[rng.integers(0, B)] = 0 if B > 1 else T                              # a sequence that pauses
        self.n.copy_(cu(n))

    def step(self):
        H, G = self.H, self.G
        torch.add(self.held, self.L, out=self.first)
        sq.sq_tree_prepare(self.rows, self.parents, self.n, self.first, self.mask, self.positions)
        sq.sq_head_norm_rotate(self.rows, G, self.rot, self.positions, self.x[:, :H * G], self.x[:, H * G:H * G + H], self.x[:, H * G + H:], self.q, self.k, self.v)
        sq.sq_centroid_score(self.sel, self.q, self.cent, self.sizes, self.logits, self.row_max, self.denom)
        sq.sq_select_mean(self.sel, self.logits, self.row_max, self.denom, self.thresh, self.sizes, self.offsets, self.keep, self.ranges, self.nr, self.nk, self.ws[0])
        sq.sq_tree_attn_q8(self.sel, self.T, self.q, *self.fixed, self.ranges, self.nr, self.nk, self.cache, self.held, self.k, self.v, self.mask, self.n, self.out,
                           self.lse, self.ws[1])
        sq.sq_tree_accept(self.rows, self.parents, self.n, self.tokens, self.target, self.held, self.count, self.path, self.token, self.new_len)
        sq.sq_cache_commit(self.rows, self.cache, self.held, self.path, self.count, self.k, self.v)
        self.held.copy_(self.new_len)

    def check(self, held):
        """This step's results from its inputs; `held` before it.  Returns the lengths behind it."""
        B, H, G, T = self.B, self.H, self.G, self.T
        parents, n = self.parents.cpu().numpy(), self.n.cpu().numpy()
        bits, positions = plain.prepare(parents, n, [self.L + x for x in held])
        assert np.array_equal(self.mask.cpu().numpy(), plain.words(bits)) and np.array_equal(self.positions.cpu().numpy(), positions)
        paths = plain.accept(parents, n, self.tokens.cpu().numpy(), self.target.cpu().numpy())
        assert self.count.tolist() == [len(p) for p in paths] and self.held.tolist() == [a + len(p) for a, p in zip(held, paths)]
        q, k, v = (x.cpu().numpy().astype(np.float64) for x in (self.q, self.k, self.v))
        out, lse, rg, nr = self.out.cpu().numpy().astype(np.float64), self.lse.cpu().numpy(), self.ranges.cpu().numpy(), self.nr.cpu().numpy()
        for b in range(B):
            t = np.arange(held[b])
            for h in range(H):
                ids = np.concatenate([np.arange(s, s + c) for s, c in rg[b, h, :nr[b, h]]] + [np.zeros(0, int)]).astype(int)
                assert len(ids) == self.nk[b, h].item()
                at = (self.table[b, t // self.page], h, t % self.page)
                user = [ref.VALUES[self.codes[i][at]] * self.scales[i][at[:2]][:, None] for i in range(2)]
                m = n[b]
                keys = [(self.value[0][h, ids], self.value[1][h, ids], None, self.scale_v[h, ids]), (*user, None, self.scales[1][at[:2]]),
                        (k[b, h, :m], v[b, h, :m], np.repeat(bits[b, :m, :m], G, 0), np.ones(m))]
                if m:
                    o, z, off, off_z = plain.attend(q[b, h * G:h * G + G, :m].transpose(1, 0, 2).reshape(m * G, 128), keys, SCALE)
                    got = out[b, h * G:h * G + G, :m].transpose(1, 0, 2).reshape(m * G, 128)
                    assert (np.abs(got - o) <= off).all()
                    assert (np.abs(lse[b, h * G:h * G + G, :m].T.reshape(m * G) - z) <= off_z).all()
        for i, x in ((0, k), (1, v)):
            plain.commit(self.codes[i], self.scales[i], self.table, list(held), [len(p) for p in paths], [x[b][:, p].transpose(1, 0, 2) for b, p in enumerate(paths)])
            assert ref.same_codes(self.cache.tensors[i].view(torch.uint8).cpu().numpy(), self.codes[i]).all()
            assert np.array_equal(self.cache.tensors[2 + i].cpu().numpy(), self.scales[i].astype(np.float32))
        return [a + len(p) for a, p in zip(held, paths)]


@pytest.mark.parametrize("B,H,G,T,page", [(2, 2, 3, 12, 16), (3, 1, 4, 33, 32), (1, 3, 1, 5, 64)])
def test_a_serving_loop(B, H, G, T, page):
    rng = np.random.default_rng(T)
    s = Server(T, B, H, G, T, page)
    held = [0] * B
    for _ in range(8):
        s.draw(rng)
        s.step()
        held = s.check(held)
    assert max(held) > 8                                        # more than one draft a step was accepted


def test_a_captured_loop():
    """Two servers' steps as graphs, replayed in turn with eager work between them, against the eager loop."""
    made = [Server(s, 2, 2, 4, 14, 16) for s in (1, 2)]
    eager = [Server(s, 2, 2, 4, 14, 16) for s in (1, 2)]
    graphs = []
    for s in made:
        s.draw(np.random.default_rng(0))
        s.step()
        for c, e in zip(s.cache.tensors, (0x7f, 0x7f, 1.0, 1.0)):
            (c.view(torch.uint8) if c.dtype == sq.F8 else c).fill_(e)
        for x in (s.held, s.out, s.lse, s.ranges):              # (rows and entries that a step leaves as they were, too)
            x.zero_()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.step()
        graphs.append(g)
    for turn in range(6):
        for s, e in zip(made, eager):
            for x in (s, e):
                x.draw(np.random.default_rng(10 + turn))
        for g in graphs:
            g.replay()
        for e in eager:
            e.step()
        torch.cuda.synchronize()
        for s, e in zip(made, eager):
            for name in ("mask", "positions", "q", "ranges", "nk", "out", "lse", "path", "count", "token", "held"):
                assert torch.equal(getattr(s, name), getattr(e, name)), (turn, name)
            for x, y in zip(s.cache.tensors, e.cache.tensors):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), turn
    assert min(eager[0].held.tolist()) > 0                      # (each sequence pauses at times)


def test_a_conversation_becomes_context():
    """Read back in 16 bits, what a cache holds prefills (K_user, V_user) and is clustered and quantized like any context."""
    rng = np.random.default_rng(4)
    s = Server(9, 1, 2, 2, 40, 32)
    n = 200
    rows = sq.make_shape(1, 2, 1, 1, n, n, 1.0)
    K, V = (cu(rng.standard_normal((1, 2, n, 128)).astype(np.float16)) for _ in range(2))
    sq.sq_cache_commit(rows, s.cache, cu(np.zeros(1, np.int32)), None, None, K, V)
    back = [empty(1, 2, n, 128) for _ in range(2)]
    sq.sq_cache_read(rows, s.cache, None, cu(np.array([n], np.int32)), *back)
    for i, x in enumerate((K, V)):
        plain.commit(s.codes[i], s.scales[i], s.table, [0], [n], [x[0].cpu().numpy().astype(np.float64).transpose(1, 0, 2)])
        t = np.arange(n)
        at = (s.table[0, t // 32], slice(None), t % 32)
        want = ref.VALUES[s.codes[i][s.table[0, t // 32], :, t % 32]] * s.scales[i][s.table[0, t // 32]][..., None]
        assert np.array_equal(back[i][0].cpu().numpy().transpose(1, 0, 2), want.astype(np.float16)), at
    # a prompt behind it: prefill over K_user and V_user against the tree call over the cache, both on the same values
    T, L = 40, s.L
    q = cu(rng.standard_normal((1, 2, T, 128)).astype(np.float16))
    none = sq.make_shape(1, 2, 1, 1, T, 0, SCALE)
    out, lse = empty(1, 2, T, 128), empty(1, 2, T, dtype=F32)
    sq.sq_tree_attn_q8(none, T, q, *[None] * 7, s.cache, cu(np.array([n], np.int32)), None, None, None, None, out, lse, sq.workspace(none, sq.SQ_CALL_TREE_ATTN_Q8, "cuda:0"))
    pre = sq.make_shape(1, 2, L, s.C, T, n, SCALE)
    Kf = empty(2, L, 128)
    nothing = torch.zeros(1, 2, s.C, 2, dtype=I32, device="cuda"), torch.zeros(1, 2, dtype=I32, device="cuda")
    other, other_lse = empty(1, 2, T, 128), empty(1, 2, T, dtype=F32)
    sq.sq_sparse_attn_prefill_shared(pre, q, Kf, Kf, *nothing, nothing[1], *back, other, other_lse, sq.workspace(pre, sq.SQ_CALL_ATTN_PREFILL_SHARED, "cuda:0"))
    # (both round probabilities to f16, 2^-11 of themselves, and the outputs)
    assert ((out - other).float().abs() <= 2 * 2.0 ** -11 * back[1].abs().max() + 2.0 ** -10 * out.abs()).all() and (lse - other_lse).abs().max() < 1e-4
    # clustered and quantized: 8 bits again, no value further than half a step from what the cache held
    flat = sq.make_shape(1, 2, n, 7, 1, 0, 1.0)
    X, perm, assign = empty(1, 2, n, 128), empty(1, 2, n, dtype=I32), empty(1, 2, n, dtype=I32)
    sizes, offsets = empty(1, 2, 7, dtype=I32), empty(1, 2, 8, dtype=I32)
    sq.sq_kmeans_normalize(flat, back[0], X)
    centers = X[:, :, ::29].contiguous()
    sq.sq_kmeans_step(flat, X, centers, centers, assign, sizes, offsets, perm, sq.workspace(flat, sq.SQ_CALL_KMEANS_STEP, "cuda:0"))
    K8, V8, ks, vs = empty(1, 2, n, 128, dtype=sq.F8), empty(1, 2, n, 128, dtype=sq.F8), empty(1, 2, 4, dtype=F32), empty(1, 2, 4, dtype=F32)
    sq.sq_kv_quantize(flat, *back, perm, K8, V8, ks, vs)
    for x, c, sc in ((back[0], K8, ks), (back[1], V8, vs)):
        got = ref.VALUES[c.view(torch.uint8).cpu().numpy()] * sc.cpu().numpy().repeat(64, 2)[:, :, :n, None]
        was = np.take_along_axis(x.cpu().numpy().astype(np.float64), perm.cpu().numpy()[..., None].astype(int), 2)
        assert (np.abs(got - was) <= np.abs(was) * 2.0 ** -4 + 2.0 ** -10 * sc.cpu().numpy().repeat(64, 2)[:, :, :n, None]).all()
