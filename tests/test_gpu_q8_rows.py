"""sq_head_norm_rotate and sq_kv_quantize against plain 64-bit implementations."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from paper_2411_09688_amd import binding as sq

pytestmark = pytest.mark.gpu
F16, F32, I32 = torch.float16, torch.float32, torch.int32


def cu(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0", dtype)


def table(n_pos, rot):
    a = np.arange(n_pos)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
    return np.stack([np.cos(a), np.sin(a)], 2).astype(np.float32)


def rows_close(got, want, x, norm):
    """fp32 arithmetic, rounded once to f16: half a step of the value, and of fp32 70 steps (the norm's sum of 128 squares, its
    root and two products) or 3 of what a pair adds up, which is at most twice the row's largest value."""
    got = got.astype(np.float64)
    big = np.abs(want).max(-1, keepdims=True) * 2
    tol = np.abs(want) * 2.0 ** -11 + 2.0 ** -25 + big * (73 if norm else 3) * 2.0 ** -24
    assert (np.abs(got - want) <= tol).all(), np.abs(got - want).max()


ROTATE = [  # B, Lq, H, G, rot, adjacent, norm, fused, n_pos
    (1, 1, 8, 4, 128, False, True, True, 64), (1, 1, 1, 1, 128, True, False, False, 1), (2, 33, 3, 2, 96, False, True, True, 40),
    (3, 17, 2, 5, 64, True, True, False, 100), (1, 300, 1, 64, 8, False, False, True, 300), (2, 5, 2, 1, 8, True, True, True, 3),
    (1, 129, 4, 1, 0, False, True, True, 0), (1, 7, 4, 3, 120, False, False, True, 9), (4, 64, 8, 1, 128, False, False, False, 64),
]


def make_rows(rng, T, H, G, fused):
    Hq = H * G
    if fused:                                                  # one projection, with something between its rows
        x = torch.from_numpy(rng.standard_normal((T, Hq + 2 * H + 1, 128)).astype(np.float16)).cuda()
        return x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:Hq + 2 * H]
    return tuple(cu(rng.standard_normal((T, n, 128)).astype(np.float16)) for n in (Hq, H, H))


def lay(x, B, Lq):
    return x.reshape(B, Lq, x.shape[1], 128).transpose(0, 2, 1, 3)


@pytest.mark.parametrize("B,Lq,H,G,rot,adjacent,norm,fused,n_pos", ROTATE)
def test_norm_rotate(B, Lq, H, G, rot, adjacent, norm, fused, n_pos):
    rng = np.random.default_rng(B * 1000 + Lq + rot)
    T = B * Lq
    q, k, v = make_rows(rng, T, H, G, fused)
    w = [(1 + 0.2 * rng.standard_normal(128)).astype(np.float16) if norm else None for _ in range(2)]
    cs = table(n_pos, rot) if rot else None
    pos = rng.integers(-3, n_pos + 3, T).astype(np.int32)      # some outside the table: the nearest row
    rot_ = sq.make_rotary(None if cs is None else cu(cs), adjacent, *(None if x is None else cu(x) for x in w), eps=2.0 ** -20)
    sh = sq.make_shape(B, H, 1, 1, Lq, 0, 1.0)
    out = [torch.full((B, n, Lq, 128), 7.0, dtype=F16, device="cuda") for n in (H * G, H, H)]
    sq.sq_head_norm_rotate(sh, G, rot_, cu(pos) if rot else None, q, k, v, *out)
    for x, o, weight in ((q, out[0], w[0]), (k, out[1], w[1])):
        want = ref.norm_rotate(x.cpu().numpy(), weight, 2.0 ** -20, cs, pos, adjacent)
        rows_close(o.cpu().numpy(), lay(want, B, Lq), None, norm)
    assert torch.equal(out[2].cpu(), torch.from_numpy(lay(v.cpu().numpy(), B, Lq).copy()))
    # each part alone
    for i, x in enumerate((q, k, v)):
        args, alone = [None] * 3, [None] * 3
        args[i], alone[i] = x, torch.empty_like(out[i])
        sq.sq_head_norm_rotate(sh, G, rot_, cu(pos) if rot else None, *args, *alone)
        assert torch.equal(alone[i], out[i])


def test_norm_rotate_keeps_infinities_and_nan_in_their_rows():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((6, 4, 128)).astype(np.float16)
    x[1, 2, 5], x[3, 0, 100], x[5, 3, 0] = np.inf, np.nan, -np.inf
    x[2, 1] = 0                                                # a row of zeros has a norm of sqrt(eps)
    cs, pos = table(16, 128), np.arange(6, dtype=np.int32)
    w = cu(np.ones(128, np.float16))
    out = torch.empty(1, 4, 6, 128, dtype=F16, device="cuda")
    sq.sq_head_norm_rotate(sq.make_shape(1, 4, 1, 1, 6, 0, 1.0), 1, sq.make_rotary(cu(cs), False, None, w), cu(pos), None, cu(x),
                           None, None, out, None)
    got = out.cpu().numpy()[0].transpose(1, 0, 2)
    want = ref.norm_rotate(x, np.ones(128), 1e-6, cs, pos, False)
    bad = np.zeros((6, 4), bool)
    bad[1, 2] = bad[3, 0] = bad[5, 3] = True
    assert np.isnan(got[3, 0]).all() and np.isnan(got[1, 2]).any() and np.isnan(got[5, 3]).any()
    rows_close(got[~bad], want[~bad], None, True)
    assert (got[2, 1] == 0).all()


QUANTIZE = [(1, 1, 1, False), (1, 2, 63, True), (2, 3, 64, False), (1, 5, 65, True), (3, 1, 200, True), (1, 4, 1000, False)]


@pytest.mark.parametrize("B,H,L,permuted", QUANTIZE)
def test_quantize(B, H, L, permuted):
    rng = np.random.default_rng(L)
    size = 2.0 ** rng.integers(-20, 12, (2, B, H, -(-L // 64)))  # blocks of very different size, down to subnormal f16
    X = [(rng.standard_normal((B, H, L, 128)) * np.repeat(s, 64, 2)[:, :, :L, None]).clip(-65504, 65504).astype(np.float16) for s in size]
    perm = np.stack([rng.permutation(L) for _ in range(B * H)]).reshape(B, H, L).astype(np.int32) if permuted else None
    sh, n = sq.make_shape(B, H, L, 1, 1, 0, 1.0), -(-L // 64)
    for with_v in (True, False):
        K8, V8 = (torch.full((B, H, L, 128), 1.0, device="cuda").to(sq.F8) for _ in range(2))
        ks, vs = (torch.zeros(B, H, n, device="cuda") for _ in range(2))
        extra = (V8, ks, vs) if with_v else (None, ks, None)
        sq.sq_kv_quantize(sh, cu(X[0]), cu(X[1]) if with_v else None, None if perm is None else cu(perm), K8, *extra)
        for x, codes, scale in ((X[0], K8, ks), (X[1], V8, vs))[:1 + with_v]:
            c, s = ref.quantize(x, perm)
            assert np.array_equal(scale.cpu().numpy(), s)
            assert np.array_equal(codes.view(torch.uint8).cpu().numpy(), c)


def test_quantize_borders_infinities_nan_and_bad_indices():
    X = np.zeros((1, 1, 64 * 7, 128), np.float16)
    b = X[0, 0].reshape(7, 64, 128)
    b[0, 3, 5] = 448 * 2.0 ** -3                               # exactly what a scale holds, and one step more
    b[1, 3, 5] = np.nextafter(np.float16(448 * 2.0 ** -3), np.float16(1000))
    b[2, 10, :7] = [np.inf, -np.inf, np.nan, 3.0, -3.0, 2.0 ** -24, 65504]
    b[3] = np.linspace(-448, 448, 64 * 128).reshape(64, 128)   # every border between codes about here
    b[4, 0, 0] = 2.0 ** -24
    b[5, :, 3] = np.nan                                        # no finite value but zeros
    b[6] = (np.arange(64 * 128) % 1024).reshape(64, 128) * 2.0 ** -9 - 1
    perm = np.arange(64 * 7, dtype=np.int32)[None, None].copy()
    perm[0, 0, 0], perm[0, 0, 1], perm[0, 0, 64] = -5, 10 ** 9, 3   # nearest rows; the same row twice
    for p in (None, perm):
        K8, ks = torch.empty(1, 1, 448, 128, dtype=sq.F8, device="cuda"), torch.empty(1, 1, 7, device="cuda")
        sq.sq_kv_quantize(sq.make_shape(1, 1, 448, 1, 1, 0, 1.0), cu(X), None, None if p is None else cu(p), K8, None, ks, None)
        c, s = ref.quantize(X, p)
        assert np.array_equal(ks.cpu().numpy(), s)
        assert ref.same_codes(K8.view(torch.uint8).cpu().numpy(), c).all()


def test_every_finite_half_is_rounded_to_the_nearest_code():
    """All 63488 finite f16 values, 8192 to a block of one exponent range, so that each scale has its values on every border."""
    bits = np.arange(65536, dtype=np.uint16)
    x = bits.view(np.float16)
    x = np.sort(x[np.isfinite(x)].astype(np.float64)).astype(np.float16)
    L = -(-len(x) // 128)
    X = np.zeros(L * 128, np.float16)
    X[:len(x)] = x
    X = X.reshape(1, 1, L, 128)
    K8, ks = torch.empty(1, 1, L, 128, dtype=sq.F8, device="cuda"), torch.empty(1, 1, -(-L // 64), device="cuda")
    sq.sq_kv_quantize(sq.make_shape(1, 1, L, 1, 1, 0, 1.0), cu(X), None, None, K8, None, ks, None)
    c, s = ref.quantize(X, None)
    assert np.array_equal(ks.cpu().numpy(), s) and np.array_equal(K8.view(torch.uint8).cpu().numpy(), c)


def test_calls_on_more_than_the_caches_hold_equal_small_ones():
    """More than 268 MB are read and written past the caches; the parts of such a call, each by itself, are not."""
    g = torch.Generator(device="cuda").manual_seed(5)
    H, L = 11, 32003                                            # 270 MB
    K, V = (torch.randn(1, H, L, 128, generator=g, device="cuda").half() for _ in range(2))
    perm = torch.stack([torch.randperm(L, generator=g, device="cuda") for _ in range(H)])[None].int()
    n = -(-L // 64)
    got = [torch.zeros(1, H, L, 128, dtype=sq.F8, device="cuda") for _ in range(2)] + [torch.zeros(1, H, n, device="cuda") for _ in range(2)]
    sq.sq_kv_quantize(sq.make_shape(1, H, L, 1, 1, 0, 1.0), K, V, perm, *got)
    for h in range(H):
        want = [torch.zeros(1, 1, L, 128, dtype=sq.F8, device="cuda") for _ in range(2)] + [torch.zeros(1, 1, n, device="cuda") for _ in range(2)]
        sq.sq_kv_quantize(sq.make_shape(1, 1, L, 1, 1, 0, 1.0), *(x[:, h:h + 1].clone() for x in (K, V, perm)), *want)
        for a, b in zip(got, want):
            assert torch.equal(a[:, h:h + 1].view(torch.uint8 if a.dtype is sq.F8 else a.dtype), b.view(torch.uint8 if b.dtype is sq.F8 else b.dtype))
    H, T, G = 5, 17001, 5                                       # 304 and 283 MB
    for rot_dim, adjacent in ((128, False), (64, True)):
        w = cu(np.linspace(0.5, 1.5, 128).astype(np.float16))
        rot = sq.make_rotary(cu(table(100, rot_dim)), adjacent, w, w, eps=2.0 ** -20)
        x = torch.randn(T, H * (G + 2), 128, generator=g, device="cuda").half()
        pos = (torch.arange(T, device="cuda") % 100).int()
        parts = (x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:])
        outs = [torch.zeros(1, h, T, 128, dtype=torch.float16, device="cuda") for h in (H * G, H, H)]
        sq.sq_head_norm_rotate(sq.make_shape(1, H, 1, 1, T, 0, 1.0), G, rot, pos, *parts, *outs)
        # ... and of an append, its queries
        table_ = torch.arange(-(-T // 64), device="cuda").int()[None]
        cache = sq.make_cache(*(torch.zeros(len(table_[0]), H, 64, 128, dtype=sq.F8, device="cuda") for _ in range(2)),
                              *(torch.zeros(len(table_[0]), H, device="cuda") for _ in range(2)), table_)
        q_out = torch.zeros(T, H * G, 128, dtype=torch.float16, device="cuda")
        sq.sq_cache_append(sq.make_shape(1, H, 1, 1, T, 0, 1.0), G, rot, cache, torch.zeros(1, dtype=torch.int32, device="cuda"), pos, *parts, q_out)
        for i in range(0, T, 2000):
            m = min(2000, T - i)
            want = [torch.zeros(1, h, m, 128, dtype=torch.float16, device="cuda") for h in (H * G, H, H)]
            sq.sq_head_norm_rotate(sq.make_shape(1, H, 1, 1, m, 0, 1.0), G, rot, pos[i:i + m].clone(), *(p[i:i + m] for p in parts), *want)
            for a, b in zip(outs, want):
                assert torch.equal(a[:, :, i:i + m], b)
        some = torch.arange(0, T, 7)
        want = ref.norm_rotate(parts[0][some.cuda()].cpu().numpy(), np.linspace(0.5, 1.5, 128).astype(np.float16), 2.0 ** -20,
                               table(100, rot_dim), some.numpy() % 100, adjacent)
        rows_close(q_out.cpu().numpy()[some], want, None, True)
