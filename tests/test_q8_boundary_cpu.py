"""The calls on 8-bit keys and values refuse bad arguments on the host, before anything is enqueued; the plain
implementations that their GPU tests compare with hold the definitions."""
import ctypes as C

import numpy as np
import pytest

import q8_reference as ref


@pytest.fixture(scope="module")
def sq():
    import os
    from paper_2411_09688_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build_library()
    binding.lib()
    return binding


def at(i, off=0):
    """A 16-byte aligned address that nothing else here uses (never read: the calls are refused first)."""
    return (1 << 40) + i * (1 << 32) + off


def refused(sq, rc, code, text):
    assert rc == code, (rc, sq.lib().sq_last_error())
    assert text in sq.lib().sq_last_error(), sq.lib().sq_last_error()


def rotary(sq, rot_dim=128, n_positions=10, eps=1e-6, cos_sin=at(20), q_weight=None, k_weight=None):
    return C.byref(sq.SqRotary(rot_dim, 0, n_positions, eps, cos_sin, q_weight, k_weight))


def cache(sq, P=16, n_pages=4, max_pages=2, **kw):
    p = dict(K8=at(30), V8=at(31), k_scale=at(32), v_scale=at(33), page_table=at(34))
    p.update(kw)
    return C.byref(sq.SqCache(P, n_pages, max_pages, p["K8"], p["V8"], p["k_scale"], p["v_scale"], p["page_table"]))


def test_norm_rotate_refuses(sq):
    INV, UNS = sq.SQ_ERR_INVALID_ARG, sq.SQ_ERR_UNSUPPORTED
    sh = sq.make_shape(2, 4, 1, 1, 3, 0, 1.0)

    def call(shape=sh, G=2, rot=None, pos=at(1), q=at(2), qs=1024, k=at(3), ks=512, v=at(4), vs=512, qo=at(5), ko=at(6), vo=at(7)):
        return sq.lib().sq_head_norm_rotate(C.byref(shape), G, rotary(sq) if rot is None else rot, pos, q, qs, k, ks, v, vs, qo, ko, vo, None)

    refused(sq, call(rot=C.POINTER(sq.SqRotary)()), INV, b"rot is NULL")
    for bad in (-8, 4, 136, 12):
        refused(sq, call(rot=rotary(sq, rot_dim=bad)), INV, b"rot_dim")
    refused(sq, call(rot=rotary(sq, eps=-1.0)), INV, b"eps")
    refused(sq, call(rot=rotary(sq, eps=float("nan"))), INV, b"eps")
    refused(sq, call(rot=rotary(sq, eps=float("inf"))), INV, b"eps")
    refused(sq, call(rot=rotary(sq, eps=1e-39)), INV, b"eps")
    refused(sq, call(rot=rotary(sq, n_positions=0)), INV, b"n_positions")
    refused(sq, call(rot=rotary(sq, cos_sin=None)), INV, b"cos_sin")
    refused(sq, call(rot=rotary(sq, q_weight=at(20, 8))), INV, b"weight")
    refused(sq, call(pos=None), INV, b"positions")
    refused(sq, call(G=0), INV, b"G = 0")
    refused(sq, call(G=65), INV, b"G = 65")
    refused(sq, call(q=None), INV, b"q and q_out go together")
    refused(sq, call(ko=None), INV, b"k and k_out go together")
    refused(sq, call(q=None, qo=None, k=None, ko=None, v=None, vo=None), INV, b"all NULL")
    refused(sq, call(qs=1023), INV, b"q's stride")
    refused(sq, call(qs=1016), INV, b"q's stride")
    refused(sq, call(vs=-512), INV, b"v's stride")
    refused(sq, call(k=at(3, 2)), INV, b"k is NULL or not 16-byte aligned")
    refused(sq, call(vo=at(7, 8)), INV, b"v_out is not 16-byte aligned")
    refused(sq, call(qo=at(2)), INV, b"q_out overlaps q")
    refused(sq, call(ko=at(4, 1024)), INV, b"k_out overlaps v")
    refused(sq, call(ko=at(5, 6 * 2048 - 16)), INV, b"q_out overlaps k_out")
    refused(sq, call(shape=sq.make_shape(2, 4, 1, 1, 3, 0, 1.0, d=64)), UNS, b"head dim")
    refused(sq, call(shape=sq.make_shape(1 << 15, 64, 1, 1, 1 << 10, 0, 1.0), qs=8192 * 2, ks=8192, vs=8192), UNS, b"too large")


def test_quantize_refuses(sq):
    INV = sq.SQ_ERR_INVALID_ARG
    sh = sq.make_shape(1, 2, 100, 1, 1, 0, 1.0)
    args = dict(K=at(1), V=at(2), perm=at(3), K8=at(4), V8=at(5), ks=at(6), vs=at(7))
    call = lambda **kw: sq.lib().sq_kv_quantize(C.byref(sh), *{**args, **kw}.values(), None)  # noqa: E731
    refused(sq, call(K=None), INV, b"K is NULL")
    refused(sq, call(K8=at(4, 4)), INV, b"K8 is not 16-byte aligned")
    refused(sq, call(V=None), INV, b"go together")
    refused(sq, call(vs=None), INV, b"go together")
    refused(sq, call(K8=at(1, 25600)), INV, b"K8 overlaps K")
    refused(sq, call(V8=at(4, 12800)), INV, b"K8 overlaps V8")
    refused(sq, call(ks=at(3)), INV, b"k_scale overlaps perm")


def test_append_refuses(sq):
    INV, UNS = sq.SQ_ERR_INVALID_ARG, sq.SQ_ERR_UNSUPPORTED
    sh = sq.make_shape(3, 2, 1, 1, 2, 0, 1.0)

    def call(G=2, rot=None, c=None, n=6, cu=None, seq=at(1), pos=at(2), q=at(3), qs=512, k=at(4), ks=256, v=at(5), vs=256, qo=at(6)):
        return sq.lib().sq_cache_append(C.byref(sh), G, rotary(sq) if rot is None else rot, cache(sq) if c is None else c, n, cu, seq, pos,
                                        q, qs, k, ks, v, vs, qo, None)

    refused(sq, call(c=C.POINTER(sq.SqCache)()), INV, b"cache is NULL")
    for P in (0, 8, 48, 128, -16):
        refused(sq, call(c=cache(sq, P=P)), INV, b"page_tokens")
    refused(sq, call(c=cache(sq, n_pages=0)), INV, b"n_pages")
    refused(sq, call(c=cache(sq, max_pages=-1)), INV, b"max_pages")
    refused(sq, call(c=cache(sq, n_pages=1 << 26)), UNS, b"cache too large")
    refused(sq, call(c=cache(sq, max_pages=1 << 20)), UNS, b"cache too large")
    for name in ("K8", "V8", "k_scale", "v_scale", "page_table"):
        refused(sq, call(c=cache(sq, **{name: None})), INV, name.encode())
    refused(sq, call(seq=None), INV, b"seq_len")
    refused(sq, call(n=-1, cu=at(7)), INV, b"negative")
    refused(sq, call(n=5), INV, b"must be B * Lq = 6")
    refused(sq, call(q=None), INV, b"go together")
    refused(sq, call(k=None), INV, b"k is NULL")
    refused(sq, call(vs=255), INV, b"v's stride")
    refused(sq, call(pos=None), INV, b"positions")
    refused(sq, call(qo=at(3, 1024)), INV, b"q_out overlaps q")
    refused(sq, call(qo=at(5)), INV, b"q_out overlaps v")
    refused(sq, call(c=cache(sq, K8=at(4))), INV, b"K8 overlaps k")
    refused(sq, call(c=cache(sq, V8=at(30, 4096))), INV, b"K8 overlaps V8")
    assert call(n=0, cu=at(7), k=None, v=None, q=None, qo=None) == sq.SQ_OK      # no tokens: nothing to do


def test_decode_refuses(sq):
    INV, UNS = sq.SQ_ERR_INVALID_ARG, sq.SQ_ERR_UNSUPPORTED
    sh = sq.make_shape(2, 3, 100, 5, 4, 0, 0.1)
    args = dict(q=at(1), K8=at(2), V8=at(3), ks=at(4), vs=at(5), ranges=at(6), nr=at(7), nk=at(8), c=cache(sq), seq=at(9), out=at(10),
                lse=at(11), ws=at(12), n=1 << 30)
    none = dict(K8=None, V8=None, ks=None, vs=None, ranges=None, nr=None, nk=None)
    call = lambda shape=sh, **kw: sq.lib().sq_sparse_attn_decode_q8(C.byref(shape), 0, *{**args, **kw}.values(), None)  # noqa: E731
    refused(sq, call(shape=sq.make_shape(2, 3, 100, 5, 17, 0, 0.1)), UNS, b"at most 16")
    refused(sq, call(q=None), INV, b"q is NULL")
    refused(sq, call(out=at(10, 8)), INV, b"out is not 16-byte aligned")
    for name in ("K8", "V8", "ks", "vs", "nr", "nk"):
        refused(sq, call(**{name: None}), INV, b"is NULL")
    refused(sq, call(ranges=None), INV, b"without ranges")
    refused(sq, call(c=None), INV, b"seq_len without a cache")
    refused(sq, call(c=None, seq=None, **none), INV, b"neither")
    refused(sq, call(c=cache(sq, P=20)), INV, b"page_tokens")
    refused(sq, call(seq=None), INV, b"seq_len")
    refused(sq, call(shape=sq.make_shape(1, 2048, 1 << 20, 5, 1, 0, 0.1)), UNS, b"too large")
    refused(sq, call(shape=sq.make_shape(1 << 14, 100, 1 << 17, 5, 4, 0, 0.1)), UNS, b"too large")
    refused(sq, call(ws=None), sq.SQ_ERR_WORKSPACE, b"workspace is NULL")
    refused(sq, call(n=1000), sq.SQ_ERR_WORKSPACE, b"needed")
    refused(sq, call(ws=at(12, 16)), sq.SQ_ERR_WORKSPACE, b"256-byte")
    refused(sq, call(shape=sq.make_shape(2, 3, 100, 5, 4, 0, 0.0)), INV, b"sm_scale")
    a = sq.workspace_bytes(sh, sq.SQ_CALL_ATTN_DECODE_Q8)
    assert a % 256 == 0 and a >= (512 + 6) * 4 * 528 and sq.workspace_bytes(sq.make_shape(2, 3, 1, 1, 4, 0, 1.0), sq.SQ_CALL_ATTN_DECODE_Q8) == a


def test_the_plain_codes():
    """Every code encodes to itself, every border to the even one of its neighbours, what lies between to the nearer."""
    codes = np.arange(256, dtype=np.uint8)
    ok = codes[(codes & 0x7f) != 0x7f]
    assert np.array_equal(ref.encode(ref.VALUES[ok]), ok)
    mid = (ref.GRID[1:] + ref.GRID[:-1]) / 2
    even = np.arange(126) + (np.arange(126) % 2)
    assert np.array_equal(ref.encode(mid), even) and np.array_equal(ref.encode(-mid), even | 0x80)
    assert np.array_equal(ref.encode(np.nextafter(mid, 0)), np.arange(126)) and np.array_equal(ref.encode(np.nextafter(mid, 500)), np.arange(1, 127))
    assert ref.GRID[-1] == 448 and ref.GRID[1] == 2.0 ** -9 and ref.encode(np.inf) == ref.encode(np.nan) == 0x7f
    import torch
    x = torch.from_numpy(np.random.default_rng(0).standard_normal(20000).astype(np.float32) * 30)
    assert np.array_equal(x.to(torch.float8_e4m3fn).view(torch.uint8).numpy(), ref.encode(x.numpy()))
    assert ref.scale_of(np.array([448.0])) == 1 and ref.scale_of(np.array([448.0001])) == 2 and ref.scale_of(np.zeros(3)) == 2.0 ** -64


def test_the_plain_rotation_keeps_lengths_and_depends_on_the_distance_only():
    rng = np.random.default_rng(1)
    a = np.arange(50)[:, None] * 10000.0 ** (-np.arange(0, 96, 2) / 96)
    cs = np.stack([np.cos(a), np.sin(a)], 2)
    x, y = rng.standard_normal((2, 1, 1, 128))
    for adjacent in (False, True):
        turn = lambda v, p: ref.norm_rotate(v, None, 0, cs, np.array([p]), adjacent)  # noqa: E731
        assert np.allclose((turn(x, 30) ** 2).sum(), (x ** 2).sum())
        assert np.allclose((turn(x, 30) * turn(y, 13)).sum(), (turn(x, 37) * turn(y, 20)).sum())
        assert np.array_equal(turn(x, 7)[..., 96:], x[..., 96:])
