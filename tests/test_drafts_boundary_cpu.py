"""The calls on drafted tokens refuse bad arguments on the host, before anything is enqueued; the plain implementations that their
GPU tests compare with hold the definitions."""
import ctypes as C

import numpy as np
import pytest

import drafts_reference as plain
from test_q8_boundary_cpu import at, cache, refused, sq  # noqa: F401


def test_prepare_refuses(sq):  # noqa: F811
    INV, UNS = sq.SQ_ERR_INVALID_ARG, sq.SQ_ERR_UNSUPPORTED
    sh = sq.make_shape(3, 1, 1, 1, 40, 0, 1.0)
    args = dict(parents=at(1), n=at(2), first=at(3), mask=at(4), positions=at(5))
    call = lambda shape=sh, **kw: sq.lib().sq_tree_prepare(C.byref(shape), *{**args, **kw}.values(), None)  # noqa: E731
    refused(sq, sq.lib().sq_tree_prepare(None, *args.values(), None), INV, b"shape is NULL")
    refused(sq, call(parents=None), INV, b"parents is NULL")
    refused(sq, call(n=at(2, 4)), INV, b"n_drafts is not 16-byte aligned")
    refused(sq, call(mask=None, positions=None), INV, b"both NULL")
    refused(sq, call(shape=sq.make_shape(3, 1, 1, 1, 1025, 0, 1.0)), UNS, b"at most 1024")
    refused(sq, call(shape=sq.make_shape(0, 1, 1, 1, 40, 0, 1.0)), INV, b"non-positive")
    refused(sq, call(positions=at(1, 464)), INV, b"positions overlaps parents")
    refused(sq, call(mask=at(5, 464)), INV, b"tree_mask overlaps positions")
    refused(sq, call(positions=at(3)), INV, b"positions overlaps first_position")


def test_accept_refuses(sq):  # noqa: F811
    INV, UNS = sq.SQ_ERR_INVALID_ARG, sq.SQ_ERR_UNSUPPORTED
    sh = sq.make_shape(3, 1, 1, 1, 40, 0, 1.0)
    args = dict(parents=at(1), n=at(2), tokens=at(3), target=at(4), seq=at(5), count=at(6), path=at(7), token=at(8), new=at(9))
    call = lambda shape=sh, **kw: sq.lib().sq_tree_accept(C.byref(shape), *{**args, **kw}.values(), None)  # noqa: E731
    for name, said in (("parents", b"parents"), ("tokens", b"tokens"), ("target", b"target"), ("count", b"n_accepted"), ("path", b"path")):
        refused(sq, call(**{name: None}), INV, said + b" is NULL")
    refused(sq, call(seq=None), INV, b"new_len without seq_len")
    refused(sq, call(new=at(5)), INV, b"new_len overlaps seq_len")
    refused(sq, call(path=at(4, 16)), INV, b"path overlaps target")
    refused(sq, call(token=at(6)), INV, b"n_accepted overlaps next_token")
    refused(sq, call(token=at(8, 8)), INV, b"next_token is not 16-byte aligned")
    refused(sq, call(shape=sq.make_shape(3, 1, 1, 1, 2000, 0, 1.0)), UNS, b"at most 1024")


def test_commit_refuses(sq):  # noqa: F811
    INV, UNS = sq.SQ_ERR_INVALID_ARG, sq.SQ_ERR_UNSUPPORTED
    sh = sq.make_shape(3, 2, 1, 1, 5, 0, 1.0)
    args = dict(c=cache(sq), seq=at(1), path=at(2), n=at(3), K=at(4), V=at(5))
    call = lambda shape=sh, **kw: sq.lib().sq_cache_commit(C.byref(shape), *{**args, **kw}.values(), None)  # noqa: E731
    refused(sq, call(c=C.POINTER(sq.SqCache)()), INV, b"cache is NULL")
    refused(sq, call(c=cache(sq, P=24)), INV, b"page_tokens")
    refused(sq, call(c=cache(sq, v_scale=None)), INV, b"v_scale")
    refused(sq, call(seq=None), INV, b"seq_len")
    refused(sq, call(K=None), INV, b"K is NULL")
    refused(sq, call(V=at(5, 8)), INV, b"V is not 16-byte aligned")
    refused(sq, call(path=at(2, 4)), INV, b"path is not 16-byte aligned")
    refused(sq, call(K=at(30, 1024)), INV, b"K8 overlaps K")
    refused(sq, call(seq=at(32, 16)), INV, b"k_scale overlaps seq_len")
    refused(sq, call(c=cache(sq, page_table=at(31))), INV, b"V8 overlaps page_table")
    refused(sq, call(shape=sq.make_shape(1 << 14, 2, 1, 1, 1 << 20, 0, 1.0)), UNS, b"too large")


def test_read_refuses(sq):  # noqa: F811
    INV, UNS = sq.SQ_ERR_INVALID_ARG, sq.SQ_ERR_UNSUPPORTED
    sh = sq.make_shape(3, 2, 1, 1, 1, 50, 1.0)
    args = dict(c=cache(sq), first=at(1), seq=at(2), K=at(3), V=at(4))
    call = lambda shape=sh, **kw: sq.lib().sq_cache_read(C.byref(shape), *{**args, **kw}.values(), None)  # noqa: E731
    refused(sq, call(shape=sq.make_shape(3, 2, 1, 1, 1, 0, 1.0)), INV, b"U = 0")
    refused(sq, call(c=C.POINTER(sq.SqCache)()), INV, b"cache is NULL")
    refused(sq, call(c=cache(sq, max_pages=0)), INV, b"max_pages")
    refused(sq, call(seq=None), INV, b"seq_len")
    refused(sq, call(first=at(1, 2)), INV, b"first is not 16-byte aligned")
    refused(sq, call(K=None), INV, b"K_out is NULL")
    refused(sq, call(V=None), INV, b"V_out is NULL")
    refused(sq, call(V=at(3, 3 * 2 * 50 * 256 - 16)), INV, b"K_out overlaps V_out")
    refused(sq, call(K=at(31, 4096)), INV, b"K_out overlaps V8")
    refused(sq, call(V=at(34)), INV, b"V_out overlaps page_table")
    refused(sq, call(shape=sq.make_shape(1 << 14, 1 << 10, 1, 1, 1, 1 << 12, 1.0)), UNS, b"too large")


def test_attention_refuses(sq):  # noqa: F811
    INV, UNS = sq.SQ_ERR_INVALID_ARG, sq.SQ_ERR_UNSUPPORTED
    sh = sq.make_shape(2, 3, 100, 5, 28, 0, 0.1)
    args = dict(T=7, q=at(1), K8=at(2), V8=at(3), ks=at(4), vs=at(5), ranges=at(6), nr=at(7), nk=at(8), c=cache(sq), seq=at(9), Kd=at(10),
                Vd=at(11), mask=at(12), n=at(13), out=at(14), lse=at(15), ws=at(16), size=1 << 40)
    no_context = dict(K8=None, V8=None, ks=None, vs=None, ranges=None, nr=None, nk=None)
    no_drafts = dict(Kd=None, Vd=None, mask=None)
    call = lambda shape=sh, **kw: sq.lib().sq_tree_attn_q8(C.byref(shape), *{**args, **kw}.values(), None)  # noqa: E731
    for bad in (0, -7, 8, 29):
        refused(sq, call(T=bad), INV, b"times 1 .. 64")
    refused(sq, call(shape=sq.make_shape(2, 3, 100, 5, 130, 0, 0.1), T=2), INV, b"times 1 .. 64")
    refused(sq, call(q=None), INV, b"q is NULL")
    refused(sq, call(out=at(14, 8)), INV, b"out is not 16-byte aligned")
    refused(sq, call(lse=at(15, 4)), INV, b"lse is not 16-byte aligned")
    for name in ("K8", "V8", "ks", "vs", "nr", "nk"):
        refused(sq, call(**{name: None}), INV, b"is NULL")
    refused(sq, call(ranges=None), INV, b"without ranges")
    refused(sq, call(c=None), INV, b"seq_len without a cache")
    refused(sq, call(c=cache(sq, P=20)), INV, b"page_tokens")
    refused(sq, call(seq=None), INV, b"seq_len")
    refused(sq, call(Vd=None), INV, b"go together")
    refused(sq, call(Kd=None, Vd=None), INV, b"tree_mask without")
    refused(sq, call(c=None, seq=None, **no_context, **no_drafts), INV, b"neither")
    refused(sq, call(mask=at(12, 4)), INV, b"tree_mask is not 16-byte aligned")
    refused(sq, call(out=at(1)), INV, b"out overlaps q")
    refused(sq, call(out=at(11, 256)), INV, b"out overlaps V_draft")
    refused(sq, call(lse=at(33)), INV, b"lse overlaps v_scale")
    refused(sq, call(lse=at(14, 2 * 3 * 28 * 256 - 16)), INV, b"out overlaps lse")
    refused(sq, call(shape=sq.make_shape(1, 2048, 1 << 20, 5, 7, 0, 0.1)), UNS, b"too large")
    refused(sq, call(shape=sq.make_shape(1 << 14, 1 << 9, 1 << 18, 5, 7, 0, 0.1)), UNS, b"too large")
    refused(sq, call(ws=None), sq.SQ_ERR_WORKSPACE, b"workspace is NULL")
    refused(sq, call(size=1000), sq.SQ_ERR_WORKSPACE, b"needed")
    refused(sq, call(ws=at(16, 16)), sq.SQ_ERR_WORKSPACE, b"256-byte")
    refused(sq, call(shape=sq.make_shape(2, 3, 100, 5, 28, 0, 0.0)), INV, b"sm_scale")
    refused(sq, call(shape=sq.make_shape(2, 3, 100, 5, 28, 0, 0.1, d=64)), UNS, b"head dim")


def test_grids_of_more_threads_than_32_bits(sq):  # noqa: F811
    """Calls whose tensors would fit the memory, but not one launch: 2^32 threads and more are refused."""
    UNS = sq.SQ_ERR_UNSUPPORTED
    far = lambda i: i + 1 << 44  # noqa: E731
    call = lambda name, shape, *args: getattr(sq.lib(), name)(C.byref(shape), *args, None)  # noqa: E731
    deep = sq.make_shape(1 << 22, 1, 1, 1, 1024, 0, 1.0)
    refused(sq, call("sq_tree_prepare", deep, far(0), None, None, None, far(1)), UNS, b"too large")
    refused(sq, call("sq_tree_accept", sq.make_shape(1 << 26, 1, 1, 1, 2, 0, 1.0), far(0), None, far(1), far(2), None, far(3), far(4), None, None), UNS, b"too large")
    many = cache(sq, n_pages=1)
    refused(sq, call("sq_cache_commit", sq.make_shape(1 << 13, 1 << 9, 1, 1, 16, 0, 1.0), many, far(0), None, None, far(1), far(2)), UNS, b"too large")
    refused(sq, call("sq_cache_read", sq.make_shape(1 << 12, 1 << 6, 1, 1, 1, 1 << 10, 1.0), many, None, far(0), far(1), far(2)), UNS, b"too large")
    one = sq.make_shape(1 << 24, 1, 1, 1, 1, 0, 1.0)
    none = [None] * 7
    refused(sq, call("sq_tree_attn_q8", one, 1, far(0), *none, None, None, far(1), far(2), None, None, far(3), None, far(4), 1 << 50), UNS, b"too large")


def test_the_plain_trees():
    parents = np.array([[-1, 0, 0, 1, 3, 9, 2, 5]])
    bits, positions = plain.prepare(parents, [8], [100])
    assert [np.flatnonzero(r).tolist() for r in bits[0]] == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 3, 4], [5], [0, 2, 6], [5, 7]]
    assert positions[0].tolist() == [100, 101, 101, 102, 103, 100, 102, 101]
    assert plain.words(np.arange(40) % 3 == 0).tolist() == [sum(1 << i for i in range(0, 31, 3)), sum(1 << i - 32 for i in range(33, 40, 3))]
    tokens, target = np.array([[9, 5, 6, 7, 8, 5, 5, 1]]), np.array([[5, 7, 0, 8, 3, 0, 0, 0]])
    assert plain.accept(parents, [8], tokens, target) == [[0, 1, 3, 4]] and plain.accept(parents, [3], tokens, target) == [[0, 1]]
    assert plain.accept(parents, [0], tokens, target) == [[]]


def test_the_plain_attention():
    """Against a softmax over all keys with -inf where a row does not see one."""
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((5, 128)), rng.standard_normal((9, 128)), rng.standard_normal((9, 128))
    seen = rng.random((5, 4)) < 0.5
    seen[2] = False
    parts = [(k[:5], v[:5], None, np.ones(5)), (k[5:], v[5:], seen, np.ones(4))]
    out, lse, off, off_lse = plain.attend(q, parts, 0.1)
    x = np.where(np.concatenate([np.ones((5, 5), bool), seen], 1), q @ k.T * 0.1, -np.inf)
    p = np.exp(x)
    assert np.allclose(out, p / p.sum(1, keepdims=True) @ v) and np.allclose(lse, np.log(p.sum(1)))
    assert 0 < off.min() and off.max() < 3e-3 and off_lse.max() < 1e-4
    out, lse, _, _ = plain.attend(q, parts[1:], 0.1)
    assert (out[2] == 0).all() and lse[2] == -np.inf
