"""sq_cache_append against a plain 64-bit implementation: codes and scales have to be equal."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from paper_2411_09688_amd import binding as sq
from test_gpu_q8_rows import cu, make_rows, rows_close, table

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -20


class Pool:
    """A cache on the device and the same on the host; codes random (whatever a reused page holds, NaN among it)."""

    def __init__(self, rng, B, H, P, width, spare=2):
        n = B * width + spare
        self.table = rng.permutation(n)[:B * width].reshape(B, width).astype(np.int32)
        self.codes = [rng.integers(0, 256, (n, H, P, 128)).astype(np.uint8) for _ in range(2)]
        self.scales = [2.0 ** rng.integers(-9, -4, (n, H)).astype(np.float64) for _ in range(2)]
        self.upload()

    def upload(self):
        self.d = [cu(c).view(sq.F8) for c in self.codes] + [cu(s.astype(np.float32)) for s in self.scales] + [cu(self.table)]
        self.cache = sq.make_cache(*self.d)

    def check(self):
        for i in range(2):
            assert np.array_equal(self.d[2 + i].cpu().numpy(), self.scales[i].astype(np.float32)), "scales"
            got = self.d[i].view(torch.uint8).cpu().numpy()
            same = ref.same_codes(got, self.codes[i])
            assert same.all(), (np.argwhere(~same)[:5], int((~same).sum()))


def layer(rng, norm, rot, adjacent, n_pos):
    w = [(1 + 0.2 * rng.standard_normal(128)).astype(np.float16) if norm else None for _ in range(2)]
    cs = table(n_pos, rot) if rot else None
    return w, cs, adjacent, sq.make_rotary(None if cs is None else cu(cs), adjacent, *(None if x is None else cu(x) for x in w), eps=EPS)


def step(pool, lay, q, k, v, pos, old, new, G, cu_tokens, Lq=1, repeat=1, stream=None):
    """One append on both sides; returns (q_out, what it has to be)."""
    w, cs, adjacent, rot = lay
    B, H = len(old), k.shape[1]
    n = k.shape[0]
    first = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q_out = torch.full((n, H * G, 128), 3.0, dtype=torch.float16, device="cuda") if q is not None else None
    for _ in range(repeat):
        sq.sq_cache_append(sq.make_shape(B, H, 1, 1, Lq, 0, 1.0), G, rot, pool.cache, cu(np.asarray(old, np.int32)), cu(pos), q, k, v,
                           q_out, cu(first) if cu_tokens else None, stream=stream)
    kr = ref.norm_rotate(k.cpu().numpy(), w[1], EPS, cs, pos, adjacent)
    for i, x in ((0, kr), (1, v.cpu().numpy().astype(np.float64))):
        ref.append(pool.codes[i], pool.scales[i], pool.table, old, new, first, x)
    if q is None:
        return
    want = np.full((n, H * G, 128), 3.0)
    used = int(first[-1])
    want[:used] = ref.norm_rotate(q.cpu().numpy(), w[0], EPS, cs, pos, adjacent)[:used]
    got = q_out.cpu().numpy()
    rows_close(got[:used], want[:used], None, w[0] is not None)
    assert (got[used:] == 3.0).all()


APPEND = [  # H, G, page, old, new, norm, rot, adjacent, ragged, pad
    (1, 1, 16, [0], [1], False, 128, False, False, 0),
    (2, 4, 64, [5, 63, 64, 0, 130], [1] * 5, True, 128, False, False, 0),
    (3, 1, 16, [15, 16, 17], [1] * 3, True, 96, True, False, 0),
    (2, 2, 32, [31, 7], [33, 33], True, 64, False, False, 0),             # Lq = 33: two or three pages each
    (1, 8, 64, [10, 0, 64, 200, 63], [0, 130, 1, 0, 64], True, 128, True, True, 3),
    (4, 1, 16, [3, 3, 3, 3], [0, 0, 0, 0], False, 128, False, True, 2),    # nothing to append
    (2, 3, 32, [0] * 300, [i % 3 for i in range(300)], False, 32, False, True, 0),   # more sequences than one round of the scan
    (5, 1, 64, [40], [1000], True, 0, False, True, 0),
    (2, 1, 16, [0, 9], [16, 7], False, 8, True, True, 1),                  # pages that end exactly
]


@pytest.mark.parametrize("H,G,P,old,new,norm,rot,adjacent,ragged,pad", APPEND)
def test_append(H, G, P, old, new, norm, rot, adjacent, ragged, pad):
    rng = np.random.default_rng(len(old) * 100 + P + rot)
    B, T = len(old), sum(new) + pad
    pool = Pool(rng, B, H, P, max(1, max(-(-(a + b) // P) for a, b in zip(old, new))))
    for c in pool.codes:                                        # what is held so far is no NaN, but for some
        c[(c & 0x7f) == 0x7f] = np.where(rng.random(int(((c & 0x7f) == 0x7f).sum())) < 0.9, 0x31, 0xff)
    pool.upload()
    lay = layer(rng, norm, rot, adjacent, 500)
    q, k, v = make_rows(rng, T, H, G, True)
    v *= 2.0 ** rng.integers(-3, 4, (T, 1, 1))[0].item()
    pos = rng.integers(0, 500, T).astype(np.int32)
    step(pool, lay, q if G > 1 else None, k, v, pos, old, new, G, ragged, Lq=new[0] if not ragged else 1)
    pool.check()


def test_a_sequence_grown_token_by_token_and_repeated_steps():
    """Values of growing size, so that the scales of a page are raised again and again, each step made twice."""
    rng = np.random.default_rng(1)
    B, H, P = 2, 2, 16
    pool = Pool(rng, B, H, P, 3)
    lay = layer(rng, False, 128, False, 64)
    old = [0, 3]
    for c in pool.codes:
        c[:] = ref.encode((rng.standard_normal(c.shape) * 100).clip(-448, 448))
    pool.upload()
    for t in range(40):
        k, v = (cu((rng.standard_normal((B, H, 128)) * 1.2 ** t * f).astype(np.float16)) for f in (1.0, 0.01))
        step(pool, lay, None, k, v, np.full(B, t, np.int32), old, [1] * B, 1, False, repeat=2)
        old = [n + 1 for n in old]
        pool.check()


def test_a_prompt_at_once_is_the_same_as_in_parts_where_the_scale_stays():
    rng = np.random.default_rng(2)
    H, P, T = 2, 64, 150
    a, b = Pool(rng, 1, H, P, 3), Pool(rng, 1, H, P, 3)
    b.codes, b.scales, b.table = [c.copy() for c in a.codes], [s.copy() for s in a.scales], a.table
    b.upload()
    lay = layer(rng, True, 128, False, 256)
    x = rng.standard_normal((2, T, H, 128)).astype(np.float16)
    x[:, ::16, :, 0] = 4.0                                     # the largest of every 16 tokens comes first (values; keys are normed)
    k, v = cu(x[0]), cu(x[1].clip(-4, 4))
    pos = np.arange(T, dtype=np.int32)
    step(a, lay, None, k, v, pos, [0], [T], 1, True)
    for lo, hi in ((0, 16), (16, 17), (17, 100), (100, 150)):
        step(b, lay, None, k[lo:hi], v[lo:hi], pos[lo:hi], [lo], [hi - lo], 1, True)
    a.check()
    b.check()
    assert np.array_equal(a.d[1].view(torch.uint8).cpu().numpy(), b.d[1].view(torch.uint8).cpu().numpy())


@pytest.mark.parametrize("m", [64.0, 1.375, 2.0 ** -6])
def test_cosines_and_sines_of_any_size(m):
    """A table may be scaled (a softmax temperature put into it): the codes are those of exact arithmetic all the same."""
    rng = np.random.default_rng(7)
    H, T = 4, 4096
    pool = Pool(rng, 1, H, 64, T // 64)
    lay = layer(rng, True, 128, False, 16)
    scaled = (lay[1] * np.float32(m)).astype(np.float32)
    lay = (lay[0], scaled, False, sq.make_rotary(cu(scaled), False, *(cu(x) for x in lay[0]), eps=EPS))
    k, v = (cu(rng.standard_normal((T, H, 128)).astype(np.float16)) for _ in range(2))
    step(pool, lay, None, k, v, (np.arange(T) % 16).astype(np.int32), [0], [T], 1, True)
    pool.check()


def test_bad_pages_and_full_sequences_drop_tokens():
    rng = np.random.default_rng(3)
    H, P = 2, 16
    pool = Pool(rng, 4, H, P, 3)
    pool.table[0, 1], pool.table[1, 0], pool.table[2, 2] = -1, 10 ** 6, -2 ** 31
    for c in pool.codes:
        c[:] = ref.encode((rng.standard_normal(c.shape) * 100).clip(-448, 448))
    pool.upload()
    lay = layer(rng, True, 128, False, 64)
    old, new = [10, 0, 30, 45], [20, 20, 10, 9]                 # the last three: past the pages there are
    k, v = (cu(rng.standard_normal((sum(new), H, 128)).astype(np.float16)) for _ in range(2))
    step(pool, lay, None, k, v, np.zeros(sum(new), np.int32), old, new, 1, True)
    pool.check()
    for held in ([-7, 48, 1000, 2 ** 31 - 1],):                # lengths outside the pages
        step(pool, lay, None, k[:4], v[:4], np.zeros(4, np.int32), held, [1] * 4, 1, False)
        pool.check()


def test_infinities_and_nan_become_nan_codes_and_set_no_scale():
    rng = np.random.default_rng(4)
    pool = Pool(rng, 1, 1, 16, 2)
    x = rng.standard_normal((2, 20, 1, 128)).astype(np.float16)
    x[1, 2, 0, 3], x[1, 3, 0, 4], x[1, 19, 0] = np.inf, np.nan, -np.inf
    x[0, 7, 0, 1] = np.nan                                     # of a key: the norm spreads it over its row
    lay = layer(rng, True, 128, False, 64)
    step(pool, lay, None, cu(x[0]), cu(x[1]), np.arange(20, dtype=np.int32), [0], [20], 1, True)
    pool.check()


@pytest.mark.parametrize("norm,rot,adjacent", [(True, 0, False), (False, 64, False), (True, 64, True), (True, 96, False), (False, 128, True)])
def test_infinities_and_nan_of_keys_stay_with_what_is_computed_from_them(norm, rot, adjacent):
    rng = np.random.default_rng(8)
    pool = Pool(rng, 1, 2, 16, 2)
    x = rng.standard_normal((2, 30, 2, 128)).astype(np.float16)
    x[0, 1, 0, 3], x[0, 2, 0, 127], x[0, 9, 1, 100], x[0, 20, 0, 70], x[0, 29, 1, 0] = np.inf, np.nan, -np.inf, np.inf, np.nan
    lay = layer(rng, norm, rot, adjacent, 64)
    step(pool, lay, None, cu(x[0]), cu(x[1]), np.arange(30, dtype=np.int32), [0], [30], 1, True)
    pool.check()


def test_on_another_stream_and_captured():
    rng = np.random.default_rng(6)
    B, H, P = 3, 2, 16
    pool = Pool(rng, B, H, P, 4)
    for c in pool.codes:
        c[:] = ref.encode((rng.standard_normal(c.shape) * 100).clip(-448, 448))
    pool.upload()
    lay = layer(rng, True, 128, False, 64)
    side = torch.cuda.Stream()
    k, v = (cu(rng.standard_normal((B, H, 128)).astype(np.float16)) for _ in range(2))
    torch.cuda.synchronize()
    old = [3, 15, 16]
    step(pool, lay, None, k, v, np.zeros(B, np.int32), old, [1] * B, 1, False, stream=side)
    torch.cuda.synchronize()
    pool.check()
    # one captured step, replayed on new rows and lengths
    seq, pos = cu(np.zeros(B, np.int32)), cu(np.zeros(B, np.int32))
    sh = sq.make_shape(B, H, 1, 1, 1, 0, 1.0)
    graph = torch.cuda.CUDAGraph()
    kb, vb = torch.zeros_like(k), torch.zeros_like(v)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sq.sq_cache_append(sh, 1, lay[3], pool.cache, seq, pos, None, kb, vb, None)
    for t in range(4):
        k, v = (rng.standard_normal((B, H, 128)).astype(np.float16) for _ in range(2))
        old = [4 + t, 16 + t, 17 + t]
        kb.copy_(cu(k)); vb.copy_(cu(v)); seq.copy_(cu(np.asarray(old, np.int32))); pos.fill_(t)
        graph.replay()
        torch.cuda.synchronize()
        kr = ref.norm_rotate(k, lay[0][1], EPS, lay[1], np.full(B, t), False)
        for i, x in ((0, kr), (1, v.astype(np.float64))):
            ref.append(pool.codes[i], pool.scales[i], pool.table, old, [1] * B, list(range(B)), x)
        pool.check()
