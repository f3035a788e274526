"""sq_tree_attn_q8 where its arithmetic and its division have least room: scales of values at both ends of what they may be, drafts that are not finite in
blocks of every size, as many blocks as workgroups share, the widest tables."""
import numpy as np
import pytest
import torch

import drafts_reference as plain
import q8_reference as ref
from paper_2411_09688_amd import binding as sq
from test_gpu_q8_rows import cu
from test_gpu_tree_attn import SCALE, Problem

pytestmark = pytest.mark.gpu

# Scales of values below 2^-40 count as 2^-40: a value, at most 448 times its scale, is then off by less than 448 * 2^-40 < 2^-31, and so is an
# output, a mean of values.
LEAST, OFF = 2.0 ** -40, 2.0 ** -31


def check(p):
    """Outputs where the oracle's are within f16's range, and all log-sum-exps."""
    out, lse = p.out.cpu().numpy().astype(np.float64), p.lse.cpu().numpy().astype(np.float64)
    for b in range(p.B):
        for h in range(p.H):
            keys, n = p.keys(b, h)
            keys = [(k, v, seen, np.maximum(s, LEAST)) for k, v, seen, s in keys]
            rows = p.q[b, h * p.G:h * p.G + p.G, :n].transpose(1, 0, 2).reshape(n * p.G, 128).astype(np.float64)
            o, z, off, off_z = plain.attend(rows, keys, SCALE)
            got = out[b, h * p.G:h * p.G + p.G, :n].transpose(1, 0, 2).reshape(n * p.G, 128)
            got_z = lse[b, h * p.G:h * p.G + p.G, :n].T.reshape(n * p.G)
            assert np.array_equal(np.isneginf(z), np.isneginf(got_z)), (b, h)
            ok = np.isfinite(z)
            assert np.all(np.abs(got_z[ok] - z[ok]) <= off_z[ok]), (b, h, got_z[:4], z[:4])
            near = np.abs(o) + off < 65504
            assert np.all(np.abs(got - o)[near] <= off[near] + OFF), (b, h)


@pytest.mark.parametrize("least", [0.0, 2.0 ** -126, 2.0 ** -120, 2.0 ** -113, 2.0 ** -41])
@pytest.mark.parametrize("share", [1.0, 0.5])
@pytest.mark.parametrize("G,T", [(2, 9), (4, 40), (8, 90)])
def test_small_scales_of_values(least, share, G, T):
    """Pages and blocks that hold next to nothing, beside ordinary ones or alone; keys' scales of zero among them."""
    p = Problem(T, 2, 2, G, T, L=900, C=25, keep=0.5, user=130, page=32)
    for a in (p.vs, p.cvs):
        a[p.rng.random(a.shape) < share] = least
    p.ks[:, ::5] = 0
    p.upload().call()
    check(p)


def test_a_wave_of_small_scales_beside_waves_of_ordinary_ones():
    """Of 512 kept keys the first quarter, one wave's, stands in blocks of a scale of 2^-120."""
    p = Problem(31, 1, 2, 4, 12, L=512, C=4, user=0, drafts=False)
    p.ranges[:] = [[[[0, 128], [128, 128], [256, 128], [384, 128]]] * 2]
    p.nr[:], p.nk[:] = 4, 512
    p.vs[:, :2] = 2.0 ** -120
    p.upload().call()
    check(p)


@pytest.mark.parametrize("least", [0.0, 2.0 ** -126, 2.0 ** -64])
def test_the_sum_keeps_keys_of_small_scales_beside_one_of_the_largest(least):
    """4096 keys, each with 2^-7 of the probability of a key whose scale is 2^40 and whose codes are zeros: 32 times its weight in all."""
    p = Problem(32, 1, 1, 1, 5, L=4096 + 64, C=2, user=0, drafts=False)
    p.ranges[:] = [[[[0, 1], [64, 4096]]]]
    p.nr[:], p.nk[:] = 2, 4097
    p.q[:] = 1
    p.K8[:] = 0
    p.K8[0, 0] = ref.encode(np.full(128, 1.0))
    p.ks[:] = 7 * np.log(2) / (128 * SCALE)                     # (the first key's score is 7 ln 2, the others' 0)
    p.ks = p.ks.astype(np.float32).astype(np.float64)
    p.V8[0, 0] = 0
    p.vs[:] = least
    p.vs[0, 0] = 2.0 ** 40
    p.upload().call()
    check(p)
    assert np.abs(p.lse.cpu().numpy() - np.log(128 + 4096)).max() < 1e-3 and (p.out == 0).all()


def test_a_batch_of_chains_behind_the_widest_tables():
    """8 prompts of 2048 tokens, 128 heads, and room for 2M tokens each: more tiles that there could be than 31 bits count, in 32768 blocks of their own."""
    B, H, G, T, P = 8, 8, 16, 2048, 16
    small = Problem(40, B, H, 1, 1, user=50, page=P, drafts=False)
    table = np.full((B, (1 << 21) // P), -1, np.int32)
    table[:, :small.table.shape[1]] = small.table
    g = torch.Generator(device="cuda").manual_seed(40)
    q = torch.randn(B, H * G, T, 128, generator=g, device="cuda", dtype=torch.float16)
    K, V = (torch.randn(B, H, T, 128, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))
    n = np.array([T, 1900, 64, 1, 0, T, T - 1, 777], np.int32)
    sh = sq.make_shape(B, H, 1, 1, G * T, 0, SCALE)
    blocks = B * H * (G * T // 64)
    assert blocks * (((1 << 21) + T) // 32) > 0x7fffffff and sq.workspace_bytes(sh, sq.SQ_CALL_TREE_ATTN_Q8) == 0
    cache = sq.make_cache(cu(small.cK).view(sq.F8), cu(small.cV).view(sq.F8), cu(small.cks.astype(np.float32)), cu(small.cvs.astype(np.float32)), cu(table))
    out, lse = torch.full_like(q, 9), torch.full((B, H * G, T), 9.0, device="cuda")
    sq.sq_tree_attn_q8(sh, T, q, *[None] * 7, cache, cu(small.held), K, V, None, cu(n), out, lse, None)
    for b, h, t in ((0, 0, 0), (0, 7, 2047), (1, 3, 1899), (2, 5, 63), (3, 1, 0), (5, 2, 1024), (6, 6, 2046), (7, 7, 776)):
        held = np.arange(small.held[b])
        at = (small.table[b, held // P], h, held % P)
        keys = [(ref.VALUES[small.cK[at]] * small.cks[at[:2]][:, None], ref.VALUES[small.cV[at]] * small.cvs[at[:2]][:, None], None, small.cvs[at[:2]]),
                (K[b, h, :t + 1].cpu().numpy().astype(np.float64), V[b, h, :t + 1].cpu().numpy().astype(np.float64), None, np.ones(t + 1))]
        rows = q[b, h * G:h * G + G, t].cpu().numpy().astype(np.float64)
        o, z, off, off_z = plain.attend(rows, keys, SCALE)
        got, got_z = (x[b, h * G:h * G + G, t].cpu().numpy().astype(np.float64) for x in (out, lse))
        assert np.all(np.abs(got - o) <= off) and np.all(np.abs(got_z - z) <= off_z), (b, h, t)
    for b in range(B):
        assert (out[b, :, int(n[b]):] == 9).all() and (lse[b, :, int(n[b]):] == 9).all()


# For each size of a block of rows: heads a K/V head, drafts, room of the table (the most keys that there could be choose 48 and 64 rows).
SIZES = {16: (2, 8, 0), 32: (2, 16, 0), 48: (4, 12, 1 << 21), 64: (3, 20, 1 << 21), "64, three of them": (4, 40, 1 << 21), "64, by their number": (8, 90, 0)}


def of_size(size, seed, **kw):
    G, T, room = SIZES[size]
    p = Problem(seed, 3 if size == "64, by their number" else 2, 2, G, T, **{**dict(L=300, C=10, user=50, mask="any"), **kw})
    if room and p.held is not None:
        p.table = np.concatenate([p.table, np.full((p.B, room // p.page - p.table.shape[1]), -1, np.int32)], 1)
    return p


def rows_of(p, x, b, h):
    """[B, H*G, T, ..] -> [(t, g), ..] of a K/V head."""
    x = x.cpu().numpy().astype(np.float64)[b, h * p.G:h * p.G + p.G]
    return np.swapaxes(x, 0, 1).reshape(p.T * p.G, *x.shape[2:])


@pytest.mark.parametrize("alone", [False, True])
@pytest.mark.parametrize("what", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("size", SIZES)
def test_drafts_keys_that_are_not_finite(size, what, alone):
    """A score of +inf or NaN makes the rows that see it not finite; one of -inf has no weight, and a row of nothing else counts as one without keys."""
    p = of_size(size, 50, **(dict(L=0, C=0, user=16) if alone else {}))
    if alone:
        p.held[:] = 0
    nothing = 0
    odd = [0, 3, p.T - 1]
    p.bits[:, 2] = False
    p.bits[:, 2, odd[1]] = True                                 # (a row that sees one such key alone)
    p.mask = plain.words(p.bits)
    for j in odd:
        p.Kd[:, :, j, 7 + j % 3] = what
    assert (p.q != 0).all()
    p.upload().call()
    p.Kd = np.where(np.isfinite(p.Kd), p.Kd, 0)                 # (for the oracle: such keys are not seen, or the row is not looked at)
    for b in range(p.B):
        for h in range(p.H):
            q, out, lse = p.q[b, h * p.G:h * p.G + p.G].transpose(1, 0, 2).reshape(p.T * p.G, 128).astype(np.float64), rows_of(p, p.out, b, h), rows_of(p, p.lse, b, h)
            seen = np.repeat(p.bits[b], p.G, 0)
            up = np.zeros_like(seen[:, 0])
            for j in odd:
                up |= seen[:, j] & (np.isnan(what) | (q[:, 7 + j % 3] * np.sign(what) > 0))
                seen[:, j] = False
            assert up.any() and not up.all()
            assert not np.isfinite(out[up]).any() and not np.isfinite(lse[up]).any()
            keys = [(k, v, seen if s is not None else None, sv) for k, v, s, sv in p.keys(b, h)[0]]
            o, z, off, off_z = plain.attend(q, keys, SCALE)
            fine, some = ~up, ~up & np.isfinite(z)
            assert np.all(np.abs(out - o)[fine] <= off[fine]) and np.array_equal(np.isneginf(lse[fine]), np.isneginf(z[fine]))
            assert np.all(np.abs(lse[some] - z[some]) <= off_z[some])
            assert (out[np.isneginf(z) & fine] == 0).all()
            nothing += (np.isneginf(z) & fine)[2 * p.G:3 * p.G].sum()
    assert (nothing > 0) == (alone and not np.isnan(what))


@pytest.mark.parametrize("what", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("size", SIZES)
def test_drafts_values_that_are_not_finite(size, what):
    """They reach the rows that see them, in their dimension, and nothing else."""
    p = of_size(size, 51)
    odd = [0, 5, p.T - 1]
    for j in odd:
        p.Vd[:, :, j, 7 + j % 3] = what
    p.upload().call()
    p.Vd = np.where(np.isfinite(p.Vd), p.Vd, 0)
    for b in range(p.B):
        for h in range(p.H):
            q, out, lse = p.q[b, h * p.G:h * p.G + p.G].transpose(1, 0, 2).reshape(p.T * p.G, 128).astype(np.float64), rows_of(p, p.out, b, h), rows_of(p, p.lse, b, h)
            hit = np.zeros(out.shape, bool)
            for j in odd:
                hit[:, 7 + j % 3] |= np.repeat(p.bits[b][:, j], p.G)
            assert hit.any() and not np.isfinite(out[hit]).any()
            o, z, off, off_z = plain.attend(q, p.keys(b, h)[0], SCALE)
            some = np.isfinite(z)
            assert np.all(np.abs(out - o)[~hit] <= off[~hit]) and np.all(np.abs(lse[some] - z[some]) <= off_z[some]) and np.array_equal(np.isneginf(lse), ~some)


@pytest.mark.parametrize("B,H,G,T", [(24, 32, 2, 5), (33, 31, 2, 5), (32, 32, 2, 5), (25, 41, 2, 5), (16, 16, 10, 25), (5, 41, 10, 25)])
def test_as_many_blocks_as_are_shared(B, H, G, T):
    """768, 1023 and 1024 blocks are shared among 512 workgroups, four a thread where they are counted; 1025 and more have one each and need no workspace."""
    p = Problem(B + T, B, H, G, T, L=100, C=5, user=20, ragged=True)
    p.n[1] = 0
    blocks = B * H * -(-G * T // 64)
    p.upload()
    assert (sq.workspace_bytes(p.shape, sq.SQ_CALL_TREE_ATTN_Q8) > 0) == (blocks <= 1024)
    p.call()
    p.check()


@pytest.mark.parametrize("size", SIZES)
def test_numbers_below_the_normal_ones_of_f16(size):
    """Queries, drafts' keys and drafts' values of 2^-15 and less, with scales and sources that make them count."""
    p = of_size(size, 52, L=0, C=0, mask=None, drafts=False)
    p.q = (p.q * np.float16(2.0 ** -17)).astype(np.float16)
    p.cks[:] = 2.0 ** 8                                         # (scores of some hundredths)
    p.upload().call()
    check(p)
    assert np.ptp(p.lse.cpu().numpy()[0]) > 0.01                # (ln 50 for all rows, were they zeros)
    p = of_size(size, 53, L=0, C=0, user=16)
    p.held[:] = 0
    p.bits[:] = np.tril(np.ones(p.bits.shape[1:], bool))
    p.mask = plain.words(p.bits)
    p.q = (p.q * np.float16(2.0 ** 9)).astype(np.float16)
    p.Kd, p.Vd = ((x * np.float16(2.0 ** -s)).astype(np.float16) for x, s in ((p.Kd, 17), (p.Vd, 18)))
    p.upload().call()
    check(p)
    out = np.abs(p.out.cpu().numpy().astype(np.float64))
    assert 0 < out.max() < 2.0 ** -15
