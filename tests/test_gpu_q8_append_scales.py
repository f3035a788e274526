"""Scales of sq_cache_append where they are hard to decide: the codes and scales have to be those of exact arithmetic."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from paper_2411_09688_amd import binding as sq
from test_gpu_q8_cache import EPS, Pool, step
from test_gpu_q8_rows import cu, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P,old,new", [(16, 0, 1), (16, 3, 5), (32, 0, 32), (64, 0, 64), (64, 17, 60)])
@pytest.mark.parametrize("what", [np.inf, -np.inf, np.nan, None])
@pytest.mark.parametrize("adjacent", [False, True])
def test_a_page_with_an_infinity_whose_finite_maximum_is_next_to_a_scales_limit(P, old, new, what, adjacent):
    """A pair (1, -2^-10) turned by (1.75, 2^-30): 1.75 + 2^-40, just more than 448 * 2^-8 holds, which 24 bits do not tell from 1.75."""
    rng = np.random.default_rng(P + new)
    rot = 128 if adjacent else 64                               # (so that some lanes do not rotate)
    cs = np.zeros((2, rot // 2, 2), np.float32)
    cs[:, :, 0] = 1.0
    cs[1, 0] = 1.75, 2.0 ** -30
    pool = Pool(rng, 1, 2, P, -(-(old + new) // P))
    for c, s in zip(pool.codes, pool.scales):
        c[:] = ref.encode((rng.standard_normal(c.shape) * 100).clip(-448, 448))
        s[:] = 2.0 ** -12
    pool.upload()
    x = (rng.random((2, new, 2, 128)) - 0.5).astype(np.float16)
    pos = np.zeros(new, np.int32)
    pos[new // 2] = 1
    x[0, new // 2, :, [0, 1 if adjacent else rot // 2]] = np.array([[1.0], [-2.0 ** -10]], np.float16)
    if what is not None:                                        # in another pair, of another token where there is one
        x[0, -1, 0, 40] = x[0, 0, 1, 127] = x[1, -1, 0, 3] = what
    assert ref.norm_rotate(x[0], None, EPS, cs, pos, adjacent)[new // 2, 0, 0] == 1.75 + 2.0 ** -40
    lay = ([None, None], cs, adjacent, sq.make_rotary(cu(cs), adjacent, eps=EPS))
    step(pool, lay, None, cu(x[0]), cu(x[1]), pos, [old], [new], 1, True, repeat=2)
    pool.check()


@pytest.mark.parametrize("P,old,new", [(16, 3, 1), (32, 31, 40), (64, 17, 60)])
@pytest.mark.parametrize("level", [2.0 ** -14, 1.0])
def test_a_page_whose_scale_is_no_power_of_two_keeps_its_values(P, old, new, level):
    """Pages filled elsewhere: a scale goes to the next power of two, and the codes with it."""
    rng = np.random.default_rng(P + new)
    H = 12
    pool = Pool(rng, 1, H, P, -(-(old + new) // P))
    for c, s in zip(pool.codes, pool.scales):
        c[:] = ref.encode((rng.standard_normal(c.shape) * 100).clip(-448, 448))
        c[:, :, 1] = np.arange(128) | 0x80                      # every code
        c[:, :, 2] = np.arange(128)
        s[:] = np.array([1.1 * 2.0 ** -7, 0.0, 3e-9, -1.5 * 2.0 ** -7, 2.0 ** -70, 1.3 * 2.0 ** -70, 2.0 ** 64, 1.9 * 2.0 ** 63, 1e-39,
                         2.0 ** -7, 1 + 2.0 ** -23, 2 - 2.0 ** -23]).astype(np.float32)
    pool.upload()
    x = (rng.standard_normal((2, new, H, 128)) * level).astype(np.float16)
    page = pool.table[0, 0]
    for c, s, rows in zip(pool.codes, pool.scales, x.astype(np.float64)):   # the old codes at the page's new scale, rounded once
        for h in range(H):
            top = max(ref.scale_of(rows[:P - old, h]), 2.0 ** np.ceil(np.log2(max(abs(s[page, h]), 2.0 ** -64))))
            v = ref.VALUES[c[page, h, :old]].astype(np.float32) * np.float32(s[page, h] / top)
            c[page, h, :old] = np.where(np.isnan(v), c[page, h, :old], ref.encode(v))
            s[page, h] = top
    lay = ([None, None], None, False, sq.make_rotary(None))
    step(pool, lay, None, cu(x[0]), cu(x[1]), np.zeros(new, np.int32), [old], [new], 1, True, repeat=2)
    pool.check()


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("power", [-100, -60, 60, 72, 76, 100])
def test_keys_that_a_scaled_table_takes_out_of_the_scales_range(norm, power):
    rng = np.random.default_rng(power + 200)
    T, H, P = 70, 2, 32
    pool = Pool(rng, 1, H, P, 3)
    cs = (table(16, 128) * 2.0 ** power).astype(np.float32)
    w = (1 + 0.2 * rng.standard_normal(128)).astype(np.float16) if norm else None
    rot = sq.make_rotary(cu(cs), False, None, None if w is None else cu(w), eps=EPS)
    k, v = (rng.standard_normal((T, H, 128)).astype(np.float16) for _ in range(2))
    pos = (np.arange(T) % 16).astype(np.int32)
    sq.sq_cache_append(sq.make_shape(1, H, 1, 1, T, 0, 1.0), 1, rot, pool.cache, cu(np.zeros(1, np.int32)), cu(pos), None, cu(k), cu(v), None)
    turned = ref.norm_rotate(k, w, EPS, cs, pos, False)
    got, scales = pool.d[0].view(torch.uint8).cpu().numpy(), pool.d[2].cpu().numpy()
    for i in range(3):
        for h in range(H):
            x = turned[i * P:(i + 1) * P, h]
            s = ref.scale_of(x)
            y = x / s
            assert scales[pool.table[0, i], h] == s
            want = ref.encode(np.where(np.abs(y) > 464, np.nan, y.clip(-448, 448)))   # (464: between the last code and what would be the next)
            assert ref.same_codes(got[pool.table[0, i], h, :len(x)], want).all()
