"""Scales of sq_cache_append where they are hard to decide: the codes and scales have to be those of exact arithmetic."""
import numpy as np
import pytest

import q8_reference as ref
from paper_2411_09688_amd import binding as sq
from test_gpu_q8_cache import EPS, Pool, step
from test_gpu_q8_rows import cu

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
