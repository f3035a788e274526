"""The calls around drafted tokens and the paged cache at their edges."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from paper_2411_09688_amd import binding as sq
from test_gpu_q8_rows import cu

pytestmark = pytest.mark.gpu
F16, F32, I32 = torch.float16, torch.float32, torch.int32


def scales_that_round_twice(n):
    """Scales for which some code's product, rounded to fp32 first, falls onto a border of f16 and then to the other side."""
    rng = np.random.default_rng(1)
    found = []
    while len(found) < n:
        s = rng.uniform(2.0 ** -16, 2.0 ** -4, 400000).astype(np.float32)
        for m in range(9, 16):                                  # (a code's mantissa; 8 is a power of two)
            p = m * s.astype(np.float64)
            found += list(s[p.astype(np.float32).astype(np.float16) != p.astype(np.float16)])
    return np.array(found[:n], np.float32)


def test_what_is_read_back_is_rounded_once():
    """Every code times scales that are no powers of two, those among them where rounding twice shows: of both signs, into f16's subnormals and past its end."""
    rng = np.random.default_rng(2)
    picked = scales_that_round_twice(60)
    scales = np.concatenate([picked, -picked[:20], picked[:40] * 2.0 ** rng.integers(-20, 20, 40), [2.0 ** -126, 2.0 ** -127, 1.5 * 2.0 ** -127],
                             [0.0, 3e38, 0.0123, 2.0 ** -30, 2.0 ** 20]]).astype(np.float32)
    n = len(scales)
    codes = np.broadcast_to(np.arange(256, dtype=np.uint8).reshape(1, 1, 2, 128).repeat(8, 2), (n, 1, 16, 128)).copy()
    cache = sq.make_cache(*(cu(codes).view(sq.F8) for _ in range(2)), cu(scales.reshape(n, 1)), cu(-scales[::-1].reshape(n, 1)), cu(np.arange(n, dtype=np.int32).reshape(1, n)))
    sh = sq.make_shape(1, 1, 1, 1, 1, 16 * n, 1.0)
    out = [torch.zeros(1, 1, 16 * n, 128, dtype=F16, device="cuda") for _ in range(2)]
    sq.sq_cache_read(sh, cache, None, cu(np.array([16 * n], np.int32)), *out)
    twice = 0
    for x, s in zip(out, (scales, -scales[::-1])):
        with np.errstate(over="ignore", invalid="ignore"):
            p = ref.VALUES[codes[:, 0]] * s.astype(np.float64)[:, None, None]      # (4 times 24 bits: exact)
            want, other = p.astype(np.float16).reshape(16 * n, 128), p.astype(np.float32).astype(np.float16).reshape(16 * n, 128)
        assert np.array_equal(x[0, 0].cpu().numpy(), want, equal_nan=True)
        twice += ((want != other) & ~np.isnan(want)).sum()
    assert twice >= 100


def test_every_code_times_every_power_of_two_is_read_back():
    n = 254
    scales = np.ldexp(1.0, np.arange(-126, 128)).astype(np.float32)
    codes = np.broadcast_to(np.arange(256, dtype=np.uint8).reshape(1, 1, 2, 128).repeat(8, 2), (n, 1, 16, 128)).copy()
    cache = sq.make_cache(*(cu(codes).view(sq.F8) for _ in range(2)), cu(scales.reshape(n, 1)), cu(-scales.reshape(n, 1)), cu(np.arange(n, dtype=np.int32).reshape(1, n)))
    sh = sq.make_shape(1, 1, 1, 1, 1, 16 * n, 1.0)
    out = [torch.zeros(1, 1, 16 * n, 128, dtype=F16, device="cuda") for _ in range(2)]
    sq.sq_cache_read(sh, cache, None, cu(np.array([16 * n], np.int32)), *out)
    for x, s in zip(out, (scales, -scales)):
        with np.errstate(over="ignore"):
            want = (ref.VALUES[codes[:, 0]] * s.astype(np.float64)[:, None, None]).astype(np.float16).reshape(16 * n, 128)
        assert np.array_equal(x[0, 0].cpu().numpy(), want, equal_nan=True)
