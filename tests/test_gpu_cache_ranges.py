"""GPU: the attention over the paged cache where numbers lie far apart (elements of q, scales), for every row tile."""
import numpy as np
import pytest
import torch

import cache_model as cm
import test_gpu_cache as base
from test_gpu_cache import bf16, f64, ints

pytestmark = pytest.mark.gpu


def _spread_q(rng, n, heads, d, log2_std):
    """Rows with one element of 256 a head, and the others smaller by 2^(log2_std - 8): bf16 values of all mantissas and both signs."""
    q = bf16(rng, (n, heads, d), 2.0 ** log2_std)
    col = rng.integers(0, d, heads)
    for h in range(heads):
        q[:, h, col[h]] = 256.0
    return q.reshape(n, heads * d), col


# log2_std -16 is 2^-24 of the largest.  Elements below 2^-31 of it may be off by 2^-40 of it (2^-32); 0.7 % of the others' elements are below
# 2^-7 of their standard deviation, so what that adds to a score is below 2^-16 * 0.007 of the sum of its products' magnitudes, a
# hundredth of the bound that fp32 sums have.
@pytest.mark.parametrize("log2_std", [4, -4, -8, -12, -16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bound", [1, 30, 1000])
def test_small_elements_of_q_beside_a_large_one_count(bound, d, log2_std):
    """Keys are zero where q is large, so that the scores come from q's small elements alone."""
    rng = np.random.default_rng(d + 10 * bound - log2_std)
    n, total, heads, H = 50, 250, 2, 2
    cache = base.make_cache(rng, [total], H, d, 16)
    q, col = _spread_q(rng, n, heads, d, log2_std)
    k, v = bf16(rng, (total, H * d)), bf16(rng, (total, H * d))
    for h in range(H):
        k[:, h * d + col[h]] = 0.0
    base.store(cache, k.cuda(), v.cuda(), None, ints([0, total]), ints([0]))
    K, V = base.load_all(cache, [total])
    scale = 2.0 ** -log2_std * 4 / d ** 0.5          # scores of standard deviation 4
    out = base.attend(cache, q.cuda(), None, ints([0, n]), ints([total - n]), bound, scale=scale)
    want = cm.attention(f64(q).reshape(n, heads, d), K[0], V[0], total - n, scale)
    base.assert_attention(f64(out).reshape(n, heads, d), *want, total)


def test_two_elements_of_q_far_apart():
    """q = (256, 2^-15, 0 ...) against keys (0, +-2^16, 0 ...): the second element decides every score."""
    n, d = 64, 128
    rng = np.random.default_rng(0)
    cache = base.make_cache(rng, [n], 1, d, 16)
    k, v = torch.zeros(n, d, dtype=torch.bfloat16), bf16(rng, (n, d))
    k[:, 1] = torch.from_numpy(np.where(rng.random(n) < 0.5, -1.0, 1.0) * 2.0 ** 16).to(torch.bfloat16)
    base.store(cache, k.cuda(), v.cuda(), None, ints([0, n]), ints([0]))
    K, V = base.load_all(cache, [n])
    q = torch.zeros(n, d, dtype=torch.bfloat16)
    q[:, 0], q[:, 1] = 256.0, 2.0 ** -15
    want = cm.attention(f64(q).reshape(n, 1, d), K[0], V[0], 0, 1.0)
    for bound in (1, 30, 1000):
        out = base.attend(cache, q.cuda(), None, ints([0, n]), ints([0]), bound, scale=1.0)
        base.assert_attention(f64(out).reshape(n, 1, d), *want, n)


@pytest.mark.parametrize("top", [1.0, 3.3e38, 1e-30, 2.0 ** -120])
def test_rows_of_q_of_every_size(top):
    """Rows whose elements reach from bf16's largest values down to its smallest normal ones, with a scale that brings the scores back."""
    n, d, total = 20, 128, 100
    rng = np.random.default_rng(3)
    cache = base.make_cache(rng, [total], 1, d, 32)
    huge = top > 1e30                                 # keys that keep the scores within fp32
    k, v = bf16(rng, (total, d), 2.0 ** -20 if huge else 1.0), bf16(rng, (total, d))
    base.store(cache, k.cuda(), v.cuda(), None, ints([0, total]), ints([0]))
    K, V = base.load_all(cache, [total])
    q = (torch.from_numpy(rng.uniform(-1, 1, (n, d))).double() * top).to(torch.bfloat16)
    scale = 8 / top / d ** 0.5 * (2.0 ** 20 if huge else 1.0)
    for bound in (1, 30, 1000):
        out = base.attend(cache, q.cuda(), None, ints([0, n]), ints([total - n]), bound, scale=scale)
        want = cm.attention(f64(q).reshape(n, 1, d), K[0], V[0], total - n, scale)
        base.assert_attention(f64(out).reshape(n, 1, d), *want, total)


@pytest.mark.parametrize("scale", [0.0, 1e-38, -3e-39, 2e-33])
@pytest.mark.parametrize("bound", [1, 30, 1000])
def test_tiny_scales_of_huge_scores(bound, scale):
    """q . K of up to 2^120 and a scale that makes little or nothing of them."""
    n, d, total = 20, 128, 100
    rng = np.random.default_rng(4)
    cache = base.make_cache(rng, [total], 1, d, 32)
    k, v = bf16(rng, (total, d), 2.0 ** 100), bf16(rng, (total, d))
    base.store(cache, k.cuda(), v.cuda(), None, ints([0, total]), ints([0]))
    K, V = base.load_all(cache, [total])
    q = bf16(rng, (n, d), 2.0 ** 15)
    out = base.attend(cache, q.cuda(), None, ints([0, n]), ints([total - n]), bound, scale=scale)
    want = cm.attention(f64(q).reshape(n, 1, d), K[0], V[0], total - n, float(np.float32(scale)))
    base.assert_attention(f64(out).reshape(n, 1, d), *want, total)
