"""GPU: spans of the paged cache's calls that cannot be used."""
import numpy as np
import pytest
import torch

import cache_model as cm
import test_gpu_cache as base
from paper_2511_00101_amd import binding as lq
from test_gpu_cache import bf16, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("starts,stored", [
    ([-4, 4, 8, 12], {1: 4, 2: 4}),                  # rows in front of the matrix
    ([-20, 4, 8, 12], {1: 4, 2: 4}),
    ([-2 ** 31, 0, 4, 8], {1: 4, 2: 4}),
    ([0, 20, 4, 8], {0: 20}),                        # rows that run backwards (spans behind them may be left out too)
    ([0, 4, 8, 99], {0: 4, 1: 4}),                   # rows behind the matrix
    ([0, 4, 2 ** 31 - 1, 2 ** 31 - 1], {0: 4}),
    ([24, 24, 25, 24], {}),
])
def test_rows_outside_the_matrix_are_reported_by_store_and_load(starts, stored):
    """A span that lies outside the row matrices is skipped and reported, wherever among the spans it stands; the good ones in front
    of it are served."""
    rng = np.random.default_rng(1)
    cache = base.make_cache(rng, [20, 20, 20], 2, 64, 16)
    k, v = bf16(rng, (24, 128)).cuda(), bf16(rng, (24, 128)).cuda()
    args = (None, ints(starts), ints([0, 0, 0]))
    for call in (lq.lora_cache_store_rows, lq.lora_cache_load_rows):
        ws = base.ws_for(cache)
        call(k.clone(), v.clone(), cache, 0, *args, ws)
        torch.cuda.synchronize()
        assert lq.device_error_word(ws) == lq.LQ_DEVICE_ERR_BAD_SEGMENT, call.__name__
    for s, n in stored.items():
        codes = cache.pages[0][cache.table[s, 0].long(), :16 * 64].view(16, 64)
        assert not (codes[:n] == 255).any() and (codes[n:] == 255).all(), s


@pytest.mark.parametrize("d,bound,n", [(128, 1, 716), (128, 1, 721), (128, 1, 1700), (128, 1, 3960), (64, 1, 815), (64, 1, 1900), (64, 1, 1950),
                                       (64, 30, 1200), (128, 30, 1700), (64, 1000, 480), (128, 1000, 500), (128, 1000, 1200)])
def test_as_many_spans_as_fit_a_workgroups_memory_and_more(d, bound, n):
    """Short sequences and a few longer ones among them, where the spans' places in on-chip memory leave room for fewer workgroups: the rows of
    some are compared with the model, the others with calls of 200 spans."""
    rng = np.random.default_rng(n)
    kinds = [(0, 1), (17, 1), (40, 2), (300, 1), (90, 1), (5, 3)]
    cache = base.make_cache(rng, [f + m for f, m in kinds], 1, d, 16)
    total = [f + m for f, m in kinds]
    starts = np.concatenate([[0], np.cumsum(total)])
    k, v = bf16(rng, (int(starts[-1]), d)), bf16(rng, (int(starts[-1]), d))
    base.store(cache, k.cuda(), v.cuda(), None, ints(starts), ints([0] * len(kinds)))
    K, V = base.load_all(cache, total)
    slot = rng.choice(len(kinds), n)
    first, rows = np.array([kinds[s][0] for s in slot]), np.array([kinds[s][1] for s in slot])
    begin = np.concatenate([[0], np.cumsum(rows)])
    q = bf16(rng, (int(begin[-1]), 2 * d)).cuda()
    out = base.attend(cache, q, ints(slot), ints(begin), ints(first), bound)
    for a in range(0, n, 200):
        b = min(a + 200, n)
        part = base.attend(cache, q[begin[a]:begin[b]], ints(slot[a:b]), ints(begin[a:b + 1] - begin[a]), ints(first[a:b]), bound)
        whole, part = base.f64(out[begin[a]:begin[b]]), base.f64(part)
        # two roundings to bf16 of sums that differ by their order (and by where their maxima were), of values up to 8
        assert np.isfinite(whole).all() and np.abs(whole - part).max() <= 2 * 8 * 2.0 ** -8
    for s in [0, 1, 199, 200, n // 2, n - 2, n - 1]:
        f, m = kinds[slot[s]]
        want = cm.attention(base.f64(q[begin[s]:begin[s + 1]]).reshape(m, 2, d), K[slot[s]], V[slot[s]], f, d ** -0.5)
        base.assert_attention(base.f64(out[begin[s]:begin[s + 1]]).reshape(m, 2, d), *want, f + m)
