"""GPU: spans of the paged cache's calls that cannot be used."""
import numpy as np
import pytest
import torch

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
