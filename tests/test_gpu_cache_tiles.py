"""GPU: what the attention over the paged cache has to hold at masks, unusable pages, scales, graphs and streams, for units of one, two and four row
tiles.  The tile follows from a bound on the rows: up to 16 rows of a key head's query heads one, up to 32 two, more than 256 four, whatever the batch."""
import numpy as np
import pytest
import torch

import cache_model as cm
import test_gpu_cache as base
from paper_2511_00101_amd import binding as lq
from test_gpu_cache import bf16, f64, ints

pytestmark = pytest.mark.gpu

G = 2                                     # query heads of a key head
BOUNDS = [8, 16, 1000]                    # one, two, four row tiles


def _cache(rng, total, H, d, T, k=None, v=None):
    cache = base.make_cache(rng, total, H, d, T)
    starts = np.concatenate([[0], np.cumsum(total)])
    k = bf16(rng, (int(starts[-1]), H * d)) if k is None else k
    v = bf16(rng, (int(starts[-1]), H * d)) if v is None else v
    base.store(cache, k.cuda(), v.cuda(), None, ints(starts), ints([0] * len(total)))
    return cache, *base.load_all(cache, total)


def _check(out, q, K, V, slots, rows, first, d, scale=None, usable=None):
    for s, slot in enumerate(slots):
        a, b = rows[s], rows[s + 1]
        with np.errstate(invalid="ignore"):
            want = cm.attention(f64(q[a:b]).reshape(b - a, -1, d), K[slot], V[slot], first[s], d ** -0.5 if scale is None else scale,
                                None if usable is None else usable.get(slot))
        base.assert_attention(f64(out[a:b]).reshape(b - a, -1, d), *[np.nan_to_num(x) if i else x for i, x in enumerate(want)], first[s] + b - a)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bound", BOUNDS)
def test_nan_and_unusable_pages_reach_the_rows_that_see_them(bound, d):
    """NaN keys and values that some rows of a tile see and others do not, in whole steps, in masked ones, and in a sequence that is
    split over workgroups; pages that cannot be used at a sequence's start, middle and end."""
    rng = np.random.default_rng(bound + d)
    H, T = 2, 16
    total = [700, 300, 640, 6000]
    at = np.concatenate([[0], np.cumsum(total)])
    k, v = bf16(rng, (int(at[-1]), H * d)), bf16(rng, (int(at[-1]), H * d))
    k[at[0] + 655, d:] = float("nan")                                # second head, for the rows from 655 on
    v[at[0] + 671, 3] = float("inf")                                 # first head, one column, from 671 on
    v[at[1] + 250, :d] = float("nan")
    v[at[3] + 5985, d + 5] = float("nan")                            # a split sequence's last positions
    v[at[3] + 5990, :3] = float("nan")
    cache, K, V = _cache(rng, total, H, d, T, k, v)
    for j, page in ((0, -1), (19, 10 ** 6), (39, -7)):
        cache.table[2, j] = page
    cache.table[3, 100] = cache.refs.numel()
    usable = {2: ~np.isin(np.arange(640) // T, [0, 19, 39]), 3: np.arange(6000) // T != 100}
    slots, first, n = [0, 1, 2, 3], [640, 245, 560, 5950], [60, 55, 80, 50]
    rows = np.concatenate([[0], np.cumsum(n)])
    q = bf16(rng, (int(rows[-1]), G * H * d)).cuda()
    out = base.attend(cache, q, ints(slots), ints(rows), ints(first), bound, expect=lq.LQ_DEVICE_ERR_BAD_SEGMENT)
    assert np.isnan(f64(out)).any() and np.isfinite(f64(out)).any()
    _check(out, q, K, V, slots, rows, first, d, usable=usable)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bound", BOUNDS)
def test_slots_in_any_order_and_scales(bound, d):
    """Slots in another order than the spans, one of them twice, scales of the caller's, scores far apart, one sequence split."""
    rng = np.random.default_rng(bound * 3 + d)
    H, T = 2, 32
    total = [90, 41, 300, 4200]
    rows_in = sum(total)
    cache, K, V = _cache(rng, total, H, d, T, bf16(rng, (rows_in, H * d), 8.0), bf16(rng, (rows_in, H * d), 100.0))
    slots, first, n = [2, 0, 3, 2, 1], [299, 50, 4170, 100, 0], [1, 40, 30, 70, 41]
    rows = np.concatenate([[0], np.cumsum(n)])
    q = bf16(rng, (int(rows[-1]), G * H * d), 8.0).cuda()
    for scale in (1.0, -0.01, 0.0):
        out = base.attend(cache, q, ints(slots), ints(rows), ints(first), bound, scale=scale)
        _check(out, q, K, V, slots, rows, first, d, scale=scale)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bound", BOUNDS)
def test_rows_without_a_usable_page_are_zero(bound, d):
    rng = np.random.default_rng(5)
    total = [4000, 60, 60]
    cache, K, V = _cache(rng, total, 1, d, 16)
    cache.table[0, :250] = -1                                        # (split over workgroups, none of which finds anything)
    cache.table[1, :4] = ints([-1, 9999, -7, 2 ** 31 - 1])
    n = 40
    q = bf16(rng, (3 * n, G * d)).cuda()
    rows = [0, n, 2 * n, 3 * n]
    out = base.attend(cache, q, None, ints(rows), ints([3960, 20, 20]), bound, expect=lq.LQ_DEVICE_ERR_BAD_SEGMENT)
    assert (out[:2 * n] == 0).all()
    _check(out, q, K, V, [2], rows[2:], [20], d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bound", BOUNDS)
@pytest.mark.parametrize("n,total", [(6, 200), (150, 200), (40, 5000)])
def test_elements_of_q_that_are_not_finite(bound, d, n, total):
    """NaN where a row's query head holds a NaN or an infinity, also where all its scores are minus infinity; the others as without it."""
    rng = np.random.default_rng(n)
    H = 2
    cache = base.make_cache(rng, [total], H, d, 32)
    k, v = bf16(rng, (total, H * d)), bf16(rng, (total, H * d))
    k[:, 0] = k[:, 0].abs() + 1                                      # first key head, column 0: positive everywhere
    base.store(cache, k.cuda(), v.cuda(), None, ints([0, total]), ints([0]))
    heads = G * H
    q = bf16(rng, (n, heads * d)).cuda()
    args = (None, ints([0, n]), ints([total - n]), bound)
    good = base.attend(cache, q, *args)
    for i, (col, value) in enumerate([(0, -float("inf")), (0, float("inf")), (d + 3, float("nan")), (heads * d - 1, float("inf"))]):
        bad, row = q.clone(), (i * 7) % n
        bad[row, col] = value
        out = base.attend(cache, bad, *args)
        want = good.clone()
        want[row, col // d * d:(col // d + 1) * d] = float("nan")
        assert torch.equal(out.isnan(), want.isnan())
        assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bound", BOUNDS)
def test_split_tiles_in_a_graph_and_on_two_streams(bound, d):
    """Sequences that several workgroups share, captured once and replayed with eager work and waits between the replays; then the same calls on two
    streams at once, each with its workspace, with rows in front of, between and behind the spans that stay as they were."""
    rng = np.random.default_rng(31)
    H, T = 2, 16
    total = [5000, 2500, 60, 9000]
    cache, _, _ = _cache(rng, total, H, d, T)
    n = [70, 1, 40, 20]
    begin = 3 + np.concatenate([[0], np.cumsum(n)])
    first, begin = ints([t - m for t, m in zip(total, n)]), ints(begin)
    end = 3 + sum(n)
    size = lq.lora_cache_attention_workspace_bytes(cache, G * H, bound)
    ws = [lq.workspace(size) for _ in range(3)]
    q = torch.zeros(end + 5, G * H * d, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7.0)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        for _ in range(2):                                           # (the second call finds the counters as the first one left them)
            lq.lora_cache_attention(q, out, cache, 0, None, begin, first, bound, ws[0])
    inputs = [bf16(rng, tuple(q.shape)).cuda() for _ in range(4)]
    wants = []
    for x in inputs:
        q.copy_(x)
        out.fill_(7.0)
        graph.replay()
        wants.append(base.attend(cache, x, None, begin, first, bound, ws=ws[1]))
        torch.cuda.synchronize()
        assert torch.equal(out, wants[-1]) and (out[:3] == 7).all() and (out[end:] == 7).all() and out[3:end].isfinite().all()
    assert lq.device_error_word(ws[0]) == 0
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [torch.full_like(q, 7.0) for _ in range(12)]
    torch.cuda.synchronize()
    for r, o in enumerate(got):
        with torch.cuda.stream(streams[r % 2]):
            lq.lora_cache_attention(inputs[r % 4], o, cache, 0, None, begin, first, bound, ws[1 + r % 2])
    torch.cuda.synchronize()
    for r, o in enumerate(got):
        assert torch.equal(o, wants[r % 4]), r
    assert lq.device_error_word(ws[1]) == 0 and lq.device_error_word(ws[2]) == 0


@pytest.mark.parametrize("d", [64, 128])
def test_a_serving_loop_of_long_prompts(d):
    """Prompts of more than 128 rows (four row tiles) and single tokens through the grouped LoRA call, reserve, store and attention, with a fork and a
    compaction between the steps: every output against the model, whose cached values follow the projections' rows."""
    rng = np.random.default_rng(41)
    H, T = 2, 16
    w = G * H * d
    cache = lq.PagedCache.empty(2, H, d, T, 120, 6, 40)
    layers = [[lq.AdapterTable.from_tensors([bf16(rng, (8, w), 0.05).cuda() for _ in range(2)], [bf16(rng, (8, c), 0.05).cuda() for _ in range(2)],
                                            [1.0, 2.0]) for c in (w, H * d, H * d)] for _ in range(2)]
    steps = [([0, 1], [150, 37], [0, 0]), ([1, 0], [140, 1], [37, 150]), ([0, 1, 4], [1, 1, 131], [151, 177, 151]), ([4, 0], [1, 1], [282, 152])]
    log = base._serve(cache, layers, steps, rng, compact_at=(3,), fork_at=(2,))
    seqs = {}
    for layer, slots, n, done, q, k, v, out in log:
        at = 0
        for s, m, f in zip(slots, n, done):
            if (layer, s) not in seqs:
                seqs[layer, s] = (cm.Rows(H, d), cm.Rows(H, d))
                if f:                                                # the forked request: what its parent (slot 0) held then
                    for mine, theirs in zip(seqs[layer, s], seqs[layer, 0]):
                        mine.values, mine.exps = theirs.values[:f].copy(), dict(theirs.exps)
            for rows, x in zip(seqs[layer, s], (k, v)):
                rows.store(f, f64(x[at:at + m]).reshape(m, H, d))
            K, V = seqs[layer, s]
            want = cm.attention(f64(q[at:at + m]).reshape(m, G * H, d), K.values, V.values, f, d ** -0.5)
            base.assert_attention(f64(out[at:at + m]).reshape(m, G * H, d), *want, f + m)
            at += m
