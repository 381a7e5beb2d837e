"""GPU: the paged 8-bit key/value cache (rows in and out, attention, page management) against the plain 64-bit model.

Tolerance of the attention, element by element: out is one rounding to bf16 (2^-8 |o|); the probabilities are rounded to bf16 before the
product with V, which moves the sum by at most 2^-8 sum p|v|, and with it the sum that it is divided by, if that is made of the rounded
ones, by as much again; a score is an fp32 sum of at most 128 products (bound 136 * 2^-24 sum |q k| scale, also for the
rounding of its scaling), which changes every p by that factor twice (its own and the divisor's); exp2 and the sums over n positions add
2^-20 + n 2^-24 at most."""
import numpy as np
import pytest
import torch

import cache_model as cm
from paper_2511_00101_amd import binding as lq
from paper_2511_00101_amd import synth

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def bf16(rng, shape, std=1.0):
    return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32) * np.float32(std)).to(torch.bfloat16)


def f64(t):
    return t.detach().double().cpu().numpy()


def make_cache(rng, total, H, d, T, n_layers=1, poison=True, spare=3):
    """A cache whose slots hold sequences of `total` positions in pages taken at random; pages poisoned with NaN codes and scales."""
    used = [-(-t // T) for t in total]
    cache = lq.PagedCache.empty(n_layers, H, d, T, sum(used) + spare, len(total) + 1, max(max(used), 1) + 1)
    order = rng.permutation(sum(used) + spare)
    table, refs, at = np.full(tuple(cache.table.shape), -1), np.zeros(len(order)), 0
    for s, k in enumerate(used):
        table[s, :k] = order[at:at + k]
        refs[order[at:at + k]] = 1
        at += k
    cache.table.copy_(ints(table))
    cache.refs.copy_(ints(refs))
    cache.lens.copy_(ints(list(total) + [0]))
    if poison:
        for p in cache.pages:
            p.fill_(255)
    return cache


def ws_for(cache, n=64):
    return lq.workspace(lq.lora_cache_workspace_bytes(cache, n))


def attend(cache, q, slots, row_starts, first, max_rows, layer=0, scale=None, out=None, ws=None, expect=0):
    heads = q.shape[1] // cache.head_dim
    ws = lq.workspace(lq.lora_cache_attention_workspace_bytes(cache, heads, max_rows)) if ws is None else ws
    out = torch.full_like(q, 7.0) if out is None else out
    lq.lora_cache_attention(q, out, cache, layer, slots, row_starts, first, max_rows, ws, scale)
    torch.cuda.synchronize()
    assert lq.device_error_word(ws) == expect
    return out


def assert_attention(got, want, mag, slack, n):
    tol = 2.0 ** -8 * np.abs(want) + (2 * 2.0 ** -8 + 2 * 136 * 2.0 ** -24 * slack + 2.0 ** -20 + n * 2.0 ** -24) * mag + 1e-30
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bad = np.abs(got - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4])


def store(cache, k, v, slots, row_starts, first, layer=0, expect=0):
    ws = ws_for(cache)
    lq.lora_cache_store_rows(k, v, cache, layer, slots, row_starts, first, ws)
    torch.cuda.synchronize()
    assert lq.device_error_word(ws) == expect


def load_all(cache, total, layer=0):
    """K and V of the first slots' sequences as float64 [position, head, d], one array a slot."""
    starts = np.concatenate([[0], np.cumsum(total)])
    w = cache.n_kv_heads * cache.head_dim
    k = torch.zeros(max(int(starts[-1]), 1), w, dtype=torch.bfloat16, device="cuda")
    v, ws = torch.zeros_like(k), ws_for(cache)
    lq.lora_cache_load_rows(k, v, cache, layer, None, ints(starts), ints([0] * len(total)), ws)
    torch.cuda.synchronize()
    assert lq.device_error_word(ws) == 0
    cut = lambda t: [f64(t[a:b]).reshape(-1, cache.n_kv_heads, cache.head_dim) for a, b in zip(starts[:-1], starts[1:])]  # noqa: E731
    return cut(k), cut(v)


# ---- rows in and out -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,d,T", [(1, 64, 16), (2, 128, 16), (3, 64, 32), (8, 128, 64), (5, 128, 256)])
def test_rows_stored_in_steps_read_back_as_the_model_has_them(H, d, T):
    """Three sequences that grow by steps of different sizes; later steps larger, so that scales grow under codes that are there, and
    values with NaN, infinities, zeros and both ends of bf16's range."""
    rng = np.random.default_rng(H * 100 + d + T)
    steps = [[17, 1, 1, 14, 40, 3], [1, 1, 1, 1, 1, 1], [33, 15, 16, 0, 300, 7]]
    total = [sum(s) for s in steps]
    cache = make_cache(rng, total, H, d, T)
    model = [(cm.Rows(H, d), cm.Rows(H, d)) for _ in steps]
    done = [0, 0, 0]
    for i in range(6):
        n = [s[i] for s in steps]
        k = bf16(rng, (sum(n) + 5, H * d), 4.0 ** (i - 2))          # rows before, between and behind the spans belong to nobody
        v = bf16(rng, (sum(n) + 5, H * d), 3.0 ** (2 - i))
        if i == 4:
            k[6, :7] = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 3.3e38, 1e-40])
            v[30, 5:9] = torch.tensor([float("nan"), 2.0 ** -110, float("inf"), 1.0])
            v[20] = 0.0
        order = [2, 0, 1]
        starts = 2 + np.concatenate([[0], np.cumsum([n[s] for s in order])])
        store(cache, k.cuda(), v.cuda(), ints(order), ints(starts), ints([done[s] for s in order]))
        for s, a in zip(order, starts):
            for m, x in zip(model[s], (k, v)):
                m.store(done[s], f64(x[a:a + n[s]]).reshape(-1, H, d))
            done[s] += n[s]
    got_k, got_v = load_all(cache, total)
    for s in range(3):
        assert np.array_equal(got_k[s], model[s][0].values, equal_nan=True)
        assert np.array_equal(got_v[s], model[s][1].values, equal_nan=True)


def test_page_layout_and_untouched_pages():
    """Codes and exponent bytes where the header says they are; pages and rows of nobody are not written."""
    H, d, T = 2, 64, 32
    rng = np.random.default_rng(5)
    cache = make_cache(rng, [40], H, d, T)
    before = cache.pages[0].clone()
    k, v = bf16(rng, (40, H * d)), bf16(rng, (40, H * d), 0.1)
    store(cache, k.cuda(), v.cuda(), None, ints([0, 40]), ints([0]))
    got = cache.pages[0].cpu().numpy()
    page = cache.table[0].cpu().numpy()
    for t in range(40):
        p, i = got[page[t // T]], t % T
        for h in range(H):
            ek, ev = p[2 * T * d * H + (h * (T // 16) + i // 16) * 2:][:2].astype(int) - 127
            blk = slice(t // 16 * 16, min(t // 16 * 16 + 16, 40))
            for x, e, codes in ((k, ek, [p[2 * T * d * h + i * d + c] for c in range(d)]),
                                (v, ev, [p[2 * T * d * h + T * d + (i // 4) * 4 * d + 4 * c + i % 4] for c in range(d)])):
                assert e == cm.block_exponent(f64(x)[blk, h * d:(h + 1) * d])
                assert np.array_equal(cm.e4m3_value(codes), cm.e4m3_round(f64(x)[t, h * d:(h + 1) * d] * 2.0 ** -e))
    others = np.setdiff1d(np.arange(len(got)), page[:2])
    assert np.array_equal(got[others], before.cpu().numpy()[others])


def test_rows_with_leading_dimensions_and_slices_of_a_projection():
    """k and v as column slices of one matrix (a fused q,k,v output), read back into slices of another, whose other columns stay."""
    H, d, T = 4, 128, 16
    rng = np.random.default_rng(6)
    cache = make_cache(rng, [21, 3], H, d, T)
    qkv = bf16(rng, (24, 3 * H * d + 8)).cuda()
    k, v = qkv[:, H * d:2 * H * d], qkv[:, 2 * H * d:3 * H * d]
    store(cache, k, v, None, ints([0, 21, 24]), ints([0, 0]))
    back = torch.full((30, 2 * H * d + 16), 3.0, dtype=torch.bfloat16, device="cuda")
    ws = ws_for(cache)
    lq.lora_cache_load_rows(back[:, :H * d], back[:, H * d + 16:], cache, 0, ints([1, 0]), ints([1, 4, 24]), ints([0, 1]), ws)
    torch.cuda.synchronize()
    model = []
    for x in (k, v):
        a, b = cm.Rows(H, d), cm.Rows(H, d)
        a.store(0, f64(x[:21]).reshape(-1, H, d))
        b.store(0, f64(x[21:24]).reshape(-1, H, d))
        model.append(np.concatenate([b.values, a.values[1:]]).reshape(23, -1))
    assert np.array_equal(f64(back[1:24, :H * d]), model[0]) and np.array_equal(f64(back[1:24, H * d + 16:]), model[1])
    assert (back[0] == 3).all() and (back[24:] == 3).all() and (back[:, H * d:H * d + 16] == 3).all()


def test_spans_that_cannot_be_used_are_skipped_and_reported():
    H, d, T = 1, 64, 16
    rng = np.random.default_rng(7)
    cache = make_cache(rng, [20, 20, 20, 20], H, d, T)
    cache.table[3, 1] = 10 ** 6                                      # a page that does not exist
    cache.refs[cache.table[2, 0].long()] = 2                         # a shared page
    k, v = bf16(rng, (24, d)).cuda(), bf16(rng, (24, d)).cuda()
    good = [0, 4, 8, 12, 16, 20]
    for slots, starts, first, stored in (
            ([0, 1, 99, -1, 5], good, [0, 0, 0, 0, 8], {0: 4, 1: 4}),                        # slots out of range
            ([0, 1, 0, 1, 0], good, [0, 17, -1, 0, 2 ** 31 - 1], {0: 4, 1: 4}),              # positions out of the sequence
            ([0, 1, 99, 1, 0], [0, 4, 2, 8, 99, 99], [0, 0, 8, 0, 0], {0: 4}),               # rows that run backwards, or past the matrix
            ([0, 2, 3, 1, 9], good, [0, 0, 16, 0, 4], {0: 4, 1: 4})):                        # a shared page, a bad page
        for p in cache.pages:
            p.fill_(255)
        ws = ws_for(cache)
        lq.lora_cache_store_rows(k, v, cache, 0, ints(slots), ints(starts), ints(first), ws)
        torch.cuda.synchronize()
        assert lq.device_error_word(ws) == lq.LQ_DEVICE_ERR_BAD_SEGMENT
        with pytest.raises(lq.LqDeviceError):
            lq.raise_on_device_error(ws)
        for s in (0, 1):
            codes = cache.pages[0][cache.table[s, 0].long(), :16 * d].view(16, d)
            n = stored.get(s, 0)
            assert (codes[n:] == 255).all() and not (codes[:n] == 255).any(), (slots, s)
        assert (cache.pages[0][cache.table[2, 0].long()] == 255).all()


# ---- attention -------------------------------------------------------------------------------------------------------
ATTENTION = [
    # heads, kv heads, d, T, spans (first, rows), max_rows
    (1, 1, 64, 16, [(0, 1)], 1),
    (4, 2, 64, 16, [(0, 1), (15, 1), (16, 1), (31, 1), (32, 1), (63, 1), (200, 1)], 1),
    (8, 8, 128, 32, [(1, 1), (100, 1), (127, 1), (128, 1)], 1),
    (32, 8, 128, 64, [(5, 1), (0, 1), (777, 1), (2100, 1)], 1),
    (16, 1, 128, 128, [(300, 1), (6, 1)], 1),
    (48, 2, 64, 16, [(70, 1), (64, 2)], 2),                       # more than 16 query heads per key head
    (6, 2, 128, 256, [(0, 5), (255, 5), (256, 3), (40, 0), (700, 4)], 5),
    (4, 4, 64, 32, [(0, 16), (17, 17), (31, 33), (100, 48)], 48),
    (8, 2, 128, 16, [(0, 70), (33, 129), (250, 1)], 129),
    (3, 1, 64, 64, [(0, 200), (1000, 65)], 200),
    (2, 2, 128, 16, [(0, 300)], 1),                              # max_rows is no bound here: still right
    (2, 1, 128, 16, [(9, 1)] * 70, 4),                           # more spans than a wave has lanes
    (1, 1, 64, 16, [(20000, 1)], 1),                             # a long axis and nothing else to spread
    (5, 5, 128, 64, [(6000, 2), (3, 2)], 2),
    (8, 4, 64, 16, [(i % 37, 1) for i in range(300)], 1),        # more units than workgroups: a unit per wave; more spans than threads
    (4, 2, 128, 16, [(i * 7 % 90, 1) for i in range(450)], 1),
    (2, 1, 64, 16, [(i % 5, 1) for i in range(1100)], 1),        # more spans than are kept
    (1, 1, 64, 16, [(i % 2, 1) for i in range(4096)], 1),        # as many spans as a call takes
    (1, 1, 128, 16, [(i % 2, 1) for i in range(4096)], 60),      # (with four tiles)
    (4, 2, 128, 16, [(5000, 3), (2500, 1), (1, 2)], 3),          # pages beyond a wave's first 64, chunks in byte counters
    (8, 2, 128, 64, [(3000, 1), (3100, 1)] + [(900, 1)] * 10, 1),   # chunks in four-bit counters
    (6, 1, 128, 32, [(4000, 5), (10, 5)], 5),                    # a draft split
    (4, 1, 64, 16, [(2600, 40), (0, 40)], 40),                   # a prompt split
    (8, 1, 128, 128, [(1500, 20), (2047, 1)], 20),
    (16, 1, 128, 16, [(700, 8)], 8),                             # 128 rows: four units of two tiles
    (12, 4, 64, 32, [(3, 14), (60, 13)] * 36, 14),               # few rows, many units: four tiles
    # four tiles by a bound far above (what the rows are does not matter)
    (4, 4, 64, 32, [(0, 16), (17, 17), (31, 33), (100, 48)], 1000),
    (8, 2, 128, 16, [(0, 70), (33, 129), (250, 1)], 1000),
    (6, 2, 128, 256, [(0, 5), (255, 5), (256, 3), (40, 0), (700, 4)], 1000),
    (4, 1, 64, 16, [(2600, 40), (0, 40)], 1000),
    (16, 1, 128, 128, [(3500, 20), (2047, 1), (9, 8)], 1000),    # two tiles and more, in chunks, with rows left over
    (2, 2, 128, 16, [(9000, 70), (20, 3)], 1000),
    (1, 1, 128, 16, [(20000, 1)], 1000),
    (8, 8, 64, 16, [(i % 29, 1 + i % 9) for i in range(140)], 1000),    # units drawn, by key heads
    (8, 8, 128, 16, [(i * 7 % 129, 1 + i % 5) for i in range(150)], 1000),
    (5, 5, 128, 32, [(i % 40, 1 + i % 3) for i in range(230)], 1000),   # by one counter
    (2, 2, 128, 16, [(i * 3 % 50, 1 + i % 70) for i in range(260)], 1000),  # more spans than are kept
    # two tiles by a bound
    (4, 4, 64, 32, [(0, 16), (17, 17), (31, 33), (100, 48)], 30),
    (3, 1, 128, 64, [(0, 100), (1000, 65), (4000, 1)], 20),
    (4, 2, 128, 16, [(i * 5 % 60, 1 + i % 11) for i in range(600)], 10),
    # many about equally long: a unit per wave beyond the short ones
    (8, 8, 64, 16, [(560 + i % 40, 1) for i in range(140)], 1),
    (16, 8, 128, 64, [(600 - i % 33, 1) for i in range(105)], 1),
]


@pytest.mark.parametrize("heads,H,d,T,spans,max_rows", ATTENTION)
def test_attention_against_the_model(heads, H, d, T, spans, max_rows):
    rng = np.random.default_rng(heads * 1000 + d + T + len(spans))
    total = [f + n for f, n in spans]
    cache = make_cache(rng, total, H, d, T)
    starts = np.concatenate([[0], np.cumsum(total)])
    k, v = bf16(rng, (int(starts[-1]), H * d)), bf16(rng, (int(starts[-1]), H * d))
    k *= torch.exp(torch.from_numpy(rng.standard_normal((1, H * d)).astype(np.float32)) * 0.5).to(torch.bfloat16)
    store(cache, k.cuda(), v.cuda(), None, ints(starts), ints([0] * len(spans)))
    K, V = load_all(cache, total)
    rows = np.concatenate([[0], np.cumsum([n for _, n in spans])]) + 3
    n_rows = int(rows[-1]) + 2
    wide = bf16(rng, (n_rows, heads * d + 24)).cuda()                # q with a leading dimension
    q = wide[:, 8:8 + heads * d]
    out_wide = torch.full((n_rows, heads * d + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    out = out_wide[:, :heads * d]
    attend(cache, q, None, ints(rows), ints([f for f, _ in spans]), max_rows, out=out)
    assert (out_wide[:, heads * d:] == 7).all() and (out[:3] == 7).all() and (out[n_rows - 2:] == 7).all()
    for s, (f, n) in enumerate(spans):
        a = int(rows[s])
        if n:
            want = cm.attention(f64(q[a:a + n]).reshape(n, heads, d), K[s], V[s], f, d ** -0.5)
            assert_attention(f64(out[a:a + n]).reshape(n, heads, d), *want, f + n)
    again = attend(cache, q, None, ints(rows), ints([f for f, _ in spans]), max_rows)
    assert torch.equal(again[3:n_rows - 2], out[3:n_rows - 2])       # the same from run to run


@pytest.mark.parametrize("max_rows,heads", [(1, 8), (40, 4)])
def test_attention_orders_slots_and_scales(max_rows, heads):
    """Slots in another order than the spans, the same slot twice, a scale of the caller's, scores far apart."""
    rng = np.random.default_rng(heads)
    H, d, T = 2, 64, 32
    total = [90, 41, 300]
    cache = make_cache(rng, total, H, d, T)
    starts = np.concatenate([[0], np.cumsum(total)])
    k, v = bf16(rng, (431, H * d), 8.0), bf16(rng, (431, H * d), 100.0)
    store(cache, k.cuda(), v.cuda(), None, ints(starts), ints([0] * 3))
    K, V = load_all(cache, total)
    slots, first = [2, 0, 2, 1], [299, 50, 100, 0]
    n = [1, max_rows, max_rows, min(max_rows, 41)]
    rows = np.concatenate([[0], np.cumsum(n)])
    q = bf16(rng, (int(rows[-1]), heads * d), 8.0).cuda()
    for scale in (1.0, -0.01, 0.0):
        out = attend(cache, q, ints(slots), ints(rows), ints(first), max_rows, scale=scale)
        for s in range(4):
            a, b = rows[s], rows[s + 1]
            want = cm.attention(f64(q[a:b]).reshape(-1, heads, d), K[slots[s]], V[slots[s]], first[s], scale)
            assert_attention(f64(out[a:b]).reshape(-1, heads, d), *want, 300)


@pytest.mark.parametrize("max_rows", [1, 50])
def test_what_a_row_does_not_see_leaves_no_trace(max_rows):
    """Pages are poisoned beyond the sequences; positions that later rows see hold NaN; a page number is unusable."""
    rng = np.random.default_rng(max_rows)
    H, heads, d, T = 2, 4, 128, 16
    total = [60, 33, 40]
    cache = make_cache(rng, total, H, d, T)
    starts = np.concatenate([[0], np.cumsum(total)])
    k, v = bf16(rng, (133, H * d)), bf16(rng, (133, H * d))
    k[41, d:] = float("nan")                                         # slot 0: keys of position 41, second head
    v[50, 3] = float("inf")                                          # values of position 50, first head, one column
    v[60 + 20, :d] = float("nan")                                    # slot 1, position 20, first head
    store(cache, k.cuda(), v.cuda(), None, ints(starts), ints([0] * 3))
    K, V = load_all(cache, total)
    cache.table[2, 1] = -5                                           # slot 2: positions 16 .. 31 unusable
    if max_rows == 1:
        slots, first = [0, 0, 0, 0, 0, 1, 1, 1, 2, 2, 2], [40, 41, 49, 50, 59, 19, 20, 32, 10, 20, 39]
        n = [1] * len(slots)
    else:
        slots, first, n = [0, 1, 2], [10, 0, 0], [50, 33, 40]
    rows = np.concatenate([[0], np.cumsum(n)])
    q = bf16(rng, (int(rows[-1]), heads * d)).cuda()
    out = attend(cache, q, ints(slots), ints(rows), ints(first), max_rows, expect=lq.LQ_DEVICE_ERR_BAD_SEGMENT)
    for s in range(len(slots)):
        a, b = rows[s], rows[s + 1]
        usable = ~((np.arange(40) >= 16) & (np.arange(40) < 32)) if slots[s] == 2 else None
        with np.errstate(invalid="ignore"):
            want = cm.attention(f64(q[a:b]).reshape(-1, heads, d), K[slots[s]], V[slots[s]], first[s], d ** -0.5, usable)
        assert_attention(f64(out[a:b]).reshape(-1, heads, d), *[np.nan_to_num(x) if i else x for i, x in enumerate(want)], 60)


@pytest.mark.parametrize("heads,H,d,n", [(4, 2, 64, 1), (4, 2, 128, 1), (8, 2, 128, 6), (4, 4, 64, 150), (4, 2, 128, 150)])
def test_rows_of_q_that_are_not_finite(heads, H, d, n):
    """NaN where a row's query head holds a NaN or an infinity (also where all its scores are minus infinity), the others as if it were not there."""
    rng = np.random.default_rng(n)
    cache = make_cache(rng, [200], H, d, 32)
    k, v = bf16(rng, (200, H * d)), bf16(rng, (200, H * d))
    k[:, 0] = k[:, 0].abs() + 1                                      # first key head, column 0: positive everywhere
    store(cache, k.cuda(), v.cuda(), None, ints([0, 200]), ints([0]))
    q = bf16(rng, (n, heads * d)).cuda()
    good = attend(cache, q, None, ints([0, n]), ints([200 - n]), n)
    for i, (col, value) in enumerate([(0, -float("inf")), (0, float("inf")), (d + 3, float("nan")), (heads * d - 1, float("inf"))]):
        bad = q.clone()
        row = (i * 7) % n
        bad[row, col] = value
        out = attend(cache, bad, None, ints([0, n]), ints([200 - n]), n)
        want = good.clone()
        want[row, col // d * d:(col // d + 1) * d] = float("nan")
        assert torch.equal(out.isnan(), want.isnan())
        assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))


def test_a_cache_of_another_device_is_refused():
    cache = make_cache(np.random.default_rng(0), [5], 1, 64, 16)
    cache.device_index += 1                                          # as if its tensors lay there
    q = torch.zeros(1, 64, dtype=torch.bfloat16, device="cuda")
    ws = ws_for(cache)
    with pytest.raises(ValueError, match="current device"):
        lq.lora_cache_attention(q, torch.zeros_like(q), cache, 0, None, ints([0, 1]), ints([4]), 1, ws)
    with pytest.raises(ValueError, match="current device"):
        lq.lora_cache_free(cache, ints([0]), ws)


def test_tensors_of_another_device_and_no_workspace_are_refused():
    cache = make_cache(np.random.default_rng(0), [5], 1, 64, 16)
    q = torch.zeros(1, 64, dtype=torch.bfloat16, device="cuda")
    good = dict(q=q, out=torch.zeros_like(q), slots=ints([0]), row_starts=ints([0, 1]), first=ints([4]),
                workspace=lq.workspace(lq.lora_cache_attention_workspace_bytes(cache, 1, 1)))
    for name in good:
        with pytest.raises(ValueError, match="another device"):
            lq.lora_cache_attention(cache=cache, layer=0, max_rows=1, **{**good, name: good[name].cpu()})
    ws = ws_for(cache)
    for call in (lambda i, w: lq.lora_cache_reserve(cache, ints([0]), i, w), lambda i, w: lq.lora_cache_free(cache, i, w),
                 lambda i, w: lq.lora_cache_fork(cache, ints([0]), i, w), lambda i, w: lq.lora_cache_compact(cache, i, w),
                 lambda i, w: lq.lora_cache_store_rows(q, good["out"], cache, 0, i, good["row_starts"], good["first"], w),
                 lambda i, w: lq.lora_cache_load_rows(q, good["out"], cache, 0, i, good["row_starts"], good["first"], w)):
        with pytest.raises(ValueError, match="another device"):
            call(torch.zeros(1, dtype=torch.int32), ws)
        with pytest.raises(ValueError, match="another device"):
            call(ints([0]), ws.cpu())
        with pytest.raises(lq.LqError) as err:
            call(ints([0]), None)
        assert err.value.status == lq.LQ_ERR_WORKSPACE
    with pytest.raises(lq.LqError) as err:
        lq.lora_cache_attention(cache=cache, layer=0, max_rows=1, **{**good, "workspace": None})
    assert err.value.status == lq.LQ_ERR_WORKSPACE
    assert cache.lens.tolist() == [5, 0]


@pytest.mark.parametrize("max_rows", [1, 20])
def test_rows_that_see_no_usable_page_are_zero(max_rows):
    rng = np.random.default_rng(3)
    cache = make_cache(rng, [40, 40], 1, 64, 16)
    cache.table[0, :3] = ints([-1, 9999, -7])
    store(cache, bf16(rng, (40, 64)).cuda(), bf16(rng, (40, 64)).cuda(), ints([1]), ints([0, 40]), ints([0]))
    n = min(max_rows, 20)
    q = bf16(rng, (2 * n, 128)).cuda()
    out = attend(cache, q, None, ints([0, n, 2 * n]), ints([20, 20]), max_rows, expect=lq.LQ_DEVICE_ERR_BAD_SEGMENT)
    assert (out[:n] == 0).all() and out[n:].isfinite().all() and (out[n:] != 0).any()


def test_attention_skips_spans_that_do_not_fit():
    rng = np.random.default_rng(4)
    cache = make_cache(rng, [40, 40], 1, 64, 16)
    store(cache, bf16(rng, (80, 64)).cuda(), bf16(rng, (80, 64)).cuda(), None, ints([0, 40, 80]), ints([0, 0]))
    q = bf16(rng, (8, 64)).cuda()
    good = attend(cache, q, ints([0, 1]), ints([0, 4, 8]), ints([30, 36]), 4)
    for slots, starts, first, live in (([0, 7], [0, 4, 8], [30, 0], [0, 4]), ([-1, 1], [0, 4, 8], [0, 36], [4, 8]),
                                       ([0, 1], [0, 4, 8], [30, 37], [0, 4]), ([0, 1], [0, 4, 99], [30, 0], [0, 4]),
                                       ([0, 1], [-4, 4, 8], [0, 36], [4, 8])):
        out = attend(cache, q, ints(slots), ints(starts), ints(first), 4, expect=lq.LQ_DEVICE_ERR_BAD_SEGMENT)
        assert torch.equal(out[live[0]:live[1]], good[live[0]:live[1]])
        rest = torch.cat([out[:live[0]], out[live[1]:]])
        assert (rest == 7).all()


@pytest.mark.parametrize("max_rows", [1, 32, 1000])
def test_calls_whose_spans_are_all_empty(max_rows):
    """Rows that belong to nobody, slots without a position: nothing is written, nothing is reported."""
    rng = np.random.default_rng(9)
    cache = make_cache(rng, [0, 33, 0], 2, 64, 16)
    pages = cache.pages[0].clone()
    slots, starts, first = ints([0, 1, 2, 0]), ints([5] * 5), ints([0, 33, 0, 0])
    k, v = bf16(rng, (20, 128)).cuda(), bf16(rng, (20, 128)).cuda()
    store(cache, k, v, slots, starts, first)
    assert torch.equal(cache.pages[0], pages)
    kept, ws = (k.clone(), v.clone()), ws_for(cache)
    lq.lora_cache_load_rows(k, v, cache, 0, slots, starts, first, ws)
    assert lq.device_error_word(ws) == 0 and torch.equal(k, kept[0]) and torch.equal(v, kept[1])
    out = attend(cache, bf16(rng, (20, 256)).cuda(), slots, starts, first, max_rows)
    assert (out == 7).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("max_rows", [1, 32, 160])
def test_spans_with_more_rows_than_there_are_do_nothing(max_rows, d):
    """row_starts that go back and forth over the same rows: reported, no row is written, and the next call is as it should be."""
    rng = np.random.default_rng(8)
    cache = make_cache(rng, [400], 1, d, 16)
    store(cache, bf16(rng, (400, d)).cuda(), bf16(rng, (400, d)).cuda(), None, ints([0, 400]), ints([0]))
    q = bf16(rng, (400, d)).cuda()
    ws = lq.workspace(lq.lora_cache_attention_workspace_bytes(cache, 1, max_rows))
    n = 61
    starts = ints([0, 400] * 31)
    out = attend(cache, q, ints([0] * n), starts, ints([0] * n), max_rows, ws=ws, expect=1)
    assert (out == 7).all()
    ws[:1].zero_()
    good = attend(cache, q, None, ints([0, 400]), ints([0]), max_rows, ws=ws)
    assert torch.equal(good, attend(cache, q, None, ints([0, 400]), ints([0]), max_rows))


def test_pages_behind_four_gigabytes():
    """A pool of more than 2^32 bytes with the sequence in its last pages."""
    H, d, T, n_pages = 8, 128, 256, 9000
    assert n_pages * lq.lora_cache_page_bytes(H, d, T) > 2 ** 32 + 2 ** 28
    rng = np.random.default_rng(8)
    cache = lq.PagedCache.empty(1, H, d, T, n_pages, 2, 4)
    cache.table[1, :3] = ints([n_pages - 1, n_pages - 3, 8200])
    cache.refs[cache.table[1, :3].long()] = 1
    cache.lens[1] = 600
    k, v = bf16(rng, (600, H * d)), bf16(rng, (600, H * d))
    store(cache, k.cuda(), v.cuda(), ints([1]), ints([0, 600]), ints([0]))
    K, V = cm.Rows(H, d), cm.Rows(H, d)
    K.store(0, f64(k).reshape(-1, H, d))
    V.store(0, f64(v).reshape(-1, H, d))
    q = bf16(rng, (2, H * d)).cuda()
    out = attend(cache, q, ints([1]), ints([0, 2]), ints([598]), 2)
    want = cm.attention(f64(q).reshape(2, H, d), K.values, V.values, 598, d ** -0.5)
    assert_attention(f64(out).reshape(2, H, d), *want, 600)


# ---- pages -----------------------------------------------------------------------------------------------------------
def assert_pages(cache, model, marks=True):
    lens, refs, table = cache.lens.cpu().numpy(), cache.refs.cpu().numpy(), cache.table.cpu().numpy()
    assert np.array_equal(lens, model.lens) and np.array_equal(refs, model.refs)
    for s in range(len(lens)):
        held = -(-int(lens[s]) // model.T)
        assert np.array_equal(table[s, :held], model.table[s, :held]), s
    if marks:
        for layer, p in enumerate(cache.pages):
            got = p.view(torch.int32)
            live = np.flatnonzero(model.refs > 0)
            want = torch.from_numpy(model.content[live] + 10 ** 6 * layer).cuda().int()
            assert (got[torch.from_numpy(live).cuda()] == want[:, None]).all()


@pytest.mark.parametrize("seed,n_pages,n_slots,max_pages,T", [(0, 40, 12, 8, 16), (1, 300, 40, 20, 32), (2, 9000, 300, 64, 16),
                                                                  (3, 8000, 9000, 12, 16), (4, 20000, 9000, 16, 16)])
def test_page_calls_against_the_model(seed, n_pages, n_slots, max_pages, T):
    """A random program of reserve, fork, free and compact, with requests that cannot be served among them."""
    rng = np.random.default_rng(seed)
    cache = lq.PagedCache.empty(2, 1, 64, T, n_pages, n_slots, max_pages)
    model = cm.Pages(n_pages, n_slots, max_pages, T)
    for layer, p in enumerate(cache.pages):
        p.view(torch.int32).copy_((torch.arange(n_pages) + 10 ** 6 * layer).int()[:, None].expand(-1, p.shape[1] // 4))
    for step in range(30):
        ws = ws_for(cache, n_slots + 4)
        model.error = 0
        n = int(rng.integers(0, n_slots))
        some = rng.choice(n_slots, n, replace=False)
        if step % 5 == 3 and n:
            some = np.concatenate([some, some[:1], [-1, n_slots]])    # a slot again, and two that do not exist
        what = rng.choice(["reserve", "reserve", "fork", "free", "compact"])
        if what == "reserve":
            add = rng.integers(-1 if step % 4 == 0 else 0, rng.choice([2, T, max_pages * T // 2]) + 1, len(some))
            model.reserve(some, add)
            lq.lora_cache_reserve(cache, ints(some), ints(add), ws)
        elif what == "fork":
            src = rng.integers(0, n_slots, len(some))
            keep = None if step % 2 else [int(rng.integers(0, model.lens[s] + 1)) for s in src]
            model.fork(src, some, keep)
            lq.lora_cache_fork(cache, ints(src), ints(some), ws, None if keep is None else ints(keep))
        elif what == "free":
            some = some[: len(some) // 2 + 1]
            model.free(some)
            lq.lora_cache_free(cache, ints(some), ws)
        else:
            n_live = ints([0])
            want = model.compact()
            lq.lora_cache_compact(cache, n_live, ws)
            assert int(n_live.item()) == want
        torch.cuda.synchronize()
        assert lq.device_error_word(ws) == model.error, (step, what)
        assert_pages(cache, model)


def test_pages_run_out_and_come_back():
    cache = lq.PagedCache.empty(1, 1, 64, 16, 5, 4, 4)
    ws = ws_for(cache)
    lq.lora_cache_reserve(cache, ints([0, 1, 2, 3]), ints([33, 17, 1, 0]), ws)      # 3 + 2 pages; the rest finds none
    torch.cuda.synchronize()
    assert lq.device_error_word(ws) == lq.LQ_DEVICE_ERR_NO_PAGES
    with pytest.raises(lq.LqDeviceError, match="free pages"):
        lq.raise_on_device_error(ws)
    assert cache.lens.tolist() == [33, 17, 0, 0] and cache.refs.tolist() == [1] * 5 and cache.table[0].tolist() == [0, 1, 2, -1]
    ws.zero_()
    lq.lora_cache_fork(cache, ints([0]), ints([2]), ws)                             # needs a page for position 32
    torch.cuda.synchronize()
    assert lq.device_error_word(ws) == lq.LQ_DEVICE_ERR_NO_PAGES and cache.lens.tolist() == [33, 17, 0, 0]
    ws.zero_()
    lq.lora_cache_fork(cache, ints([0]), ints([2]), ws, keep=ints([32]))            # full pages only: nothing to copy
    lq.lora_cache_free(cache, ints([0]), ws)
    lq.lora_cache_reserve(cache, ints([3]), ints([16]), ws)
    torch.cuda.synchronize()
    assert lq.device_error_word(ws) == 0
    assert cache.refs.tolist() == [1] * 5 and cache.table[2, :2].tolist() == [0, 1] and cache.table[3, 0].item() == 2


@pytest.mark.parametrize("n_pages", [(1 << 21) + 5, 4000])
def test_requests_for_more_pages_than_32_bits_count(n_pages):
    """1024 requests, each of all pages: the ones before the first of them are served, and nothing else is touched."""
    n, T = 1024, 16
    dev = dict(dtype=torch.int32, device="cuda")
    cache = lq.PagedCache(1, 64, T, [], torch.full((n, n_pages), -1, **dev), torch.zeros(n, **dev), torch.zeros(n_pages, **dev))
    add = torch.full((n,), n_pages * T, **dev)
    add[0], add[1] = 3 * T, 0
    ws = ws_for(cache, n)
    lq.lora_cache_reserve(cache, torch.arange(n, **dev), add, ws)
    assert lq.device_error_word(ws) == lq.LQ_DEVICE_ERR_NO_PAGES
    assert cache.lens.sum().item() == cache.lens[0].item() == 3 * T
    assert cache.refs.sum().item() == cache.refs[:3].sum().item() == 3
    assert cache.table[0, :3].tolist() == [0, 1, 2]
    cache.table[0, :3] = -1
    assert cache.table.max().item() == -1


def test_page_calls_with_unusable_tables():
    """Lengths and page numbers that nothing of the library wrote: reported, nothing out of range touched."""
    cache = lq.PagedCache.empty(1, 1, 64, 16, 6, 4, 3)
    cache.lens.copy_(ints([49, -3, 20, 16]))                                        # beyond the row, negative, fine, fine
    cache.table.copy_(ints([[0, 1, 2], [0, 1, 2], [77, -2, 0], [5, -1, -1]]))
    cache.refs.copy_(ints([1, 1, 1, 0, 0, 1]))
    for call in (lambda ws: lq.lora_cache_reserve(cache, ints([0, 1]), ints([1, 1]), ws),
                 lambda ws: lq.lora_cache_fork(cache, ints([2]), ints([3]), ws),    # the target is not empty
                 lambda ws: lq.lora_cache_compact(cache, None, ws),
                 lambda ws: lq.lora_cache_free(cache, ints([0, 1, 2]), ws)):
        ws = ws_for(cache)
        call(ws)
        torch.cuda.synchronize()
        assert lq.device_error_word(ws) == lq.LQ_DEVICE_ERR_BAD_SEGMENT
    assert cache.refs.tolist() == [1, 1, 1, 1, 0, 0]                                # compact moved page 5 to 3; the frees hit nothing
    assert cache.table[3, 0].item() == 3 and cache.lens.tolist() == [0, 0, 0, 16]


# ---- together ----------------------------------------------------------------------------------------------------------
def _serve(cache, layers, steps, rng, compact_at=(), fork_at=()):
    """A serving loop: q, k, v by the grouped LoRA call, reserve, store, attention, per layer.  Returns the outputs of every step and the
    inputs that the check needs."""
    H, d = cache.n_kv_heads, cache.head_dim
    heads, w = 2 * H, 2 * H * d
    ws = ws_for(cache)
    log = []
    for i, (slots, n, done) in enumerate(steps):
        if i in fork_at:
            lq.lora_cache_fork(cache, ints([slots[0]]), ints([slots[-1]]), ws)
        if i in compact_at:
            lq.lora_cache_compact(cache, None, ws)
        T = sum(n)
        starts, first = ints(np.concatenate([[0], np.cumsum(n)])), ints(done)
        lq.lora_cache_reserve(cache, ints(slots), ints(n), ws)
        x = bf16(rng, (T, w)).cuda()
        seg = lq.SegmentTables.empty(T, 2)
        kind = lq.LQ_SEG_DECODE if max(n) == 1 else lq.LQ_SEG_PREFILL
        lq.lora_build_segments(ints(rng.integers(0, 2, T)), torch.full((T,), kind, dtype=torch.uint8, device="cuda"), layers[0][0].ranks, seg,
                               lq.workspace(lq.lora_build_workspace_bytes(T, 2)))
        for layer, ads in enumerate(layers):
            ys = [bf16(rng, (T, c)).cuda() for c in (w, H * d, H * d)]
            lq.lora_segmented_forward_group(x, ys, ads, seg, None, lq.workspace(lq.lora_forward_group_workspace_bytes(3, T, 8)),
                                            lq.LQ_VARIANT_AUTO)
            lq.lora_cache_store_rows(ys[1], ys[2], cache, layer, ints(slots), starts, first, ws)
            out = torch.zeros(T, w, dtype=torch.bfloat16, device="cuda")
            aws = lq.workspace(lq.lora_cache_attention_workspace_bytes(cache, heads, max(n)))
            lq.lora_cache_attention(ys[0], out, cache, layer, ints(slots), starts, first, max(n), aws)
            torch.cuda.synchronize()
            assert lq.device_error_word(aws) == 0
            log.append((layer, slots, n, done, *ys, out))
            x = out
    assert lq.device_error_word(ws) == 0
    return log


def test_a_serving_loop_with_lora_projections():
    """Prompts, decode steps, a forked request and a compaction between them, two layers: every attention output against the model, whose
    cached values follow the projections' rows."""
    rng = np.random.default_rng(11)
    H, d, T = 2, 64, 16
    cache = lq.PagedCache.empty(2, H, d, T, 40, 6, 10)
    w = 2 * H * d
    layers = [[lq.AdapterTable.from_tensors([bf16(rng, (8, w), 0.05).cuda() for _ in range(2)], [bf16(rng, (8, c), 0.05).cuda() for _ in range(2)],
                                            [1.0, 2.0]) for c in (w, H * d, H * d)] for _ in range(2)]
    steps = [([0, 1, 2], [50, 3, 17], [0, 0, 0]), ([2, 0, 1], [1, 1, 1], [17, 50, 3]), ([0, 1, 4], [1, 1, 1], [51, 4, 51]),
             ([4, 0], [1, 1], [52, 52]), ([1, 4, 0], [40, 1, 1], [5, 53, 53])]
    log = _serve(cache, layers, steps, rng, compact_at=(3,), fork_at=(2,))
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
            want = cm.attention(f64(q[at:at + m]).reshape(m, 2 * H, d), K.values, V.values, f, d ** -0.5)
            assert_attention(f64(out[at:at + m]).reshape(m, 2 * H, d), *want, f + m)
            at += m


def test_a_captured_step_replays():
    """Reserve, store and attention of a decode step captured into a graph; replays with eager work between them match eager steps."""
    rng = np.random.default_rng(12)
    H, d, T, S = 2, 128, 16, 3
    caches = []
    for _ in range(2):
        c = lq.PagedCache.empty(1, H, d, T, 30, S, 8)
        ws = ws_for(c)
        lq.lora_cache_reserve(c, ints(range(S)), ints([10, 20, 45]), ws)
        caches.append((c, ws))
    k0, v0 = bf16(rng, (75, H * d)).cuda(), bf16(rng, (75, H * d)).cuda()
    for c, ws in caches:
        lq.lora_cache_store_rows(k0, v0, c, 0, None, ints([0, 10, 30, 75]), ints([0, 0, 0]), ws)
    buf = [torch.zeros(S, w * d, dtype=torch.bfloat16, device="cuda") for w in (4 * H, H, H, 4 * H)]
    starts, one, slots = ints(range(S + 1)), ints([1] * S), ints(range(S))

    def step(c, ws, aws, first, q, k, v, out):
        lq.lora_cache_reserve(c, slots, one, ws)
        lq.lora_cache_store_rows(k, v, c, 0, slots, starts, first, ws)
        lq.lora_cache_attention(q, out, c, 0, slots, starts, first, 1, aws)
        first.add_(1)

    firsts = [ints([10, 20, 45]), ints([10, 20, 45])]
    aws = [lq.workspace(lq.lora_cache_attention_workspace_bytes(c, 4 * H, 1)) for c, _ in caches]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(*caches[0], aws[0], firsts[0], *buf)
    for i in range(6):
        inputs = [bf16(rng, tuple(b.shape), 1.0 + i).cuda() for b in buf[:3]]
        for b, x in zip(buf, inputs):
            b.copy_(x)
        graph.replay()
        out = torch.zeros_like(buf[3])
        step(*caches[1], aws[1], firsts[1], *inputs, out)
        torch.cuda.synchronize()
        assert torch.equal(buf[3], out) and out.isfinite().all(), i
        assert torch.equal(caches[0][0].lens, caches[1][0].lens) and torch.equal(caches[0][0].table, caches[1][0].table)
    for c, ws in caches:
        assert lq.device_error_word(ws) == 0


def test_captured_page_calls_and_split_sequences():
    """Every call in one graph, with sequences that several workgroups share; replays with eager work and a wait between them."""
    rng = np.random.default_rng(21)
    H, d, T, S = 2, 128, 16, 4
    lens = [5000, 2500, 30]
    twins = []
    k0, v0 = bf16(rng, (sum(lens), H * d)).cuda(), bf16(rng, (sum(lens), H * d)).cuda()
    for _ in range(2):
        c = lq.PagedCache.empty(2, H, d, T, 1000, S, 400)
        ws = ws_for(c)
        lq.lora_cache_reserve(c, ints([2, 0, 1]), ints([30, 5000, 2500]), ws)
        for layer in range(2):
            lq.lora_cache_store_rows(k0, v0, c, layer, None, ints(np.concatenate([[0], np.cumsum(lens)])), ints([0, 0, 0]), ws)
        aws = lq.workspace(lq.lora_cache_attention_workspace_bytes(c, 4 * H, 40))
        twins.append((c, ws, aws, ints(lens)))
    buf = [torch.zeros(42, w * d, dtype=torch.bfloat16, device="cuda") for w in (4 * H, H, H)] + [
        torch.zeros(42, 4 * H * d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    slots, add, starts, last, spare, cut = ints([0, 1, 2]), ints([1, 40, 1]), ints([0, 1, 41, 42]), ints([0]), ints([3]), ints([4099])

    def step(c, ws, aws, first, q, k, v, out, single):
        lq.lora_cache_reserve(c, slots, add, ws)
        lq.lora_cache_store_rows(k, v, c, 1, slots, starts, first, ws)
        lq.lora_cache_attention(q, out, c, 1, slots, starts, first, 40, aws)
        lq.lora_cache_fork(c, last, spare, ws, cut)
        lq.lora_cache_free(c, slots[1:2], ws)
        lq.lora_cache_compact(c, None, ws)
        lq.lora_cache_attention(q[:1], single, c, 1, spare, starts[:2], cut - 1, 1, aws)
        lq.lora_cache_free(c, spare, ws)
        lq.lora_cache_reserve(c, slots[1:2], first[1:2], ws)
        first.add_(add)
        first[1:2].sub_(40)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(*twins[0], *buf[:4], buf[4][:1])
    for i in range(4):
        inputs = [bf16(rng, tuple(b.shape), 1.0 + i).cuda() for b in buf[:3]]
        for b, x in zip(buf, inputs):
            b.copy_(x)
        graph.replay()
        out, single = torch.zeros_like(buf[3]), torch.zeros_like(buf[4])
        step(*twins[1], *inputs, out, single[:1])
        torch.cuda.synchronize()
        assert torch.equal(buf[3], out) and torch.equal(buf[4], single), i
        for name in ("lens", "table", "refs"):
            assert torch.equal(getattr(twins[0][0], name), getattr(twins[1][0], name)), (i, name)
    for c, ws, aws, _ in twins:
        assert lq.device_error_word(ws) == 0 and lq.device_error_word(aws) == 0


def test_calls_on_two_streams_and_rows_of_padding():
    """Two streams at once, each with its workspace; rows before, between and behind the spans stay as they were."""
    rng = np.random.default_rng(22)
    H, d, T = 2, 128, 32
    lens = [3000, 700, 40, 1500]
    cache = make_cache(rng, lens, H, d, T)
    starts = ints(np.concatenate([[0], np.cumsum(lens)]))
    rows = sum(lens)
    store(cache, bf16(rng, (rows, H * d)).cuda(), bf16(rng, (rows, H * d)).cuda(), None, starts, ints([0] * 4))
    calls = []
    for max_rows in (1, 5, 100):
        n = [max_rows, 1, min(max_rows, 40), 1]
        first = [t - m for t, m in zip(lens, n)]
        begin = 3 + np.concatenate([[0], np.cumsum(n)])
        q = bf16(rng, (int(begin[-1]) + 6, 2 * H * d)).cuda()
        calls.append((q, ints(begin), ints(first), max_rows, int(begin[-1])))
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [lq.workspace(lq.lora_cache_attention_workspace_bytes(cache, 2 * H, 100)) for _ in range(2)]
    want = [attend(cache, q, None, begin, first, m) for q, begin, first, m, _ in calls]
    torch.cuda.synchronize()
    got = [[torch.full_like(c[0], 7.0) for c in calls] for _ in range(8)]
    torch.cuda.synchronize()
    for r in range(8):
        with torch.cuda.stream(streams[r % 2]):
            for (q, begin, first, m, _), out in zip(calls, got[r]):
                lq.lora_cache_attention(q, out, cache, 0, None, begin, first, m, ws[r % 2])
    torch.cuda.synchronize()
    for outs in got:
        for out, w, (_, _, _, _, end) in zip(outs, want, calls):
            assert torch.equal(out, w) and (out[:3] == 7).all() and (out[end:] == 7).all() and out[3:end].isfinite().all()
    k = torch.full((rows + 9, H * d), 7.0, dtype=torch.bfloat16, device="cuda")
    v, wr = k.clone(), ws_for(cache)
    lq.lora_cache_load_rows(k, v, cache, 0, None, starts + 4, ints([0] * 4), wr)
    assert lq.device_error_word(wr) == 0
    for x in (k, v):
        assert (x[:4] == 7).all() and (x[rows + 4:] == 7).all() and x[4:rows + 4].isfinite().all()
