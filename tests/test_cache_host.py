"""The paged cache without a GPU: sizes, refusals (before anything is launched), and the plain model that the GPU tests use."""
import ctypes
import os

import numpy as np
import pytest

import cache_model as cm


@pytest.fixture(scope="module")
def lq():
    from paper_2511_00101_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2511_00101_amd import build
        build.build_library()
    return binding


def test_page_bytes(lq):
    assert lq.lora_cache_page_bytes(8, 128, 64) == 8 * 2 * 64 * 128 + 8 * 4 * 2 + 64     # padded to 128 bytes
    assert lq.lora_cache_page_bytes(1, 64, 16) == 2 * 16 * 64 + 128         # two exponent bytes, padded
    for bad in ((0, 128, 64), (257, 128, 64), (8, 96, 64), (8, 128, 8), (8, 128, 48), (8, 128, 512), (-1, 64, 16)):
        assert lq.lora_cache_page_bytes(*bad) == 0


ONE, TWO, WS = 0x10000, 0x20000, 0x40000        # never dereferenced: nothing is launched


def _struct(lq, **kw):
    v = dict(n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=10, n_slots=4, max_pages=5, table=ONE, lens=ONE, refs=ONE)
    v.update(kw)
    return lq._CacheStruct(*v.values())


BAD_CACHES = [(dict(table=None), 1), (dict(lens=None), 1), (dict(refs=None), 1), (dict(n_kv_heads=0), 1), (dict(n_pages=0), 1),
              (dict(n_slots=-1), 1), (dict(max_pages=0), 1), (dict(head_dim=80), 2), (dict(page_tokens=24), 2),
              (dict(n_kv_heads=300), 2), (dict(max_pages=1 << 27), 2), (dict(n_pages=(1 << 22) + 1), 2),
              (dict(n_slots=(1 << 22) + 1), 2)]


def _calls(lq, c, ws=WS, ws_bytes=1 << 30, n=0):
    """Every call of the cache that takes a workspace, with n requests / spans (0: returns before a launch)."""
    L, r = lq.lib(), ctypes.addressof(c) if c is not None else None
    return {
        "reserve": L.lora_cache_reserve(r, ONE, ONE, n, ws, ws_bytes, None),
        "fork": L.lora_cache_fork(r, ONE, ONE, None, n, ONE, 1, ws, ws_bytes, None),
        "free": L.lora_cache_free(r, ONE, n, ws, ws_bytes, None),
        "store": L.lora_cache_store_rows(ONE, 128, TWO, 128, 0, r, ONE, ONE, ONE, ONE, n, ws, ws_bytes, None),
        "load": L.lora_cache_load_rows(ONE, 128, TWO, 128, 0, r, ONE, ONE, ONE, ONE, n, ws, ws_bytes, None),
        "attention": L.lora_cache_attention(ONE, 128, TWO, 128, 0, 2, 1.0, r, ONE, ONE, ONE, ONE, n, 1, ws, ws_bytes, None),
    }


@pytest.mark.parametrize("fields,status", BAD_CACHES)
def test_cache_argument_is_checked(lq, fields, status):
    assert set(_calls(lq, _struct(lq, **fields)).values()) == {status}
    c = _struct(lq, **fields)
    assert lq.lib().lora_cache_compact(ctypes.addressof(c), ONE, 1, None, WS, 1 << 30, None) == status


def test_no_cache_small_workspace_and_empty_calls(lq):
    assert set(_calls(lq, None).values()) == {lq.LQ_ERR_INVALID_ARG}
    c = _struct(lq)
    assert set(_calls(lq, c).values()) == {lq.LQ_OK}
    assert set(_calls(lq, c, ws=None).values()) == {lq.LQ_ERR_WORKSPACE}
    assert set(_calls(lq, c, ws=WS + 4).values()) == {lq.LQ_ERR_WORKSPACE}
    assert set(_calls(lq, c, ws_bytes=4095).values()) == {lq.LQ_ERR_WORKSPACE}
    assert set(_calls(lq, c, n=-1).values()) == {lq.LQ_ERR_INVALID_ARG}
    assert lq.lib().lora_cache_compact(ctypes.addressof(c), ONE, 1, None, WS, 4095, None) == lq.LQ_ERR_WORKSPACE
    need = lq.lib().lora_cache_workspace_bytes(ctypes.addressof(c), 100)
    assert 4096 < need < 8192
    assert lq.lib().lora_cache_workspace_bytes(None, 1) == 0
    many = _calls(lq, c, n=(1 << 22) + 1)           # more than a launch could take
    assert {many[k] for k in ("reserve", "fork", "free", "attention")} == {lq.LQ_ERR_UNSUPPORTED}
    assert lq.lib().lora_cache_attention_workspace_bytes(ctypes.addressof(c), 0, 1) == 0
    assert lq.lib().lora_cache_attention_workspace_bytes(ctypes.addressof(c), 2, 1) >= 4096


def test_row_calls_refuse_before_launching(lq):
    c = _struct(lq)
    r, L = ctypes.addressof(c), lq.lib()

    def rows(k=ONE, ldk=128, v=TWO, ldv=128, n_rows=4, pages=ONE, starts=ONE, first=ONE, n=2, ws=WS, ws_bytes=1 << 30):
        got = {f(k, ldk, v, ldv, n_rows, r, pages, ONE, starts, first, n, ws, ws_bytes, None) for f in (L.lora_cache_store_rows, L.lora_cache_load_rows)}
        assert len(got) == 1
        return got.pop()

    for bad in (dict(k=None), dict(v=None), dict(k=TWO), dict(ldk=120), dict(ldv=64), dict(n_rows=-1), dict(pages=None), dict(starts=None),
                dict(first=None)):
        assert rows(**bad) == lq.LQ_ERR_INVALID_ARG, bad
    for bad in (dict(ldk=132), dict(ldv=129), dict(k=ONE + 8), dict(pages=ONE + 4),
                dict(n_rows=1 << 28), dict(n=1 << 24)):
        assert rows(**bad) == lq.LQ_ERR_UNSUPPORTED, bad
    assert rows(ws_bytes=100) == lq.LQ_ERR_WORKSPACE
    assert rows(n_rows=0, k=None, v=None) == lq.LQ_OK

    def attend(q=ONE, ldq=256, out=TWO, ldo=256, n_rows=4, heads=4, scale=1.0, pages=ONE, n=2, max_rows=4, ws=WS, ws_bytes=1 << 30):
        return L.lora_cache_attention(q, ldq, out, ldo, n_rows, heads, scale, r, pages, ONE, ONE, ONE, n, max_rows, ws, ws_bytes, None)

    for bad in (dict(q=None), dict(out=None), dict(out=ONE), dict(ldq=248), dict(ldo=128), dict(heads=3), dict(heads=0), dict(max_rows=0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(pages=None), dict(n_rows=-1)):
        assert attend(**bad) == lq.LQ_ERR_INVALID_ARG, bad
    for bad in (dict(ldq=260), dict(out=TWO + 2), dict(heads=258, ldq=1 << 16, ldo=1 << 16), dict(n=4097),
                dict(n_rows=(1 << 22) + 1)):
        assert attend(**bad) == lq.LQ_ERR_UNSUPPORTED, bad
    assert attend(ws_bytes=64) == lq.LQ_ERR_WORKSPACE
    assert attend(n_rows=0, q=None, out=None) == lq.LQ_OK


def test_model_rounds_to_the_nearest_code():
    codes = np.arange(256)
    values = cm.e4m3_value(codes)
    fine = np.sort(values[np.isfinite(values)])
    assert fine.max() == 448 and np.isnan(values[[127, 255]]).all() and np.isfinite(values).sum() == 254
    assert np.array_equal(cm.e4m3_round(fine), fine)
    x = np.random.default_rng(0).uniform(-500, 500, 4000) * np.random.default_rng(1).choice([1, 1e-2, 1e-4], 4000)
    best = np.abs(np.clip(x, -448, 448)[:, None] - fine[None]).min(1)
    assert np.array_equal(np.abs(np.clip(x, -448, 448) - cm.e4m3_round(x)), best)
    mid = (values[0x40:0x48] + values[0x41:0x49]) / 2                          # ties: to the even code
    assert np.array_equal(cm.e4m3_round(mid), values[[0x40, 0x42, 0x42, 0x44, 0x44, 0x46, 0x46, 0x48]])


def test_model_exponent_is_the_least_that_fits():
    rng = np.random.default_rng(2)
    for x in list(rng.uniform(1e-20, 1e20, 200)) + [448.0, 448.0000001, 1.75, 1.7500001, 2.0 ** -92, 1e-38, 3e38]:
        e = cm.block_exponent(np.array([x, np.nan, np.inf]))
        assert -100 <= e <= 119
        assert e == 119 or x <= 448 * 2.0 ** e
        assert e == -100 or x > 448 * 2.0 ** (e - 1)


def test_model_pages_by_hand():
    p = cm.Pages(6, 4, 3, 16)
    p.reserve([2, 0, 2], [20, 16, 5])                          # the second mention of slot 2 is skipped
    assert p.error == cm.BAD and p.table[2, :2].tolist() == [0, 1] and p.table[0, 0] == 2 and p.lens.tolist() == [16, 0, 20, 0]
    p.fork([2], [1])                                           # shares page 0, copies page 1 into 3
    assert p.table[1, :2].tolist() == [0, 3] and p.refs.tolist() == [2, 1, 1, 1, 0, 0] and p.content[3] == 1
    p.free([2])
    assert p.refs.tolist() == [1, 0, 1, 1, 0, 0]
    assert p.compact() == 3 and p.refs.tolist() == [1, 1, 1, 0, 0, 0] and p.table[1, :2].tolist() == [0, 1] and p.content[1] == 1
    p.error = 0
    p.reserve([3, 0], [48, 48])                                # 3 pages, then too many positions for slot 0's row
    assert p.error == cm.BAD and p.lens[3] == 48
    p.free([1, 1])
    p.reserve([1, 2], [40, 10])                                # 3 pages of the 2 that are free: neither is served
    assert p.error == cm.BAD | cm.NO_PAGES and p.lens[1] == p.lens[2] == 0
