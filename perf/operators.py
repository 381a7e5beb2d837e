"""The work that a serving step has the paged key/value cache do, as measurable cases.

The cache holds keys and values in 8 bits (e4m3 codes, one power-of-two scale for every block of 16 positions and head) in pages of
one layer each; a page table per slot, the slots' lengths and the pages' reference counts say what lies where.  Every case is a plain
dict; `op` names the call of its pass:

  attend   attention of the rows of `seqs` requests over their cached positions: single tokens (rows = 1), drafts, prompts
  store    the rows of a step quantised into the pages, and the touched blocks read back as bf16 rows
  reserve  pages for the tokens that a step adds
  fork     new slots that share their parents' full pages and get a copy of the last, partly filled one, in every layer's pool
  free     finished requests, half of those in the table, give their pages back
  compact  live pages move to the lowest numbers, in every layer's pool, and the tables follow

and the rest of it the sizes.  `rows` and `past` are the largest number of a request's new rows and of its earlier positions; with
`ragged` the requests' numbers are spread below them.  Where `own` is false a pass computes the same by elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16            # positions that share a scale
E_MIN, E_MAX = -100, 119

_BASE = dict(op="attend", seqs=1, rows=1, past=0, ragged=True, heads=32, kv_heads=8, head_dim=128, page_tokens=64, slots=0, pages=0,
             layers=1, share=0.0)


def _case(**kw):
    return dict(_BASE, **kw)


def listed():
    return [
        # the first tokens of a few short chats on a small model: launch and round trips only
        _case(name="attend_short", seqs=4, rows=1, past=60, heads=8, kv_heads=2, head_dim=64, page_tokens=16),
        # a busy server's decode step: 256 requests of up to 4096 positions, one layer of the 8B shapes
        _case(name="attend_decode_256", seqs=256, past=4096),
        # few requests over long documents: a long axis to split, no grouped heads
        _case(name="attend_long_3", seqs=3, past=32768, heads=32, kv_heads=32, page_tokens=128),
        # drafted tokens of speculative decoding checked in one step
        _case(name="attend_drafts", seqs=48, rows=5, past=3000, heads=32, kv_heads=8, head_dim=64, page_tokens=32),
        # chunked prompts of odd lengths behind cached prefixes
        _case(name="attend_chunks", seqs=9, rows=777, past=2500, page_tokens=16),
        # two long prompts from their first token
        _case(name="attend_prompts_8k", seqs=2, rows=8192, past=0, ragged=False),
        # the decode step's new keys and values, one row a request
        _case(name="store_decode_256", op="store", seqs=256, past=4096),
        # prompts entering the cache, blocks begun by an earlier chunk among them
        _case(name="store_prompts", op="store", seqs=12, rows=2048, past=100, page_tokens=32),
        # pages for a decode step of a server with many open requests
        _case(name="reserve_step", op="reserve", seqs=512, rows=40, past=2000, slots=1024, pages=65536, page_tokens=16),
        # parallel samples: children of running requests, eight layers
        _case(name="fork_samples", op="fork", seqs=64, past=1500, slots=256, pages=4096, layers=8, page_tokens=64),
        # finished requests leave
        _case(name="free_finished", op="free", seqs=400, past=3000, slots=1024, pages=65536, page_tokens=16, share=0.2),
        # a pool with holes put together, eight layers
        _case(name="compact_pool", op="compact", seqs=48, past=1200, slots=128, pages=1500, layers=8, page_tokens=32, share=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend"] * 6 + ["store"] * 2 + ["reserve", "fork", "free", "compact"])
    c = _case(op=op, head_dim=rng.choice([64, 128, 128]), page_tokens=rng.choice([16, 32, 64, 128, 256]), ragged=rng.random() < 0.8)
    c["kv_heads"] = rng.choice([1, 2, 4, 5, 8, 8, 16, 32])
    c["heads"] = c["kv_heads"] * rng.choice([g for g in (1, 2, 3, 4, 6, 8, 16) if g * c["kv_heads"] <= 64])
    if op in ("attend", "store"):
        kind = rng.choice(["decode", "decode", "draft", "prompt"])
        c["seqs"] = _log(rng, 1, 300 if kind == "decode" else 64 if kind == "draft" else 12)
        c["rows"] = 1 if kind == "decode" else rng.randint(2, 16) if kind == "draft" else _log(rng, 17, 6000)
        c["past"] = rng.choice([0, _log(rng, 1, 30000), _log(rng, 1, 4000)])
    else:
        c["page_tokens"] = rng.choice([16, 32, 64, 128])
        c["seqs"], c["past"] = _log(rng, 2, 512 if op in ("reserve", "free") else 64), _log(rng, 1, 3000)
        c["rows"] = _log(rng, 1, 500)
        c["slots"] = c["seqs"] * (2 if op == "fork" else 1) + _log(rng, 8, 500)
        c["layers"] = rng.randint(1, 12) if op in ("fork", "compact") else 1
        c["share"] = rng.choice([0.0, 0.2])
        c["pages"] = int(_pages_of(c) * rng.uniform(1.02, 3.0)) + c["seqs"] + 16
    while not _within(c):
        for key in ("past", "rows", "seqs"):
            c[key] = max(2 if key == "seqs" and op not in ("attend", "store") else 1, c[key] * 3 // 4)
        if op not in ("attend", "store"):
            c["pages"] = max(_pages_of(c) + c["seqs"] + 16, c["pages"] * 3 // 4)
    return c


def _within(c):
    """No more than the largest listed case, and a plain form whose scores fit the card."""
    w = work(c)
    if w["bytes"] > 7e8 or w["flops"] > 1e12:
        return False
    if c["op"] in ("fork", "compact", "reserve", "free"):
        return c["layers"] * c["pages"] * _page_bytes(c) < 1.5e9 if c["op"] in ("fork", "compact") else True
    length = c["past"] + c["rows"]
    scores = c["seqs"] * c["heads"] * c["rows"] * length * 4.0
    return scores < 1.8e10 and c["seqs"] * length * c["kv_heads"] * c["head_dim"] * 4.0 < 6e9


# ---- sizes of a case (the same for every seed) -------------------------------------------------------------------------
def _spread(n, most, least, ragged, step=0.618033988749895):
    """n whole numbers in [least, most], spread evenly over the logarithm of the range."""
    if not ragged:
        return [most] * n
    lo = max(1, most // 16)
    return [max(least, int(round(lo * (most / lo) ** ((i + 1) * step % 1.0)))) if most else least for i in range(n)]


def _sizes(c):
    rows = _spread(c["seqs"], c["rows"], 1, c["ragged"] and c["rows"] > 16)
    rows[0] = c["rows"]
    past = _spread(c["seqs"], c["past"], 0, c["ragged"], 0.7548776662466927)
    return rows, past


def _page_bytes(c):
    H, T, d = c["kv_heads"], c["page_tokens"], c["head_dim"]
    return -(-(H * 2 * T * d + H * (T // BLOCK) * 2) // 128) * 128


def _pages_of(c):
    return sum(-(-p // c["page_tokens"]) for p in _sizes(c)[1])


def work(case):
    c = dict(_BASE, **case)
    rows, past = _sizes(c)
    d, H = c["head_dim"], c["kv_heads"]
    if c["op"] == "attend":
        pairs = sum(r * p + r * (r + 1) // 2 for r, p in zip(rows, past))
        cached = sum(r + p for r, p in zip(rows, past))
        return {"bytes": cached * H * (2 * d + 2 / BLOCK) + 4 * sum(rows) * c["heads"] * d, "flops": 4 * d * c["heads"] * pairs}
    if c["op"] == "store":
        read = sum(p % BLOCK + r for r, p in zip(rows, past))
        return {"bytes": H * 2 * d * (sum(rows) * 3 + read * 3), "flops": 0}
    entries = 4 * (_pages_of(c) + c["seqs"])
    if c["op"] == "reserve":
        T = c["page_tokens"]
        new = sum(-(-(p + r) // T) - -(-p // T) for r, p in zip(_sizes(dict(c, ragged=True))[0], past))
        return {"bytes": 4 * c["pages"] + 4 * c["seqs"] * 4 + 8 * new, "flops": 0}
    if c["op"] == "free":
        return {"bytes": 3 * entries // 2, "flops": 0}
    if c["op"] == "fork":
        copies = sum(p % c["page_tokens"] != 0 for p in past)
        return {"bytes": 4 * c["pages"] + 3 * entries + 2 * copies * c["layers"] * _page_bytes(c), "flops": 0}
    live = _pages_of(c)
    moved = live * (1 - live / c["pages"])
    return {"bytes": 4 * c["pages"] + 2 * entries + 2 * moved * c["layers"] * _page_bytes(c), "flops": 0}


# ---- what the program has in hand --------------------------------------------------------------------------------------
def _ints(v, dev="cuda"):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def prepare(case, seed):
    c = dict(_BASE, **case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    rows, past = _sizes(c)
    T, H, d, S = c["page_tokens"], c["kv_heads"], c["head_dim"], c["seqs"]
    n = _page_bytes(c)
    if c["op"] in ("attend", "store"):
        total = [r + p for r, p in zip(rows, past)]
        used = [-(-t // T) for t in total]
        n_pages, n_slots, width = sum(used) + 3, S + 2, max(used) + 1
        slots = rng.permutation(n_slots)[:S]
        order = rng.permutation(n_pages)
        table = np.full((n_slots, width), -1, np.int32)
        lens = np.zeros(n_slots, np.int32)
        at = 0
        for s, k, t in zip(slots, used, total):
            table[s, :k] = order[at:at + k]
            lens[s] = t
            at += k
        refs = np.zeros(n_pages, np.int32)
        refs[order[:at]] = 1
        pages = torch.empty(n_pages, n, dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 28) // n)
        for i in range(0, n_pages, step):
            part = torch.randn(min(step, n_pages - i), n, device="cuda", generator=gen)
            pages[i:i + step] = (part * 100).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        n_scales = n - H * 2 * T * d
        pages[:, H * 2 * T * d:] = torch.randint(118, 122, (n_pages, n_scales), device="cuda", generator=gen, dtype=torch.uint8)
        starts = np.concatenate([[0], np.cumsum(rows)])
        st = dict(c=c, pages=[pages], table=_ints(table), lens=_ints(lens), refs=_ints(refs), slots=_ints(slots), row_starts=_ints(starts),
                  first=_ints(past), max_rows=max(rows), n_rows=int(starts[-1]))
        if c["op"] == "attend":
            st["q"] = torch.randn(st["n_rows"], c["heads"] * d, device="cuda", generator=gen).to(torch.bfloat16)
            st["out"] = torch.zeros_like(st["q"])
            return st
        # keys have channels that are larger than the others, values do not
        gain = torch.exp(0.7 * torch.randn(1, H * d, device="cuda", generator=gen))
        st["k"] = (torch.randn(st["n_rows"], H * d, device="cuda", generator=gen) * gain).to(torch.bfloat16)
        st["v"] = torch.randn(st["n_rows"], H * d, device="cuda", generator=gen).to(torch.bfloat16)
        # the blocks that the rows touch, and the rows of those blocks as they are read back
        begin = [p // BLOCK * BLOCK for p in past]
        back = np.concatenate([[0], np.cumsum([t - b for t, b in zip(total, begin)])])
        st["back_starts"], st["back_first"] = _ints(back), _ints(begin)
        st["block_seq"] = torch.tensor([s for s in range(S) for _ in range(begin[s], total[s], BLOCK)], device="cuda")
        st["block_at"] = torch.tensor([b for s in range(S) for b in range(begin[s], total[s], BLOCK)], device="cuda")
        st["k_back"] = torch.zeros(int(back[-1]), H * d, dtype=torch.bfloat16, device="cuda")
        st["v_back"] = torch.zeros_like(st["k_back"])
        return st
    # page management: some slots share the first part of their pages with the slot before them
    n_slots, n_pages = c["slots"], c["pages"]
    slots = rng.permutation(n_slots)
    order = rng.permutation(n_pages)
    width = -(-(c["past"] + c["rows"]) // T) + 1
    table = np.full((n_slots, width), -1, np.int32)
    lens = np.zeros(n_slots, np.int32)
    refs = np.zeros(n_pages, np.int32)
    at = 0
    for i in range(S):
        k = -(-past[i] // T)
        both = min(past[i] // T, past[i - 1] // T) if i and rng.random() < c["share"] else 0
        table[slots[i], :both] = table[slots[i - 1], :both]
        table[slots[i], both:k] = order[at:at + k - both]
        at += k - both
        refs[table[slots[i], :k]] += 1
        lens[slots[i]] = past[i]
    kept = torch.cat([_ints(table).view(-1), _ints(lens), _ints(refs)])
    state = kept.clone()
    t, le, rf = state.split([n_slots * width, n_slots, n_pages])
    st = dict(c=c, kept=kept, state=state, table=t.view(n_slots, width), lens=le, refs=rf, slots=_ints(slots[:S]), most=-(-c["rows"] // T) + 1)
    st["pages"] = []
    if c["op"] == "free":
        st["slots"] = _ints(slots[:(S + 1) // 2])
    if c["op"] in ("fork", "compact"):
        pool = torch.empty(c["layers"], n_pages, n // 4, dtype=torch.int32, device="cuda")
        pool.random_(generator=gen)
        st["pool"], st["pages"] = pool, [p.view(torch.uint8) for p in pool]
    if c["op"] == "reserve":
        st["add"] = _ints(_sizes(dict(c, ragged=True))[0])
    if c["op"] == "fork":
        st["dst"] = _ints(slots[S:2 * S])
    if c["op"] == "compact":
        st["n_live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return st


# ---- the calls of the framework ------------------------------------------------------------------------------------------
def _library(st):
    """The handle and the workspace that a program makes once and keeps."""
    if "cache" not in st:
        from paper_2511_00101_amd import binding as lq
        c = st["c"]
        st["lq"] = lq
        st["cache"] = lq.PagedCache(c["kv_heads"], c["head_dim"], c["page_tokens"], st["pages"], st["table"], st["lens"], st["refs"])
        if c["op"] == "attend":
            size = lq.lora_cache_attention_workspace_bytes(st["cache"], c["heads"], st["max_rows"])
        else:
            size = lq.lora_cache_workspace_bytes(st["cache"], c["seqs"])
        st["workspace"] = lq.workspace(size)
    return st["lq"], st["cache"], st["workspace"]


def _own_run(st):
    lq, cache, ws = _library(st)
    op = st["c"]["op"]
    if op == "attend":
        lq.lora_cache_attention(st["q"], st["out"], cache, 0, st["slots"], st["row_starts"], st["first"], st["max_rows"], ws)
        return st["out"]
    if op == "store":
        lq.lora_cache_store_rows(st["k"], st["v"], cache, 0, st["slots"], st["row_starts"], st["first"], ws)
        lq.lora_cache_load_rows(st["k_back"], st["v_back"], cache, 0, st["slots"], st["back_starts"], st["back_first"], ws)
        return {"k": st["k_back"], "v": st["v_back"]}
    st["state"].copy_(st["kept"])       # the tables as they are before the step
    if op == "reserve":
        lq.lora_cache_reserve(cache, st["slots"], st["add"], ws)
    elif op == "free":
        lq.lora_cache_free(cache, st["slots"], ws)
    elif op == "fork":
        lq.lora_cache_fork(cache, st["slots"], st["dst"], ws)
    else:
        lq.lora_cache_compact(cache, st["n_live"], ws)
    return _tables(st)


def _tables(st):
    out = {"table": st["table"], "lens": st["lens"], "refs": st["refs"]}
    if "pool" in st:
        out["pool"] = st["pool"]
    if "n_live" in st:
        out["n_live"] = st["n_live"]
    return out


# ---- the plain forms -------------------------------------------------------------------------------------------------------
def _views(pages, c):
    """Pages as K codes [page, head, token, d], V codes [page, head, token / 4, d, token % 4] and exponent bytes [page, head, block, 2]."""
    H, T, d = c["kv_heads"], c["page_tokens"], c["head_dim"]
    codes = pages[..., :H * 2 * T * d].unflatten(-1, (H, 2, T * d))
    scales = pages[..., H * 2 * T * d:H * 2 * T * d + H * (T // BLOCK) * 2].unflatten(-1, (H, T // BLOCK, 2))
    return codes[..., 0, :].unflatten(-1, (T, d)), codes[..., 1, :].unflatten(-1, (T // 4, d, 4)), scales


def _values(codes, scales):
    """fp32 values of codes [..., token, d] with the exponent bytes [..., block] of their blocks of 16 tokens."""
    e = scales.to(torch.int32) - 127
    x = codes.contiguous().view(torch.float8_e4m3fn).float()
    return torch.ldexp(x.unflatten(-2, (-1, BLOCK)), e[..., None, None]).flatten(-3, -2)


def _gathered(st, n_pos):
    """K and V of the batch's sequences, [seq, head, position, d] in fp32, up to n_pos positions."""
    c = st["c"]
    P = -(-n_pos // c["page_tokens"])
    pg = st["table"][st["slots"].long(), :P].clamp(min=0).long()
    K, V, sc = _views(st["pages"][0][pg], c)                      # [seq, page, head, ...]
    V = V.transpose(-1, -2).flatten(-3, -2)                       # [seq, page, head, token, d]
    put = lambda codes, s: _values(codes, s).transpose(1, 2).flatten(2, 3)  # noqa: E731
    return put(K, sc[..., 0]), put(V, sc[..., 1])


def _attend(st):
    c = st["c"]
    d, H, G = c["head_dim"], c["kv_heads"], c["heads"] // c["kv_heads"]
    rows, past = _sizes(c)
    L, R = max(r + p for r, p in zip(rows, past)), st["max_rows"]
    K, V = _gathered(st, L)
    starts, first = st["row_starts"].long(), st["first"].long()
    i = torch.arange(R, device="cuda")
    at = (starts[:-1, None] + i).clamp(max=st["n_rows"] - 1)     # [seq, row]
    q = st["q"].float()[at].view(-1, R, H, G, d).permute(0, 2, 3, 1, 4).reshape(-1, H, G * R, d)
    s = torch.matmul(q, K.transpose(-1, -2)).mul_(d ** -0.5).view(-1, H, G, R, K.shape[2])
    seen = torch.arange(K.shape[2], device="cuda") <= (first[:, None] + i)[..., None]       # [seq, row, position]
    s.masked_fill_(~seen[:, None, None], float("-inf"))
    s.sub_(s.amax(-1, keepdim=True)).exp_()
    s.div_(s.sum(-1, keepdim=True))
    V = torch.where((torch.arange(V.shape[2], device="cuda") < st["lens"][st["slots"].long()][:, None])[:, None, :, None], V, 0.0)
    o = torch.matmul(s.view(-1, H, G * R, K.shape[2]), V).view(-1, H, G, R, d).permute(0, 3, 1, 2, 4).reshape(-1, R, H * G * d)
    real = i < (starts[1:] - starts[:-1])[:, None]
    st["out"].copy_(o[real].to(torch.bfloat16))
    return st["out"]


def _quantised(x, new, kept, old_codes, old_e):
    """Codes and exponents of blocks [block, head, token, d]: `new` tokens from x, `kept` ones from their codes."""
    amax = torch.where(new & x.isfinite(), x.abs(), 0.0).amax((-1, -2))
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, torch.where(m <= 0.875, e - 9, e - 8), E_MIN).clamp(E_MIN, E_MAX)
    e = torch.where(kept.any(-1).any(-1), torch.maximum(e, old_e), e)
    old = torch.ldexp(old_codes.contiguous().view(torch.float8_e4m3fn).float(), old_e[..., None, None])
    x = torch.where(new, x, torch.where(kept, old, 0.0))
    code = torch.ldexp(x, -e[..., None, None])
    code = torch.where(code.isfinite(), code.clamp(-448, 448), float("nan")).to(torch.float8_e4m3fn)
    return code.view(torch.uint8), e, torch.ldexp(code.float(), e[..., None, None])


def _store(st):
    c = st["c"]
    T, H, d = c["page_tokens"], c["kv_heads"], c["head_dim"]
    seq, at = st["block_seq"], st["block_at"]
    slot = st["slots"].long()[seq]
    pg, blk = st["table"][slot, at // T].long(), at % T // BLOCK
    pos = at[:, None] + torch.arange(BLOCK, device="cuda")                    # [block, token]
    begin = st["first"].long()[seq][:, None]
    n = (st["row_starts"][1:] - st["row_starts"][:-1]).long()[seq][:, None]
    new, kept = (pos >= begin) & (pos < begin + n), pos < begin
    row = (st["row_starts"].long()[seq][:, None] + pos - begin).clamp(0, st["n_rows"] - 1)
    K, V, sc = _views(st["pages"][0], c)
    Kb, Vb = K.unflatten(2, (T // BLOCK, BLOCK)), V.unflatten(2, (T // BLOCK, BLOCK // 4))
    back = (st["back_starts"].long()[seq][:, None] + pos - st["back_first"].long()[seq][:, None])[new | kept]
    mask = lambda m: m[:, None, :, None]                                       # noqa: E731
    rows = lambda x: x.float()[row].view(-1, BLOCK, H, d).transpose(1, 2)      # noqa: E731
    kc, ke, kv = _quantised(rows(st["k"]), mask(new), mask(kept), Kb[pg, :, blk], sc[pg, :, blk, 0].int() - 127)
    Kb[pg, :, blk] = torch.where(mask(new | kept), kc, Kb[pg, :, blk])
    vo = Vb[pg, :, blk].transpose(-1, -2).flatten(-3, -2)
    vc, ve, vv = _quantised(rows(st["v"]), mask(new), mask(kept), vo, sc[pg, :, blk, 1].int() - 127)
    Vb[pg, :, blk] = torch.where(mask(new | kept), vc, vo).unflatten(-2, (BLOCK // 4, 4)).transpose(-1, -2)
    sc[pg, :, blk] = (torch.stack([ke, ve], -1) + 127).to(torch.uint8)
    for_rows = lambda x: x.transpose(1, 2).flatten(-2)[new | kept].to(torch.bfloat16)  # noqa: E731
    st["k_back"][back], st["v_back"][back] = for_rows(kv), for_rows(vv)
    return {"k": st["k_back"], "v": st["v_back"]}


def _lowest_free(refs):
    """Numbers of the free pages in order, -1 behind the last one, and how many there are."""
    free = refs == 0
    rank = torch.cumsum(free, 0) - 1
    found = torch.full((refs.numel() + 1,), -1, dtype=torch.int64, device="cuda")
    found[torch.where(free, rank, refs.numel())] = torch.where(free, torch.arange(refs.numel(), device="cuda"), -1)
    return found[:-1], free.sum()


def _reserve(st):
    T = st["c"]["page_tokens"]
    table, lens, refs, slot = st["table"], st["lens"], st["refs"], st["slots"].long()
    have = (lens[slot] + T - 1) // T
    need = (lens[slot] + st["add"] + T - 1) // T - have
    upto = torch.cumsum(need, 0)
    found, n_free = _lowest_free(refs)
    served = upto <= n_free
    j = torch.arange(st["most"], device="cuda")
    take = (j < need[:, None]) & served[:, None]
    page = found[((upto - need)[:, None] + j).clamp(max=refs.numel() - 1)]
    col = (have[:, None] + j).clamp(max=table.shape[1] - 1).long()
    s, k = slot[:, None].expand_as(col)[take], col[take]
    table[s, k] = page[take].int()
    refs[page[take]] = 1
    lens[slot] += torch.where(served, st["add"], 0)
    return _tables(st)


def _free(st):
    T = st["c"]["page_tokens"]
    table, lens, refs, slot = st["table"], st["lens"], st["refs"], st["slots"].long()
    held = torch.arange(table.shape[1], device="cuda") < ((lens[slot] + T - 1) // T)[:, None]
    refs.index_put_((table[slot][held].long(),), torch.tensor(-1, dtype=torch.int32, device="cuda"), accumulate=True)
    table[slot] = torch.where(held, -1, table[slot])
    lens[slot] = 0
    return _tables(st)


def _fork(st):
    T = st["c"]["page_tokens"]
    table, lens, refs, src, dst = st["table"], st["lens"], st["refs"], st["slots"].long(), st["dst"].long()
    n = lens[src]
    full, part = n // T, (n % T > 0).long()
    found, _ = _lowest_free(refs)
    page = found[torch.cumsum(part, 0) - part]
    j = torch.arange(table.shape[1], device="cuda")
    shared = j < full[:, None]
    refs.index_put_((table[src][shared].long(),), torch.tensor(1, dtype=torch.int32, device="cuda"), accumulate=True)
    last = table[src, full.clamp(max=table.shape[1] - 1).long()].long()
    table[dst] = torch.where(shared, table[src], torch.where((j == full[:, None]) & (part > 0)[:, None], page[:, None].int(), table[dst]))
    lens[dst] = n
    p = part > 0
    refs[page[p]] = 1
    st["pool"][:, page[p]] = st["pool"][:, last[p]]
    return _tables(st)


def _compact(st):
    T = st["c"]["page_tokens"]
    table, lens, refs = st["table"], st["lens"], st["refs"]
    live = refs > 0
    n_live = live.sum()
    number = torch.arange(refs.numel(), device="cuda")
    src, dst = number[live & (number >= n_live)], number[~live & (number < n_live)]
    to = number.clone()
    to[src] = dst
    held = torch.arange(table.shape[1], device="cuda") < ((lens + T - 1) // T)[:, None]
    table[held] = to[table[held].long()].int()
    refs[dst] = refs[src]
    refs[src] = 0
    st["pool"][:, dst] = st["pool"][:, src]
    st["n_live"].copy_(n_live)
    return _tables(st)


def run(state):
    if own:
        return _own_run(state)
    op = state["c"]["op"]
    if op == "attend":
        return _attend(state)
    if op == "store":
        return _store(state)
    state["state"].copy_(state["kept"])       # the tables as they are before the step
    return {"reserve": _reserve, "free": _free, "fork": _fork, "compact": _compact}[op](state)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------
def exact(case, seed):
    c = dict(_BASE, **case)
    if c["op"] not in ("attend", "store"):
        return None                            # whole numbers only
    st = prepare(case, seed)
    T, H, d = c["page_tokens"], c["kv_heads"], c["head_dim"]
    table, slots = st["table"].cpu().numpy(), st["slots"].cpu().numpy()
    starts, first = st["row_starts"].cpu().numpy(), st["first"].cpu().numpy()
    e4m3 = torch.arange(256, dtype=torch.int32, device="cuda")
    mant, expo = (e4m3 & 7).double(), (e4m3 >> 3) & 15
    value = torch.where(expo == 0, mant / 8 * 2.0 ** -6, (1 + mant / 8) * torch.exp2((expo - 7).double()))
    value = torch.where((e4m3 & 127) == 127, float("nan"), value) * torch.where(e4m3 >= 128, -1.0, 1.0)
    base, nb = H * 2 * T * d, T // BLOCK

    def cached(s, n):
        """K and V of the first n positions of a sequence, [head, position, d]."""
        raw = st["pages"][0][torch.from_numpy(table[slots[s], :-(-n // T)].astype(np.int64)).cuda()].int()
        codes = value[raw[:, :base]].view(-1, H, 2, T * d)
        scale = torch.exp2(raw[:, base:base + H * nb * 2].double() - 127).view(-1, H, nb, 2).repeat_interleave(BLOCK, dim=2)
        k = codes[:, :, 0].reshape(-1, H, T, d) * scale[..., 0, None]
        v = codes[:, :, 1].reshape(-1, H, T // 4, d, 4).permute(0, 1, 2, 4, 3).reshape(-1, H, T, d) * scale[..., 1, None]
        return [x.transpose(0, 1).reshape(H, -1, d)[:, :n] for x in (k, v)]

    if c["op"] == "attend":
        G = c["heads"] // H
        out = torch.empty(st["n_rows"], H, G, d, dtype=torch.float64, device="cuda")
        for s in range(c["seqs"]):
            a, b, p = int(starts[s]), int(starts[s + 1]), int(first[s])
            k, v = cached(s, p + b - a)
            q = st["q"][a:b].double().view(b - a, H, G, d)
            step = max(1, int(3e8) // max(1, c["heads"] * (p + b - a)))
            for r in range(0, b - a, step):
                n = min(step, b - a - r)
                w = torch.matmul(q[r:r + n].permute(1, 2, 0, 3).reshape(H, G * n, d), k.transpose(-1, -2).contiguous()) / math.sqrt(d)
                later = torch.arange(k.shape[1], device="cuda")[None] > torch.arange(p + r, p + r + n, device="cuda")[:, None]
                w = torch.softmax(w.view(H, G, n, -1).masked_fill(later, -math.inf), -1)
                out[a + r:a + r + n] = torch.matmul(w.view(H, G * n, -1), v).view(H, G, n, d).permute(2, 0, 1, 3)
        return out.view(st["n_rows"], -1)
    back = {"k": [], "v": []}
    for s in range(c["seqs"]):
        a, b, p = int(starts[s]), int(starts[s + 1]), int(first[s])
        begin, keep = p // BLOCK * BLOCK, p % BLOCK
        n = keep + b - a
        raw = st["pages"][0][torch.from_numpy(table[slots[s], begin // T:begin // T + 1].astype(np.int64)).cuda()].int()
        old_scale = raw[0, base:base + H * nb * 2].view(H, nb, 2)[:, begin % T // BLOCK].double() - 127
        old = cached(s, p) if keep else None
        for i, name in enumerate(("k", "v")):
            x = torch.zeros(H, -(-n // BLOCK) * BLOCK, d, dtype=torch.float64, device="cuda")
            x[:, keep:n] = st[name][a:b].double().view(b - a, H, d).transpose(0, 1)
            big = x.view(H, -1, BLOCK * d).abs().amax(-1)
            e = torch.ceil(torch.log2(big / 448)).clamp(E_MIN, E_MAX)
            if keep:
                x[:, :keep] = old[i][:, begin:p]
                e[:, 0] = torch.maximum(e[:, 0], old_scale[:, i])
            e = e.repeat_interleave(BLOCK, dim=1)[..., None]
            y = x / torch.exp2(e)
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
            y = (torch.round(y / step) * step).clamp(-448, 448) * torch.exp2(e)
            back[name].append(y[:, :n].transpose(0, 1).reshape(n, -1))
    return {name: torch.cat(v) for name, v in back.items()}
