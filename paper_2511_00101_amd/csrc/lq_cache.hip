// The paged key/value cache: rows in and out (quantisation to e4m3 with a power-of-two scale per block of 16 positions and
// head), and the pages themselves (reserve, fork, free, compact).
#include "lq_cache.h"
#include "lq_internal.h"

namespace lq {

lq_status cache_view(const lq_cache* c, void* workspace, CacheView* out)
{
    if (!c || !c->table || !c->lens || !c->refs) return LQ_ERR_INVALID_ARG;
    if (c->n_kv_heads <= 0 || c->n_pages <= 0 || c->n_slots <= 0 || c->max_pages <= 0) return LQ_ERR_INVALID_ARG;
    const size_t bytes = lora_cache_page_bytes(c->n_kv_heads, c->head_dim, c->page_tokens);
    if (!bytes || (int64_t)c->max_pages * c->page_tokens > (1 << 30) || c->n_pages > kMaxPages) return LQ_ERR_UNSUPPORTED;
    out->n_kv_heads = c->n_kv_heads;
    out->t_log2 = __builtin_ctz((unsigned)c->page_tokens);
    out->n_pages = c->n_pages;
    out->n_slots = c->n_slots;
    out->max_pages = c->max_pages;
    out->max_len = c->max_pages * c->page_tokens;
    out->page_bytes = (long long)bytes;
    out->scale_off = c->n_kv_heads * 2 * c->page_tokens * c->head_dim;
    out->table = c->table;
    out->lens = c->lens;
    out->refs = c->refs;
    out->err = static_cast<int*>(workspace);
    return LQ_OK;
}

lq_status check_spans(const lq_cache* c, const void* pages, const int32_t* row_starts, const int32_t* first, int32_t n_seqs, int32_t n_rows)
{
    if (!c || n_seqs < 0 || n_rows < 0) return LQ_ERR_INVALID_ARG;
    if (n_seqs > 0 && (!pages || !row_starts || !first)) return LQ_ERR_INVALID_ARG;
    if (!aligned16(pages)) return LQ_ERR_UNSUPPORTED;
    return LQ_OK;
}

namespace {

constexpr int kMaxPageTokens = 256;

// =================================================================================================
// Rows into and out of the pages.  One wave takes one block of 16 positions of one head, K and V: lane (kg = lane / 16,
// m = lane % 16) holds positions 4 kg .. 4 kg + 3, columns m * D .. of them (D = head_dim / 16).  So a wave's load of one position
// of the four groups is four whole rows, and a lane has the four positions that a word of V's layout takes together.
// A span's blocks are found without a table of them: span s owns the items from row_starts[s] / 16 + 2 s on, which are enough
// for n rows at any offset (at most (n + 14) / 16 + 1 blocks); the others have nothing to do.
// =================================================================================================
struct BlockJob { int row0, n, first, pos0; const uint8_t* page; int in_page; bool ok; };  // pos0: first position of the block

template <bool STORE>
__device__ __forceinline__ BlockJob find_block(const CacheView& c, const Spans& sp, const uint8_t* pages, int item)
{
    BlockJob j;
    j.ok = false;
    const int s = last_not_above(sp.n_seqs, item, [&](int k) { return (sp.row_starts[k] >> 4) + 2 * k; });
    if (s < 0) return j;
    const Span u = load_span(c, sp, s);
    const int local = item - ((u.row0 >> 4) + 2 * s);
    if (u.n <= 0 || local < 0 || local > ((u.first + u.n - 1) >> 4) - (u.first >> 4)) return j;
    j.row0 = u.row0;
    j.n = u.n;
    j.first = u.first;
    j.pos0 = ((u.first >> 4) + local) * kBlock;
    const int page = c.table[(long long)u.slot * c.max_pages + (j.pos0 >> c.t_log2)];
    if (page < 0 || page >= c.n_pages || (STORE && c.refs[page] != 1)) {
        atomicOr(c.err, kErrBadSegment);
        return j;
    }
    j.page = pages + page * c.page_bytes;
    j.in_page = j.pos0 & ((1 << c.t_log2) - 1);
    j.ok = true;
    return j;
}

template <int N>
__device__ __forceinline__ void load_bf16(const u16* p, float* f)   // N = 4 or 8 consecutive elements
{
    if constexpr (N == 8) unpack8(*reinterpret_cast<const u32x4*>(p), f);
    else {
        const u32x2 w = *reinterpret_cast<const u32x2*>(p);
        f[0] = bf16_lo(w.x); f[1] = bf16_hi(w.x);
        f[2] = bf16_lo(w.y); f[3] = bf16_hi(w.y);
    }
}

__device__ __forceinline__ bool finite(float v) { return fabsf(v) < __builtin_inff(); }

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) v = fmaxf(v, __shfl_xor(v, d, kWave));
    return v;
}

// least e with amax <= 448 * 2^e (448 = 1.75 * 2^8), within [-100, 119]
__device__ __forceinline__ int scale_exponent(float amax)
{
    const unsigned int u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 127 - ((u & 0x7fffffu) <= 0x600000u ? 8 : 7);
    return min(max(e, -100), 119);
}

// two values, already brought to the block's scale, as two e4m3 codes in the low 16 bits
__device__ __forceinline__ unsigned int encode2(float a, float b)
{
    a = finite(a) ? fminf(fmaxf(a, -448.f), 448.f) : __builtin_nanf("");
    b = finite(b) ? fminf(fmaxf(b, -448.f), 448.f) : __builtin_nanf("");
    return (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu;
}
__device__ __forceinline__ unsigned int encode4(const float* f, float r)
{
    return encode2(f[0] * r, f[1] * r) | encode2(f[2] * r, f[3] * r) << 16;
}

// the four codes of a word times a power of two
__device__ __forceinline__ void decode4(unsigned int w, float s, float* f)
{
    const unsigned int lo = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
    const unsigned int hi = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true));
    f[0] = bf16_lo(lo); f[1] = bf16_hi(lo); f[2] = bf16_lo(hi); f[3] = bf16_hi(hi);
}

template <int HD>
__global__ __launch_bounds__(256) void store_rows_kernel(CacheView c, Spans sp, uint8_t* pages, const u16* k, long long ldk,
                                                          const u16* v, long long ldv, int n_items)
{
    constexpr int D = HD / 16, W = D / 4;       // elements per lane and position; words of codes of them
    const int wid = uniform((int)blockIdx.x * 4 + (int)threadIdx.x / kWave);
    const int item = wid / c.n_kv_heads, head = wid - item * c.n_kv_heads;
    if (item >= n_items) return;
    const BlockJob j = find_block<true>(c, sp, pages, item);
    if (!j.ok) return;
    const int lane = lane_id(), kg = lane >> 4, m = lane & 15;
    const int T = 1 << c.t_log2;
    const bool has_old = j.first > j.pos0;
    uint8_t* kc = const_cast<uint8_t*>(j.page) + (long long)head * 2 * T * HD + (j.in_page + 4 * kg) * HD + m * D;
    uint8_t* vc = const_cast<uint8_t*>(j.page) + (long long)(head * 2 + 1) * T * HD + (j.in_page + 4 * kg) * HD + m * D * 4;
    uint8_t* se = const_cast<uint8_t*>(j.page) + c.scale_off + (head * (T / kBlock) + j.in_page / kBlock) * 2;
    const int pos = j.pos0 + 4 * kg;            // this lane's positions: pos .. pos + 3

    float kv[2][4][D];
    float amax[2] = {0.f, 0.f};
    unsigned int is_new = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int i = pos + t - j.first;
        const bool live = i >= 0 && i < j.n;
        is_new |= live ? 1u << t : 0u;
        const long long row = j.row0 + (live ? i : 0);
        load_bf16<D>(k + row * ldk + head * HD + m * D, kv[0][t]);
        load_bf16<D>(v + row * ldv + head * HD + m * D, kv[1][t]);
        if (!live) continue;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int d = 0; d < D; ++d) amax[x] = fmaxf(amax[x], finite(kv[x][t][d]) ? fabsf(kv[x][t][d]) : 0.f);
    }
    int e[2], e_old[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        e[x] = scale_exponent(wave_max(amax[x]));
        e_old[x] = has_old ? (int)se[x] - 127 : e[x];
        e[x] = max(e[x], e_old[x]);
    }
    unsigned int is_old = 0;                    // positions whose codes stay (brought to the new exponent)
#pragma unroll
    for (int t = 0; t < 4; ++t) is_old |= pos + t < j.first ? 1u << t : 0u;

    // K: a position's codes are contiguous
    const float rk = block_scale((unsigned)(127 - e[0])), rv = block_scale((unsigned)(127 - e[1]));
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const bool again = (is_old >> t & 1u) && e[0] != e_old[0];
        if (!(is_new >> t & 1u) && !again) continue;
        unsigned int w[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            float f[4];
            if (again) {
                decode4(reinterpret_cast<const unsigned int*>(kc + t * HD)[i], block_scale((unsigned)(127 + e_old[0])), f);
                w[i] = encode4(f, rk);
            } else {
                w[i] = encode4(&kv[0][t][4 * i], rk);
            }
        }
#pragma unroll
        for (int i = 0; i < W; ++i) reinterpret_cast<unsigned int*>(kc + t * HD)[i] = w[i];
    }
    // V: a word holds four positions of a column
    const unsigned int sel = (is_new & 1u ? 0xffu : 0u) | (is_new & 2u ? 0xff00u : 0u) | (is_new & 4u ? 0xff0000u : 0u) | (is_new & 8u ? 0xff000000u : 0u);
    const bool again = is_old && e[1] != e_old[1];
    if (is_new || again) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            unsigned int old = 0;
            if (is_new != 15u) {
                old = reinterpret_cast<const unsigned int*>(vc)[d];
                if (again) {
                    float f[4];
                    decode4(old, block_scale((unsigned)(127 + e_old[1])), f);
                    old = encode4(f, rv);
                }
            }
            const float f[4] = {kv[1][0][d], kv[1][1][d], kv[1][2][d], kv[1][3][d]};
            reinterpret_cast<unsigned int*>(vc)[d] = (encode4(f, rv) & sel) | (old & ~sel);
        }
    }
    if (lane < 2) se[lane] = (uint8_t)((lane == 0 ? e[0] : e[1]) + 127);
}

template <int HD>
__global__ __launch_bounds__(256) void load_rows_kernel(CacheView c, Spans sp, const uint8_t* pages, u16* k, long long ldk,
                                                         u16* v, long long ldv, int n_items)
{
    constexpr int D = HD / 16, W = D / 4;
    const int wid = uniform((int)blockIdx.x * 4 + (int)threadIdx.x / kWave);
    const int item = wid / c.n_kv_heads, head = wid - item * c.n_kv_heads;
    if (item >= n_items) return;
    const BlockJob j = find_block<false>(c, sp, pages, item);
    if (!j.ok) return;
    const int lane = lane_id(), kg = lane >> 4, m = lane & 15;
    const int T = 1 << c.t_log2;
    const uint8_t* kc = j.page + (long long)head * 2 * T * HD + (j.in_page + 4 * kg) * HD + m * D;
    const uint8_t* vc = j.page + (long long)(head * 2 + 1) * T * HD + (j.in_page + 4 * kg) * HD + m * D * 4;
    const uint8_t* se = j.page + c.scale_off + (head * (T / kBlock) + j.in_page / kBlock) * 2;
    const float sk = block_scale(se[0]), sv = block_scale(se[1]);
    unsigned int vw[D];
#pragma unroll
    for (int d = 0; d < D; ++d) vw[d] = reinterpret_cast<const unsigned int*>(vc)[d];
    float vf[D][4];
#pragma unroll
    for (int d = 0; d < D; ++d) decode4(vw[d], sv, vf[d]);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int i = j.pos0 + 4 * kg + t - j.first;
        if (i < 0 || i >= j.n) continue;
        const long long row = j.row0 + i;
        u16* ko = k + row * ldk + head * HD + m * D;
        u16* vo = v + row * ldv + head * HD + m * D;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            float f[4];
            decode4(reinterpret_cast<const unsigned int*>(kc + t * HD)[w], sk, f);
            reinterpret_cast<u32x2*>(ko)[w] = u32x2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
            reinterpret_cast<u32x2*>(vo)[w] = u32x2{pack_bf16x2(vf[4 * w][t], vf[4 * w + 1][t]), pack_bf16x2(vf[4 * w + 2][t], vf[4 * w + 3][t])};
        }
    }
}

// =================================================================================================
// Page management.  The state is three integer arrays; every call is a function of them that does not depend on the order in
// which workgroups run.  Pages are counted in segments of 4096; the plan of the requests (which slot, how many pages, running
// sum) is made by one workgroup while others count the free pages, and the next launch hands the lowest free
// pages out: every segment's workgroup adds up the counts before it, and finds the request of a free page by its rank.
// =================================================================================================
constexpr int kSegPages = 4096;
constexpr int kPlanThreads = 256;

// The workspace behind its header.
struct PagePlan {
    int* seg_free;      // [segments] free pages (compact: pages in use)
    int* slot;          // per request: slot that gets pages, or -1
    int* have;          // per request: first new entry of the slot's table row
    int* add;           // per request: what its length becomes (fork) or grows by (reserve)
    int* src;           // fork: source slot
    int* upto;          // running sum of the pages wanted, this request's included
    int* page;          // fork: page that the last, partly filled one is copied into; -1: none
    int* from;          // fork: the page copied
    int* mark;          // [n_slots] first request that lists the slot
    int* list_src;      // [n_pages] compact
    int* list_dst;      // [n_pages]
    int* rank;          // [n_pages]
    int* totals;        // [4]
};

size_t plan_ints(int n_pages, int n_slots, int n)
{
    return (size_t)(n_pages + kSegPages - 1) / kSegPages + 7 * (size_t)n + (size_t)n_slots + 3 * (size_t)n_pages + 4;
}

PagePlan plan_of(void* workspace, int n_pages, int n_slots, int n)
{
    PagePlan p;
    int* at = reinterpret_cast<int*>(static_cast<char*>(workspace) + kWsHeaderBytes);
    const auto take = [&](size_t k) { int* q = at; at += k; return q; };
    p.seg_free = take((size_t)(n_pages + kSegPages - 1) / kSegPages);
    p.slot = take(n); p.have = take(n); p.add = take(n); p.src = take(n); p.upto = take(n); p.page = take(n); p.from = take(n);
    p.mark = take(n_slots);
    p.list_src = take(n_pages); p.list_dst = take(n_pages); p.rank = take(n_pages);
    p.totals = take(4);
    return p;
}

__device__ __forceinline__ int wave_sum(int v)
{
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor(v, d, kWave);
    return v;
}
// sum over the workgroup of kPlanThreads threads (slot: kPlanThreads / 64 ints of LDS)
__device__ __forceinline__ int block_sum(int v, int* slot)
{
    v = wave_sum(v);
    __syncthreads();
    if (lane_id() == 0) slot[threadIdx.x / kWave] = v;
    __syncthreads();
    int s = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / kWave; ++w) s += slot[w];
    return s;
}
// inclusive prefix sum over the workgroup; total: the whole sum
__device__ __forceinline__ int block_scan(int v, int* slot, int* total)
{
    const int inc = wave_inclusive_scan(v);
    __syncthreads();
    if (lane_id() == kWave - 1) slot[threadIdx.x / kWave] = inc;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / kWave; ++w) {
        if (w < (int)threadIdx.x / kWave) before += slot[w];
        all += slot[w];
    }
    *total = all;
    return inc + before;
}

// pages of segment seg with refs > 0 (LIVE) or refs <= 0, counted by the workgroup
template <bool LIVE>
__device__ __forceinline__ void count_segment(const CacheView& c, int seg, int* seg_count, int* slot)
{
    int n = 0;
    for (int i = (int)threadIdx.x; i < kSegPages; i += kPlanThreads) {
        const int p = seg * kSegPages + i;
        if (p < c.n_pages) n += (c.refs[p] > 0) == LIVE;
    }
    n = block_sum(n, slot);
    if (threadIdx.x == 0) seg_count[seg] = n;
}

struct Requests { const int32_t* slots; const int32_t* dst; const int32_t* amount; int n; };  // dst: fork; amount: add or keep

// Launch 1: workgroup 0 plans the requests, the others count.
template <bool FORK>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(CacheView c, PagePlan p, Requests rq)
{
    __shared__ int slot_sums[kPlanThreads / kWave];
    if (blockIdx.x > 0) {
        count_segment<false>(c, (int)blockIdx.x - 1, p.seg_free, slot_sums);
        return;
    }
    const int32_t* changed = FORK ? rq.dst : rq.slots;     // slots that the call writes
    const auto in_range = [&](int s) { return s >= 0 && s < c.n_slots; };
    for (int i = (int)threadIdx.x; i < rq.n; i += kPlanThreads)
        if (in_range(changed[i])) __hip_atomic_store(p.mark + changed[i], 0x7fffffff, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    for (int i = (int)threadIdx.x; i < rq.n; i += kPlanThreads)
        if (in_range(changed[i])) __hip_atomic_fetch_min(p.mark + changed[i], i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const int T = 1 << c.t_log2;
    int base = 0;
    for (int i0 = 0; i0 < rq.n; i0 += kPlanThreads) {
        const int i = i0 + (int)threadIdx.x;
        int need = 0;
        if (i < rq.n) {
            const int s = changed[i];
            bool ok = in_range(s) && __hip_atomic_load(p.mark + s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i;
            const int len = ok ? c.lens[s] : 0;
            int have = 0, add = 0, from = -1, src = -1;
            if (FORK) {
                src = rq.slots[i];
                ok = ok && in_range(src) && len == 0;
                const int all = ok ? c.lens[src] : 0;
                add = rq.amount ? rq.amount[i] : all;
                ok = ok && all <= c.max_len && add >= 0 && add <= all;
                if (ok) {
                    have = add >> c.t_log2;
                    need = (add & (T - 1)) != 0;
                    if (need) {
                        from = c.table[(long long)src * c.max_pages + have];
                        ok = from >= 0 && from < c.n_pages;
                    }
                }
            } else {
                add = rq.amount[i];
                ok = ok && add >= 0 && len >= 0 && len <= c.max_len && add <= c.max_len - len;
                if (ok) {
                    have = (len + T - 1) >> c.t_log2;
                    need = ((len + add + T - 1) >> c.t_log2) - have;
                }
            }
            need = min(need, c.n_pages + 1);      // (more is not to be had; keeps the sums within 32 bits)
            if (!ok) {
                need = 0;
                atomicOr(c.err, kErrBadSegment);
            }
            p.slot[i] = ok ? s : -1;
            p.have[i] = have;
            p.add[i] = add;
            if (FORK) {
                p.src[i] = src;
                p.from[i] = from;
                p.page[i] = -1;
            }
        }
        int total;
        const int inc = block_scan(need, slot_sums, &total);
        if (i < rq.n) p.upto[i] = min(base + inc, c.n_pages + 1);
        base = min(base + total, c.n_pages + 1);
        __syncthreads();
    }
}

// first request whose running sum is above r, of n
__device__ __forceinline__ int request_of(const int* upto, int n, int r)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (upto[mid] > r) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Launch 2: workgroup g < segments hands out the free pages of segment g; the others (fork: one request each wave; reserve: lengths)
// bring the slots' state up to date.
template <bool FORK>
__global__ __launch_bounds__(kPlanThreads) void assign_kernel(CacheView c, PagePlan p, int n, int n_seg)
{
    __shared__ int sums[kPlanThreads / kWave];
    int before = 0, all = 0;
    const int seg = (int)blockIdx.x;
    for (int s = (int)threadIdx.x; s < n_seg; s += kPlanThreads) {
        const int f = p.seg_free[s];
        all += f;
        before += s < seg ? f : 0;
    }
    all = block_sum(all, sums);
    before = block_sum(before, sums);
    const int wanted = p.upto[n - 1];
    if (seg < n_seg) {
        if (before >= wanted) return;
        for (int i0 = 0; i0 < kSegPages; i0 += kPlanThreads) {
            const int page = seg * kSegPages + i0 + (int)threadIdx.x;
            const bool is_free = page < c.n_pages && c.refs[page] <= 0;
            int total;
            const int r = before + block_scan(is_free ? 1 : 0, sums, &total) - 1;
            if (is_free && r < wanted) {
                const int i = request_of(p.upto, n, r);
                if (p.upto[i] <= all) {
                    const int mine = r - (i ? p.upto[i - 1] : 0);
                    c.table[(long long)p.slot[i] * c.max_pages + p.have[i] + mine] = page;
                    c.refs[page] = 1;
                    if (FORK) p.page[i] = page;
                }
            }
            before += total;
            if (before >= wanted) break;
        }
        return;
    }
    if (!FORK) {
        for (int i = (seg - n_seg) * kPlanThreads + (int)threadIdx.x; i < n; i += kPlanThreads * ((int)gridDim.x - n_seg)) {
            if (p.upto[i] > all) atomicOr(c.err, kErrNoPages);
            else if (p.slot[i] >= 0) c.lens[p.slot[i]] += p.add[i];
        }
        return;
    }
    const int i = (seg - n_seg) * (kPlanThreads / kWave) + (int)threadIdx.x / kWave;
    if (i >= n) return;
    if (p.upto[i] > all) {
        if (lane_id() == 0) atomicOr(c.err, kErrNoPages);
        return;
    }
    const int dst = p.slot[i];
    if (dst < 0) return;
    const int32_t* from = c.table + (long long)p.src[i] * c.max_pages;
    int32_t* to = c.table + (long long)dst * c.max_pages;
    for (int j = lane_id(); j < p.have[i]; j += kWave) {
        const int page = from[j];
        to[j] = page;
        if (page >= 0 && page < c.n_pages) atomicAdd(c.refs + page, 1);
        else atomicOr(c.err, kErrBadSegment);
    }
    if (lane_id() == 0) c.lens[dst] = p.add[i];
}

// ---- whole pages, in every pool: 16 KB a step of a workgroup --------------------------------------------------------
constexpr int kCopyThreads = 256, kCopyBytes = 16384;

__device__ __forceinline__ void copy_piece(const uint8_t* src, uint8_t* dst, int bytes)   // a multiple of 16, at most kCopyBytes
{
    u32x4 v[kCopyBytes / (16 * kCopyThreads)];
    constexpr int N = kCopyBytes / (16 * kCopyThreads);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int at = (k * kCopyThreads + (int)threadIdx.x) * 16;
        if (at < bytes) v[k] = *reinterpret_cast<const u32x4*>(src + at);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int at = (k * kCopyThreads + (int)threadIdx.x) * 16;
        if (at < bytes) *reinterpret_cast<u32x4*>(dst + at) = v[k];
    }
}

__global__ __launch_bounds__(kCopyThreads) void copy_pages_kernel(CacheView c, const int* src, const int* dst, const int* n_dev, int n_host,
                                                                  void* const* pools, int n_pools)
{
    const int n = n_dev ? *n_dev : n_host;
    const int pieces = (int)((c.page_bytes + kCopyBytes - 1) / kCopyBytes);
    const long long units = (long long)n * n_pools * pieces;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const int piece = (int)(u % pieces);
        const int i = (int)(u / pieces % n), pool = (int)(u / pieces / n);
        const int from = src[i], to = dst[i];
        if (to < 0 || from < 0) continue;
        const long long at = (long long)piece * kCopyBytes;
        uint8_t* base = static_cast<uint8_t*>(pools[pool]);
        copy_piece(base + from * c.page_bytes + at, base + to * c.page_bytes + at, (int)min((long long)kCopyBytes, c.page_bytes - at));
    }
}

__global__ __launch_bounds__(kPlanThreads) void free_kernel(CacheView c, const int32_t* slots)
{
    __shared__ int s_len;
    const int s = slots[blockIdx.x];
    if (s < 0 || s >= c.n_slots) {
        if (threadIdx.x == 0) atomicOr(c.err, kErrBadSegment);
        return;
    }
    // (a slot that is listed again finds length 0)
    if (threadIdx.x == 0) s_len = atomicExch(c.lens + s, 0);
    __syncthreads();
    const int len = s_len;
    if (len < 0 || len > c.max_len) {
        if (threadIdx.x == 0) atomicOr(c.err, kErrBadSegment);
        return;
    }
    const int held = (len + (1 << c.t_log2) - 1) >> c.t_log2;
    int32_t* row = c.table + (long long)s * c.max_pages;
    for (int j = (int)threadIdx.x; j < held; j += kPlanThreads) {
        const int page = row[j];
        row[j] = -1;
        const bool ok = page >= 0 && page < c.n_pages;
        if (ok && atomicSub(c.refs + page, 1) > 0) continue;
        if (ok) atomicAdd(c.refs + page, 1);       // it was free already
        atomicOr(c.err, kErrBadSegment);
    }
}

// ---- compact --------------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(kPlanThreads) void count_live_kernel(CacheView c, PagePlan p)
{
    __shared__ int sums[kPlanThreads / kWave];
    count_segment<true>(c, (int)blockIdx.x, p.seg_free, sums);
}

// Lists of the pages that move and of where they go, and every page's place in the list (-1: stays).
__global__ __launch_bounds__(kPlanThreads) void list_moves_kernel(CacheView c, PagePlan p, int n_seg)
{
    __shared__ int sums[kPlanThreads / kWave];
    const int seg = (int)blockIdx.x;
    int before = 0, n_live = 0;
    for (int s = (int)threadIdx.x; s < n_seg; s += kPlanThreads) {
        const int f = p.seg_free[s];
        n_live += f;
        before += s < seg ? f : 0;
    }
    n_live = block_sum(n_live, sums);
    before = block_sum(before, sums);
    // pages in use among the first n_live: whole segments by their counts, the one that n_live cuts by its refs
    const int cut = n_live / kSegPages;
    int low = 0;
    for (int s = (int)threadIdx.x; s < min(cut, n_seg); s += kPlanThreads) low += p.seg_free[s];
    for (int i = cut * kSegPages + (int)threadIdx.x; i < n_live; i += kPlanThreads) low += c.refs[i] > 0;
    low = block_sum(low, sums);
    if (seg == 0 && threadIdx.x == 0) {
        p.totals[0] = n_live - low;
        p.totals[1] = n_live;
    }
    for (int i0 = 0; i0 < kSegPages; i0 += kPlanThreads) {
        const int page = seg * kSegPages + i0 + (int)threadIdx.x;
        const bool live = page < c.n_pages && c.refs[page] > 0;
        int total;
        const int upto = before + block_scan(live ? 1 : 0, sums, &total);   // pages in use up to this one
        int rank = -1;
        if (live && page >= n_live) {
            rank = upto - 1 - low;
            p.list_src[rank] = page;
        }
        if (!live && page < n_live) p.list_dst[page - upto] = page;
        if (page < c.n_pages) p.rank[page] = rank;
        before += total;
    }
}

// The first workgroups move the refs, the others rewrite a slot's table row each.
__global__ __launch_bounds__(kPlanThreads) void follow_moves_kernel(CacheView c, PagePlan p, int n_ref_groups, int32_t* n_live)
{
    const int moves = p.totals[0];
    if ((int)blockIdx.x < n_ref_groups) {
        for (int i = (int)blockIdx.x * kPlanThreads + (int)threadIdx.x; i < moves; i += n_ref_groups * kPlanThreads) {
            const int from = p.list_src[i], to = p.list_dst[i];
            c.refs[to] = c.refs[from];
            c.refs[from] = 0;
        }
        if (n_live && blockIdx.x == 0 && threadIdx.x == 0) *n_live = p.totals[1];
        return;
    }
    const int s = (int)blockIdx.x - n_ref_groups;
    const int len = c.lens[s];
    if (len < 0 || len > c.max_len) {
        if (threadIdx.x == 0) atomicOr(c.err, kErrBadSegment);
        return;
    }
    const int held = (len + (1 << c.t_log2) - 1) >> c.t_log2;
    int32_t* row = c.table + (long long)s * c.max_pages;
    for (int j = (int)threadIdx.x; j < held; j += kPlanThreads) {
        const int page = row[j];
        if (page < 0 || page >= c.n_pages) {
            atomicOr(c.err, kErrBadSegment);
            continue;
        }
        const int r = p.rank[page];
        if (r >= 0) row[j] = p.list_dst[r];
    }
}

int segments_of(int n_pages) { return (n_pages + kSegPages - 1) / kSegPages; }

lq_status launched() { return hipGetLastError() == hipSuccess ? LQ_OK : LQ_ERR_HIP; }

// what the page calls share; n = 0 requests is valid for all of them
lq_status page_call(const lq_cache* c, int32_t n, void* workspace, size_t workspace_bytes, CacheView* view)
{
    if (n < 0) return LQ_ERR_INVALID_ARG;
    const lq_status st = cache_view(c, workspace, view);
    if (st != LQ_OK) return st;
    if (!workspace || !aligned16(workspace) || workspace_bytes < lora_cache_workspace_bytes(c, n)) return LQ_ERR_WORKSPACE;
    return LQ_OK;
}

int copy_grid(long long most)
{
    return (int)(most < 1 ? 1 : most < 4096 ? most : 4096);
}

template <bool STORE>
lq_status move_cache_rows(void* k, int64_t ldk, void* v, int64_t ldv, int32_t n_rows, const lq_cache* host_cache, void* pages,
                          const int32_t* slots, const int32_t* row_starts, const int32_t* first, int32_t n_seqs,
                          void* workspace, size_t workspace_bytes, void* stream)
{
    CacheView c;
    lq_status st = check_spans(host_cache, pages, row_starts, first, n_seqs, n_rows);
    if (st == LQ_OK) st = cache_view(host_cache, workspace, &c);
    if (st != LQ_OK) return st;
    const int64_t width = (int64_t)host_cache->n_kv_heads * host_cache->head_dim;
    if (ldk < width || ldv < width) return LQ_ERR_INVALID_ARG;
    if (n_rows > 0 && (!k || !v || k == v)) return LQ_ERR_INVALID_ARG;
    if ((ldk % 8) || (ldv % 8) || !aligned16(k) || !aligned16(v)) return LQ_ERR_UNSUPPORTED;
    const int64_t items = (int64_t)n_rows / kBlock + 2 * (int64_t)n_seqs;
    if (items * host_cache->n_kv_heads > 0x7fffffff) return LQ_ERR_UNSUPPORTED;
    if (!workspace || !aligned16(workspace) || workspace_bytes < LQ_CACHE_MIN_WORKSPACE) return LQ_ERR_WORKSPACE;
    if (n_seqs == 0 || n_rows == 0) return LQ_OK;
    const Spans sp{slots, row_starts, first, n_seqs, n_rows};
    const dim3 grid((unsigned)((items * host_cache->n_kv_heads + 3) / 4)), block(256);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    uint8_t* pg = static_cast<uint8_t*>(pages);
    if constexpr (STORE) {
        const auto kernel = host_cache->head_dim == 128 ? store_rows_kernel<128> : store_rows_kernel<64>;
        hipLaunchKernelGGL(kernel, grid, block, 0, hs, c, sp, pg, static_cast<const u16*>(k), (long long)ldk,
                           static_cast<const u16*>(v), (long long)ldv, (int)items);
    } else {
        const auto kernel = host_cache->head_dim == 128 ? load_rows_kernel<128> : load_rows_kernel<64>;
        hipLaunchKernelGGL(kernel, grid, block, 0, hs, c, sp, pg, static_cast<u16*>(k), (long long)ldk, static_cast<u16*>(v),
                           (long long)ldv, (int)items);
    }
    return launched();
}

}  // namespace
}  // namespace lq

extern "C" size_t lora_cache_page_bytes(int32_t n_kv_heads, int32_t head_dim, int32_t page_tokens)
{
    if (n_kv_heads <= 0 || n_kv_heads > LQ_CACHE_MAX_HEADS || (head_dim != 64 && head_dim != 128)) return 0;
    if (page_tokens < LQ_CACHE_BLOCK || page_tokens > lq::kMaxPageTokens || (page_tokens & (page_tokens - 1))) return 0;
    const size_t bytes = (size_t)n_kv_heads * 2 * page_tokens * head_dim + (size_t)n_kv_heads * (page_tokens / LQ_CACHE_BLOCK) * 2;
    return (bytes + 127) / 128 * 128;
}

extern "C" size_t lora_cache_workspace_bytes(const lq_cache* host_cache, int32_t n_seqs)
{
    if (!host_cache || n_seqs < 0 || host_cache->n_pages <= 0 || host_cache->n_slots <= 0) return 0;
    return lq::kWsHeaderBytes + 4 * lq::plan_ints(host_cache->n_pages, host_cache->n_slots, n_seqs);
}

extern "C" lq_status lora_cache_reserve(const lq_cache* host_cache, const int32_t* slots, const int32_t* add, int32_t n_seqs,
                                        void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace lq;
    CacheView c;
    if (n_seqs > 0 && (!slots || !add)) return LQ_ERR_INVALID_ARG;
    const lq_status st = page_call(host_cache, n_seqs, workspace, workspace_bytes, &c);
    if (st != LQ_OK || n_seqs == 0) return st;
    const PagePlan p = plan_of(workspace, c.n_pages, c.n_slots, n_seqs);
    const int n_seg = segments_of(c.n_pages);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(plan_kernel<false>, dim3(1 + n_seg), dim3(kPlanThreads), 0, hs, c, p, Requests{slots, nullptr, add, n_seqs});
    hipLaunchKernelGGL(assign_kernel<false>, dim3(n_seg + 1), dim3(kPlanThreads), 0, hs, c, p, n_seqs, n_seg);
    return launched();
}

extern "C" lq_status lora_cache_fork(const lq_cache* host_cache, const int32_t* src_slots, const int32_t* dst_slots, const int32_t* keep,
                                     int32_t n_seqs, void* const* pools, int32_t n_pools, void* workspace, size_t workspace_bytes,
                                     void* stream)
{
    using namespace lq;
    CacheView c;
    if (n_pools < 0 || (n_pools > 0 && !pools) || (n_seqs > 0 && (!src_slots || !dst_slots))) return LQ_ERR_INVALID_ARG;
    const lq_status st = page_call(host_cache, n_seqs, workspace, workspace_bytes, &c);
    if (st != LQ_OK || n_seqs == 0) return st;
    const PagePlan p = plan_of(workspace, c.n_pages, c.n_slots, n_seqs);
    const int n_seg = segments_of(c.n_pages);
    const int waves = kPlanThreads / kWave;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(plan_kernel<true>, dim3(1 + n_seg), dim3(kPlanThreads), 0, hs, c, p, Requests{src_slots, dst_slots, keep, n_seqs});
    hipLaunchKernelGGL(assign_kernel<true>, dim3(n_seg + (n_seqs + waves - 1) / waves), dim3(kPlanThreads), 0, hs, c, p, n_seqs, n_seg);
    if (n_pools > 0) {
        const long long most = (long long)n_seqs * n_pools * ((c.page_bytes + kCopyBytes - 1) / kCopyBytes);
        hipLaunchKernelGGL(copy_pages_kernel, dim3(copy_grid(most)), dim3(kCopyThreads), 0, hs, c, p.from, p.page, nullptr, n_seqs, pools,
                           n_pools);
    }
    return launched();
}

extern "C" lq_status lora_cache_free(const lq_cache* host_cache, const int32_t* slots, int32_t n_seqs, void* workspace,
                                     size_t workspace_bytes, void* stream)
{
    using namespace lq;
    CacheView c;
    if (n_seqs > 0 && !slots) return LQ_ERR_INVALID_ARG;
    const lq_status st = page_call(host_cache, n_seqs, workspace, workspace_bytes, &c);
    if (st != LQ_OK || n_seqs == 0) return st;
    hipLaunchKernelGGL(free_kernel, dim3(n_seqs), dim3(kPlanThreads), 0, static_cast<hipStream_t>(stream), c, slots);
    return launched();
}

extern "C" lq_status lora_cache_compact(const lq_cache* host_cache, void* const* pools, int32_t n_pools, int32_t* n_live, void* workspace,
                                        size_t workspace_bytes, void* stream)
{
    using namespace lq;
    CacheView c;
    if (n_pools < 0 || (n_pools > 0 && !pools)) return LQ_ERR_INVALID_ARG;
    const lq_status st = page_call(host_cache, 0, workspace, workspace_bytes, &c);
    if (st != LQ_OK) return st;
    const PagePlan p = plan_of(workspace, c.n_pages, c.n_slots, 0);
    const int n_seg = segments_of(c.n_pages);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(count_live_kernel, dim3(n_seg), dim3(kPlanThreads), 0, hs, c, p);
    hipLaunchKernelGGL(list_moves_kernel, dim3(n_seg), dim3(kPlanThreads), 0, hs, c, p, n_seg);
    const int ref_groups = n_seg < 64 ? n_seg : 64;
    hipLaunchKernelGGL(follow_moves_kernel, dim3(ref_groups + c.n_slots), dim3(kPlanThreads), 0, hs, c, p, ref_groups, n_live);
    if (n_pools > 0) {
        const long long most = ((long long)c.n_pages / 2 + 1) * n_pools * ((c.page_bytes + kCopyBytes - 1) / kCopyBytes);
        hipLaunchKernelGGL(copy_pages_kernel, dim3(copy_grid(most)), dim3(kCopyThreads), 0, hs, c, p.list_src, p.list_dst, p.totals, 0, pools,
                           n_pools);
    }
    return launched();
}

extern "C" lq_status lora_cache_store_rows(const void* k, int64_t ldk, const void* v, int64_t ldv, int32_t n_rows, const lq_cache* host_cache,
                                           void* pages, const int32_t* slots, const int32_t* row_starts, const int32_t* first, int32_t n_seqs,
                                           void* workspace, size_t workspace_bytes, void* stream)
{
    return lq::move_cache_rows<true>(const_cast<void*>(k), ldk, const_cast<void*>(v), ldv, n_rows, host_cache, pages, slots, row_starts, first,
                                     n_seqs, workspace, workspace_bytes, stream);
}

extern "C" lq_status lora_cache_load_rows(void* k, int64_t ldk, void* v, int64_t ldv, int32_t n_rows, const lq_cache* host_cache,
                                          const void* pages, const int32_t* slots, const int32_t* row_starts, const int32_t* first,
                                          int32_t n_seqs, void* workspace, size_t workspace_bytes, void* stream)
{
    return lq::move_cache_rows<false>(k, ldk, v, ldv, n_rows, host_cache, const_cast<void*>(pages), slots, row_starts, first, n_seqs, workspace,
                                      workspace_bytes, stream);
}
