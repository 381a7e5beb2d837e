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
    if (!bytes || (int64_t)c->max_pages * c->page_tokens > (1 << 30) || c->n_pages > kMaxPages || c->n_slots > kMaxSlots)
        return LQ_ERR_UNSUPPORTED;
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
constexpr int kMaxRowWaves = 1 << 25;           // (a launch has fewer than 2^32 threads)

// =================================================================================================
// Rows into and out of the pages.  One wave takes one block of 16 positions of one head, K and V: lane (kg = lane / 16,
// m = lane % 16) holds positions 4 kg .. 4 kg + 3, columns m * D .. of them (D = head_dim / 16).  So a wave's load of one position
// of the four groups is four whole rows, and a lane has the four positions that a word of V's layout takes together.
// A span's blocks are found without a table of them: span s owns the items from row_starts[s] / 16 + 2 s on, which are enough
// for n rows at any offset (at most (n + 14) / 16 + 1 blocks); the others have nothing to do.
// Bound and measured (8 key heads of 128; a store and a load in turn, and in brackets either repeated alone in a graph): one row each of 256 sequences is a chain
// of five dependent round trips, 7.0 us to store (6.6) and 6.6 to read back (4.7) for 15 MB; 12 prompts of up to 2048 rows by bandwidth, 15.3 (12.0) and 12.2 us
// (11.7) for 60 MB each: 3.9 and 4.9 TB/s where a copy reaches 5.1.  Storing, a block's elements are looked at as packed magnitudes and converted in pairs,
// the scale being an operand of the conversion; with the elements widened to fp32 one by one the vector instructions took half of the cycles (alone 8.0 and
// 15.0 us to store).
// =================================================================================================
// A wave's start is a chain of dependent round trips (spans, span, table and rows, page); nothing of a trip waits for a check of the one
// before: indexes are brought into range instead, and what was found is looked at when all of it is there.
struct BlockJob { int slot, row0, n, first, pos0, page, len; bool rows_ok; };  // pos0: first position of the block

// span and block of an item, with its length and page requested; false: nothing to do
__device__ __forceinline__ bool find_block(const CacheView& c, const Spans& sp, int item, BlockJob& j)
{
    const int s = uniform(last_not_above(sp.n_seqs, item, [&](int k) { return (sp.row_starts[k] >> 4) + 2 * k; }));
    if (s < 0) return false;
    j.slot = sp.slots ? sp.slots[s] : s;
    j.row0 = sp.row_starts[s];
    int end = sp.row_starts[s + 1];
    j.first = sp.first[s];
    // (lane 0's values, read here: the loads are one round trip, none of them moved behind a branch)
    j.slot = uniform(j.slot);
    j.row0 = uniform(j.row0);
    end = uniform(end);
    j.first = uniform(j.first);
    j.rows_ok = bool(j.row0 >= 0) & bool(end >= j.row0) & bool(end <= sp.n_rows);
    j.n = j.rows_ok ? end - j.row0 : 0;
    const int local = item - ((j.row0 >> 4) + 2 * s);
    const bool reach = bool(j.first >= 0) & bool(j.n <= c.max_len - j.first);
    if (local < 0 || j.n == 0) return false;           // (row_starts that decrease; no rows, or none inside the matrices)
    // (a span whose positions cannot be used is reported by the wave of its first item)
    if (local > 0 && (!reach || local > ((j.first + j.n - 1) >> 4) - (j.first >> 4))) return false;
    j.rows_ok = reach;
    j.pos0 = j.rows_ok ? ((j.first >> 4) + local) * kBlock : 0;
    const int slot = min(max(j.slot, 0), c.n_slots - 1);
    j.len = c.lens[slot];
    j.page = c.table[(long long)slot * c.max_pages + (j.pos0 >> c.t_log2)];
    j.rows_ok = j.rows_ok & bool(j.slot == slot);
    return true;
}
// Spans whose rows are not inside the matrices, 64 by a wave behind those with items: no search needs to find one (row_starts that decrease, or
// begin in front of the matrices), and the waves with items wait for nothing more (256 rows read back 4.3 -> 4.7 us, 8000 rows of one prompt 11.0 -> 10.5).
__device__ __forceinline__ void report_rows(const CacheView& c, const Spans& sp, int wave)
{
    const int s = wave * kWave + lane_id();
    if (s >= sp.n_seqs) return;
    const int begin = sp.row_starts[s], end = sp.row_starts[s + 1];
    if (begin < 0 || end < begin || end > sp.n_rows) atomicOr(c.err, kErrBadSegment);
}
__device__ __forceinline__ bool usable(const CacheView& c, BlockJob& j)
{
    j.len = uniform(j.len);
    j.page = uniform(j.page);
    return j.rows_ok & bool(j.len >= 0) & bool(j.len <= c.max_len) & bool(j.first <= j.len) & bool(j.n <= j.len - j.first) & bool(j.page >= 0) &
           bool(j.page < c.n_pages);
}

template <int N>
struct Packed {                                  // N = 4 or 8 consecutive bf16 elements
    unsigned int w[N / 2];
    __device__ __forceinline__ void load(const u16* p)
    {
        if constexpr (N == 8) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(p);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            const u32x2 v = *reinterpret_cast<const u32x2*>(p);
            w[0] = v.x; w[1] = v.y;
        }
    }
    // here the loads are waited for (and not behind a branch that they were moved across)
    __device__ __forceinline__ void arrive()
    {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) asm volatile("" : "+v"(w[i]));
    }
    __device__ __forceinline__ float at(int i) const { return i % 2 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]); }
};

// N words at a time: 1, 2, 4 or 8
template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, unsigned int (&w)[N])
{
    if constexpr (N == 1) w[0] = *reinterpret_cast<const unsigned int*>(p);
    else if constexpr (N == 2) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(p);
        w[0] = v.x; w[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(p + 4 * i);
            w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
        }
    }
}
template <int N>
__device__ __forceinline__ void store_words(uint8_t* p, const unsigned int (&w)[N])
{
    if constexpr (N == 1) *reinterpret_cast<unsigned int*>(p) = w[0];
    else if constexpr (N == 2) *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
    else {
#pragma unroll
        for (int i = 0; i < N; i += 4) *reinterpret_cast<u32x4*>(p + 4 * i) = u32x4{w[i], w[i + 1], w[i + 2], w[i + 3]};
    }
}

__device__ __forceinline__ bool finite(float v) { return fabsf(v) < __builtin_inff(); }

// largest of the wave's values, in every lane: rotations within rows of 16 lanes, then rows and halves swapped
__device__ __forceinline__ unsigned int wave_max(unsigned int v)
{
    typedef __attribute__((ext_vector_type(2))) unsigned int pair;
#define LQ_ROTATED(n) (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + (n), 0xf, 0xf, false)
    v = max(v, LQ_ROTATED(1));
    v = max(v, LQ_ROTATED(2));
    v = max(v, LQ_ROTATED(4));
    v = max(v, LQ_ROTATED(8));
#undef LQ_ROTATED
    const pair a = __builtin_bit_cast(pair, __builtin_amdgcn_permlane16_swap(v, v, false, false));
    v = max(a.x, a.y);
    const pair b = __builtin_bit_cast(pair, __builtin_amdgcn_permlane32_swap(v, v, false, false));
    return max(b.x, b.y);
}

constexpr unsigned int kBf16Inf = 0x7f80;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
// larger of each half, as unsigned numbers (of magnitudes: NaN, infinity, finite values by size)
__device__ __forceinline__ unsigned int larger_halves(unsigned int a, unsigned int b)
{
    return __builtin_bit_cast(unsigned int, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// codes of four bf16 values, finite and at most 448 * scale (a power of two)
__device__ __forceinline__ unsigned int encode4_in_range(unsigned int w01, unsigned int w23, float scale)
{
    typedef __attribute__((ext_vector_type(2))) short s16x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    s16x2 c = {0, 0};
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, w01), scale, false);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, w23), scale, true);
    return __builtin_bit_cast(unsigned int, c);
}

// least e with amax <= 448 * 2^e (448 = 1.75 * 2^8), within [-100, 119]
constexpr int kLargestExponent = 119;
__device__ __forceinline__ int scale_exponent(float amax)
{
    const unsigned int u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 127 - ((u & 0x7fffffu) <= 0x600000u ? 8 : 7);
    return min(max(e, -100), kLargestExponent);
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
    if (item >= n_items) {
        report_rows(c, sp, wid - n_items * c.n_kv_heads);
        return;
    }
    BlockJob j;
    if (!find_block(c, sp, item, j)) return;
    const int lane = lane_id(), kg = lane >> 4, m = lane & 15;
    const int T = 1 << c.t_log2;
    const int pos = j.pos0 + 4 * kg;            // this lane's positions: pos .. pos + 3

    Packed<D> kv[2][4];                         // bf16 pairs
    unsigned int is_new = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int i = pos + t - j.first;
        const bool live = i >= 0 && i < j.n;
        is_new |= live ? 1u << t : 0u;
        const long long row = min(max(j.row0 + (live ? i : 0), 0), sp.n_rows - 1);
        kv[0][t].load(k + row * ldk + head * HD + m * D);
        kv[1][t].load(v + row * ldv + head * HD + m * D);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        kv[0][t].arrive();
        kv[1][t].arrive();
    }
    if (!usable(c, j)) {
        if (lane == 0) atomicOr(c.err, kErrBadSegment);
        return;
    }
    const bool has_old = j.first > j.pos0;
    const int in_page = j.pos0 & (T - 1);
    uint8_t* page = pages + j.page * c.page_bytes;
    uint8_t* kc = page + (long long)head * 2 * T * HD + (in_page + 4 * kg) * HD + m * D;
    uint8_t* vc = page + (long long)(head * 2 + 1) * T * HD + (in_page + 4 * kg) * HD + m * D * 4;
    uint8_t* se = page + c.scale_off + (head * (T / kBlock) + in_page / kBlock) * 2;
    const int refs = c.refs[j.page];
    unsigned int old_k[4][W] = {}, old_v[D] = {};
    unsigned int old_e = 0;
    if (has_old) {
        old_e = *reinterpret_cast<const u16*>(se);
#pragma unroll
        for (int t = 0; t < 4; ++t) load_words(kc + t * HD, old_k[t]);
        load_words(vc, old_v);
    }
    unsigned int amax[2];                       // largest magnitude of the new elements, as bf16
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        unsigned int m = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < D / 2; ++i) m = larger_halves(m, kv[x][t].w[i] & (is_new >> t & 1u ? 0x7fff7fffu : 0u));
        amax[x] = wave_max(max(m & 0xffffu, m >> 16));
    }
    bool in_range[2] = {amax[0] < kBf16Inf, amax[1] < kBf16Inf};    // wave uniform
    if (!in_range[0] || !in_range[1]) {         // the largest of the finite ones
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            unsigned int m = 0;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int d = 0; d < D; ++d) {
                    const unsigned int v = kv[x][t].w[d / 2] >> (16 * (d % 2)) & 0x7fffu;
                    m = max(m, (is_new >> t & 1u) && v < kBf16Inf ? v : 0u);
                }
            amax[x] = wave_max(m);
        }
    }
    int e[2], e_old[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        e[x] = scale_exponent(__uint_as_float(amax[x] << 16));
        in_range[x] = in_range[x] && e[x] < kLargestExponent;
        e_old[x] = has_old ? (int)(old_e >> (8 * x) & 0xffu) - 127 : e[x];
        e[x] = max(e[x], e_old[x]);
    }
    unsigned int is_old = 0;                    // positions whose codes stay (brought to the new exponent)
#pragma unroll
    for (int t = 0; t < 4; ++t) is_old |= pos + t < j.first ? 1u << t : 0u;

    const float r[2] = {block_scale((unsigned)(127 - e[0])), block_scale((unsigned)(127 - e[1]))};
    const float scale[2] = {block_scale((unsigned)(127 + e[0])), block_scale((unsigned)(127 + e[1]))};
    // the kept codes at the new exponents (positions behind the last row, which share a word of V with others, are nobody's)
    const bool again[2] = {has_old && e[0] != e_old[0], has_old && e[1] != e_old[1]};      // wave uniform
    if (again[0]) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                float f[4];
                decode4(old_k[t][i], block_scale((unsigned)(127 + e_old[0])), f);
                old_k[t][i] = encode4(f, r[0]);
            }
    }
    if (again[1]) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            float f[4];
            decode4(old_v[d], block_scale((unsigned)(127 + e_old[1])), f);
            old_v[d] = encode4(f, r[1]);
        }
    }
    if (refs != 1) {                            // a shared page
        if (lane == 0) atomicOr(c.err, kErrBadSegment);
        return;
    }
    // K: a position's codes are contiguous
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const bool fresh = is_new >> t & 1u;
        unsigned int w[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            unsigned int code;
            if (in_range[0]) code = encode4_in_range(kv[0][t].w[2 * i], kv[0][t].w[2 * i + 1], scale[0]);
            else {
                const float f[4] = {kv[0][t].at(4 * i), kv[0][t].at(4 * i + 1), kv[0][t].at(4 * i + 2), kv[0][t].at(4 * i + 3)};
                code = encode4(f, r[0]);
            }
            w[i] = fresh ? code : old_k[t][i];
        }
        if (fresh || (again[0] && (is_old >> t & 1u))) store_words(kc + t * HD, w);
    }
    // V: a word holds four positions of a column
    const unsigned int sel = (is_new & 1u ? 0xffu : 0u) | (is_new & 2u ? 0xff00u : 0u) | (is_new & 4u ? 0xff0000u : 0u) | (is_new & 8u ? 0xff000000u : 0u);
    unsigned int w[D];
    if (in_range[1]) {
#pragma unroll
        for (int d = 0; d < D; d += 2) {        // two columns: codes of two positions a word, then bytes sorted by column
            const unsigned int low = encode4_in_range(kv[1][0].w[d / 2], kv[1][1].w[d / 2], scale[1]);
            const unsigned int high = encode4_in_range(kv[1][2].w[d / 2], kv[1][3].w[d / 2], scale[1]);
            w[d] = __builtin_amdgcn_perm(high, low, 0x06040200u);
            w[d + 1] = __builtin_amdgcn_perm(high, low, 0x07050301u);
        }
    } else {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const float f[4] = {kv[1][0].at(d), kv[1][1].at(d), kv[1][2].at(d), kv[1][3].at(d)};
            w[d] = encode4(f, r[1]);
        }
    }
#pragma unroll
    for (int d = 0; d < D; ++d) w[d] = (w[d] & sel) | (old_v[d] & ~sel);
    if (is_new || (is_old && again[1])) store_words(vc, w);
    if (lane < 2) se[lane] = (uint8_t)((lane == 0 ? e[0] : e[1]) + 127);
}

template <int HD>
__global__ __launch_bounds__(256) void load_rows_kernel(CacheView c, Spans sp, const uint8_t* pages, u16* k, long long ldk,
                                                         u16* v, long long ldv, int n_items)
{
    constexpr int D = HD / 16, W = D / 4;
    const int wid = uniform((int)blockIdx.x * 4 + (int)threadIdx.x / kWave);
    const int item = wid / c.n_kv_heads, head = wid - item * c.n_kv_heads;
    if (item >= n_items) {
        report_rows(c, sp, wid - n_items * c.n_kv_heads);
        return;
    }
    BlockJob j;
    if (!find_block(c, sp, item, j)) return;
    const int lane = lane_id(), kg = lane >> 4, m = lane & 15;
    const int T = 1 << c.t_log2;
    if (!usable(c, j)) {
        if (lane == 0) atomicOr(c.err, kErrBadSegment);
        return;
    }
    const int in_page = j.pos0 & (T - 1);
    const uint8_t* page = pages + j.page * c.page_bytes;
    const uint8_t* kc = page + (long long)head * 2 * T * HD + (in_page + 4 * kg) * HD + m * D;
    const uint8_t* vc = page + (long long)(head * 2 + 1) * T * HD + (in_page + 4 * kg) * HD + m * D * 4;
    const uint8_t* se = page + c.scale_off + (head * (T / kBlock) + in_page / kBlock) * 2;
    unsigned int kw[4][W];
#pragma unroll
    for (int t = 0; t < 4; ++t) load_words(kc + t * HD, kw[t]);
    const float sk = block_scale(se[0]), sv = block_scale(se[1]);
    unsigned int vw[D];
    load_words(vc, vw);
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
        unsigned int wk[D / 2], wv[D / 2];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            float f[4];
            decode4(kw[t][w], sk, f);
            wk[2 * w] = pack_bf16x2(f[0], f[1]);
            wk[2 * w + 1] = pack_bf16x2(f[2], f[3]);
            wv[2 * w] = pack_bf16x2(vf[4 * w][t], vf[4 * w + 1][t]);
            wv[2 * w + 1] = pack_bf16x2(vf[4 * w + 2][t], vf[4 * w + 3][t]);
        }
        store_words(reinterpret_cast<uint8_t*>(ko), wk);
        store_words(reinterpret_cast<uint8_t*>(vo), wv);
    }
}

// =================================================================================================
// Page management.  The state is three integer arrays; every call is a function of them that does not depend on the order in
// which workgroups run.  First the plan: which request gets how many pages (a running sum), and which pages are free (a rank).
// Up to kSmallPages pages one workgroup does all of it in one launch; beyond, pages are counted in segments by a workgroup each beside
// the requests' plan, and a second launch hands out.  What the plan leaves (table rows, copies of pages) is the last launch's.
// Bound and measured: reserve and free by latency (a few KB): 512 requests of a page each 7.6 us of 8192 pages, 9.6 of 65536 (kernels 3.3 and
// 4.2); 400 slots freed 3.4.  A fork's and a compaction's copies by bandwidth: 132 MB of a fork in 27 us behind a plan of 5.6, 381 MB of a
// compaction in 71 behind lists of 4.7 (4.9 and 5.4 TB/s, read and written; a large copy reaches 5.1).
// =================================================================================================
constexpr int kSegPages = 4096;
// Pages up to which one workgroup does it, 1024 a round, all rounds' counts requested up front (64 requests of a page each, of 40 each: with
// 8192 pages 6.7 and 9.7 us in one launch, 7.8 and 10.9 in two; with 16000 8.3 and 11.5 against 9.0 and 11.2, and smaller pools wait
// 0.3 us longer for the loads of the larger).
constexpr int kSmallPages = 8192;
constexpr int kRefGroups = 16;          // workgroups that move the counts of a compaction's pages
constexpr int kMarkSlots = 8192;        // slots whose first mention is looked for in LDS; of more, in the workspace
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / kWave;
constexpr int kSegThreads = 256;

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

int segments_of(int n_pages) { return (n_pages + kSegPages - 1) / kSegPages; }

size_t plan_ints(int n_pages, int n_slots, int n)
{
    return (size_t)segments_of(n_pages) + 7 * (size_t)n + (size_t)n_slots + 3 * (size_t)n_pages + 4;
}

PagePlan plan_of(void* workspace, int n_pages, int n_slots, int n)
{
    PagePlan p;
    int* at = reinterpret_cast<int*>(static_cast<char*>(workspace) + kWsHeaderBytes);
    const auto take = [&](size_t k) { int* q = at; at += k; return q; };
    p.seg_free = take(segments_of(n_pages));
    p.slot = take(n); p.have = take(n); p.add = take(n); p.src = take(n); p.upto = take(n); p.page = take(n); p.from = take(n);
    p.mark = take(n_slots);
    p.list_src = take(n_pages); p.list_dst = take(n_pages); p.rank = take(n_pages);
    p.totals = take(4);
    return p;
}

__device__ __forceinline__ int wave_sum(int v) { return lane_value(wave_inclusive_scan(v), kWave - 1); }

// sum over a workgroup of WAVES waves, in every thread (slot: WAVES ints of LDS)
template <int WAVES>
__device__ __forceinline__ int block_sum(int v, int* slot)
{
    v = wave_sum(v);
    __syncthreads();
    if (lane_id() == 0) slot[threadIdx.x / kWave] = v;
    __syncthreads();
    int s = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += slot[w];
    return s;
}
// inclusive prefix sum over the workgroup; total: the whole sum.  What would pass kScanCap, summed over the waves before, stays there: 1024
// requests of all pages each do not fit 32 bits.
constexpr int kScanCap = 2 * kMaxPages;
template <int WAVES>
__device__ __forceinline__ int block_scan(int v, int* slot, int* total)
{
    static_assert((long long)kWave * (kMaxPages + 1) + 2 * (long long)kScanCap < 1ll << 31, "a wave's sum behind capped ones fits");
    const int inc = wave_inclusive_scan(v);
    __syncthreads();
    if (lane_id() == kWave - 1) slot[threadIdx.x / kWave] = inc;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < (int)threadIdx.x / kWave) before = min(before + slot[w], kScanCap);
        all = min(all + slot[w], kScanCap);
    }
    *total = all;
    return inc + before;
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

struct Requests { const int32_t* slots; const int32_t* dst; const int32_t* amount; int n; };  // dst: fork; amount: add or keep

// The requests' plan, by one workgroup of kPlanThreads.
template <bool FORK>
__device__ void plan_requests(const CacheView& c, const PagePlan& p, const Requests& rq, int* marks, int* sums)
{
    const int32_t* changed = FORK ? rq.dst : rq.slots;     // slots that the call writes
    const auto in_range = [&](int s) { return s >= 0 && s < c.n_slots; };
    // the first request that lists a slot is the one that counts
    const bool in_lds = c.n_slots <= kMarkSlots;
    for (int i = (int)threadIdx.x; i < rq.n; i += kPlanThreads) {
        const int s = changed[i];
        if (!in_range(s)) continue;
        if (in_lds) marks[s] = 0x7fffffff;
        else __hip_atomic_store(p.mark + s, 0x7fffffff, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < rq.n; i += kPlanThreads) {
        const int s = changed[i];
        if (!in_range(s)) continue;
        if (in_lds) atomicMin(marks + s, i);
        else __hip_atomic_fetch_min(p.mark + s, i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    const int T = 1 << c.t_log2;
    int base = 0;
    for (int i0 = 0; i0 < rq.n; i0 += kPlanThreads) {
        const int i = i0 + (int)threadIdx.x;
        int need = 0;
        if (i < rq.n) {
            const int s = changed[i], slot = min(max(s, 0), c.n_slots - 1);
            const int len = c.lens[slot];
            const int first = in_lds ? marks[slot] : __hip_atomic_load(p.mark + slot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            bool ok = in_range(s) && first == i;
            int have = 0, add = 0, from = -1, src = -1;
            if (FORK) {
                src = rq.slots[i];
                const int parent = min(max(src, 0), c.n_slots - 1);
                const int all = c.lens[parent];
                add = rq.amount ? rq.amount[i] : all;
                ok = ok && in_range(src) && len == 0 && all <= c.max_len && add >= 0 && add <= all;
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
        const int inc = block_scan<kPlanWaves>(need, sums, &total);
        if (i < rq.n) p.upto[i] = min(base + inc, c.n_pages + 1);
        base = min(base + total, c.n_pages + 1);
        __syncthreads();
    }
}

// Hands free page `page` of rank r (counted among the free pages) to its request; all: free pages there are.
template <bool FORK>
__device__ __forceinline__ void hand_out(const CacheView& c, const PagePlan& p, const int* upto, int n, int page, int r, int all)
{
    const int i = request_of(upto, n, r);
    if (upto[i] > all) return;                   // this request is not served
    const int mine = r - (i ? upto[i - 1] : 0);
    c.table[(long long)p.slot[i] * c.max_pages + p.have[i] + mine] = page;
    c.refs[page] = 1;
    if (FORK) p.page[i] = page;
}

// Requests that the free pages do not reach are taken out of the plan and reported; lengths of the others (reserve).
template <bool FORK>
__device__ __forceinline__ void settle(const CacheView& c, const PagePlan& p, const int* upto, int i, int all)
{
    if (upto[i] > all) {
        atomicOr(c.err, kErrNoPages);
        p.slot[i] = -1;
    } else if (!FORK && p.slot[i] >= 0) c.lens[p.slot[i]] += p.add[i];
}

// Running sums of the requests in LDS, where they are looked up (of more than kMarkSlots requests: in the workspace).
template <int THREADS>
__device__ __forceinline__ const int* keep_sums(const PagePlan& p, int n, int* lds)
{
    if (n > kMarkSlots) return p.upto;
    for (int i = (int)threadIdx.x; i < n; i += THREADS) lds[i] = p.upto[i];
    return lds;
}

// Up to kSmallPages pages: plan and hand-out by one workgroup.
template <bool FORK>
__global__ __launch_bounds__(kPlanThreads) void plan_small_kernel(CacheView c, PagePlan p, Requests rq)
{
    constexpr int ROUNDS = kSmallPages / kPlanThreads;
    __shared__ int marks[kMarkSlots];
    __shared__ int sums[kPlanWaves];
    // whether page r * 1024 + thread is free: bit r
    unsigned int is_free = 0;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int page = r * kPlanThreads + (int)threadIdx.x;
        is_free |= c.refs[min(page, c.n_pages - 1)] <= 0 && page < c.n_pages ? 1u << r : 0u;
    }
    plan_requests<FORK>(c, p, rq, marks, sums);
    const int* upto = keep_sums<kPlanThreads>(p, rq.n, marks);
    const int all = block_sum<kPlanWaves>(__popc(is_free), sums);       // (its barriers: the sums are there)
    const int wanted = upto[rq.n - 1];
    int before = 0;
    for (int r = 0; r * kPlanThreads < c.n_pages && before < wanted; ++r) {
        const bool mine = is_free >> r & 1u;
        int total;
        const int rank = before + block_scan<kPlanWaves>(mine ? 1 : 0, sums, &total) - 1;
        if (mine && rank < wanted) hand_out<FORK>(c, p, upto, rq.n, r * kPlanThreads + (int)threadIdx.x, rank, all);
        before += total;
    }
    for (int i = (int)threadIdx.x; i < rq.n; i += kPlanThreads) settle<FORK>(c, p, upto, i, all);
}

// Beyond kSmallPages, first launch: workgroup 0 plans, the others count the free pages of a segment each.
template <bool LIVE, int THREADS>
__device__ __forceinline__ void count_segment(const CacheView& c, int seg, int* seg_count, int* sums)
{
    int n = 0;
    for (int i = (int)threadIdx.x; i < kSegPages; i += THREADS) {
        const int p = seg * kSegPages + i;
        if (p < c.n_pages) n += (c.refs[p] > 0) == LIVE;
    }
    n = block_sum<THREADS / kWave>(n, sums);
    if (threadIdx.x == 0) seg_count[seg] = n;
}

template <bool FORK>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(CacheView c, PagePlan p, Requests rq)
{
    __shared__ int marks[kMarkSlots];
    __shared__ int sums[kPlanWaves];
    if (blockIdx.x > 0) count_segment<false, kPlanThreads>(c, (int)blockIdx.x - 1, p.seg_free, sums);
    else plan_requests<FORK>(c, p, rq, marks, sums);
}

// Second launch: workgroup g < segments hands out the free pages of segment g, the last one settles the requests.
template <bool FORK>
__global__ __launch_bounds__(kPlanThreads) void assign_kernel(CacheView c, PagePlan p, int n, int n_seg)
{
    constexpr int WAVES = kPlanWaves, ROUNDS = kSegPages / kPlanThreads;
    __shared__ int lds[kMarkSlots];
    __shared__ int sums[WAVES];
    int before = 0, all = 0;
    const int seg = (int)blockIdx.x;
    unsigned int is_free = 0;                   // whether page r * 1024 + thread of the segment is free: bit r
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int page = seg * kSegPages + r * kPlanThreads + (int)threadIdx.x;
        is_free |= c.refs[min(page, c.n_pages - 1)] <= 0 && page < c.n_pages ? 1u << r : 0u;
    }
    for (int s = (int)threadIdx.x; s < n_seg; s += kPlanThreads) {
        const int f = p.seg_free[s];
        all += f;
        before += s < seg ? f : 0;
    }
    const int* upto = keep_sums<kPlanThreads>(p, n, lds);
    all = block_sum<WAVES>(all, sums);
    before = block_sum<WAVES>(before, sums);
    if (seg == n_seg) {
        for (int i = (int)threadIdx.x; i < n; i += kPlanThreads) settle<FORK>(c, p, upto, i, all);
        return;
    }
    const int wanted = upto[n - 1];
    for (int r = 0; r < ROUNDS && before < wanted; ++r) {
        const bool mine = is_free >> r & 1u;
        int total;
        const int rank = before + block_scan<WAVES>(mine ? 1 : 0, sums, &total) - 1;
        if (mine && rank < wanted) hand_out<FORK>(c, p, upto, n, seg * kSegPages + r * kPlanThreads + (int)threadIdx.x, rank, all);
        before += total;
    }
}

// ---- compact: lists of the pages that move and of where they go, and every page's place in the list (-1: stays) --------
// pages in use up to `page`, itself included: upto; among the first n_live pages: low
__device__ __forceinline__ void list_page(const CacheView& c, const PagePlan& p, int page, bool live, int upto, int n_live, int low)
{
    if (page >= c.n_pages) return;
    int rank = -1;
    if (live && page >= n_live) {
        rank = upto - 1 - low;
        p.list_src[rank] = page;
    }
    if (!live && page < n_live) p.list_dst[page - upto] = page;
    p.rank[page] = rank;
}

__global__ __launch_bounds__(kPlanThreads) void list_small_kernel(CacheView c, PagePlan p)
{
    __shared__ int sums[kPlanWaves];
    int n = 0;
#pragma unroll 8
    for (int i = (int)threadIdx.x; i < c.n_pages; i += kPlanThreads) n += c.refs[i] > 0;
    const int n_live = block_sum<kPlanWaves>(n, sums);
    n = 0;
#pragma unroll 8
    for (int i = (int)threadIdx.x; i < n_live; i += kPlanThreads) n += c.refs[i] > 0;
    const int low = block_sum<kPlanWaves>(n, sums);
    if (threadIdx.x == 0) {
        p.totals[0] = n_live - low;
        p.totals[1] = n_live;
    }
    int before = 0;
    for (int p0 = 0; p0 < c.n_pages; p0 += kPlanThreads) {
        const int page = p0 + (int)threadIdx.x;
        const bool live = page < c.n_pages && c.refs[page] > 0;
        int total;
        const int upto = before + block_scan<kPlanWaves>(live ? 1 : 0, sums, &total);
        list_page(c, p, page, live, upto, n_live, low);
        before += total;
    }
}

__global__ __launch_bounds__(kSegThreads) void count_live_kernel(CacheView c, PagePlan p)
{
    __shared__ int sums[kSegThreads / kWave];
    count_segment<true, kSegThreads>(c, (int)blockIdx.x, p.seg_free, sums);
}

__global__ __launch_bounds__(kSegThreads) void list_moves_kernel(CacheView c, PagePlan p, int n_seg)
{
    constexpr int WAVES = kSegThreads / kWave;
    __shared__ int sums[WAVES];
    const int seg = (int)blockIdx.x;
    int before = 0, n_live = 0;
    for (int s = (int)threadIdx.x; s < n_seg; s += kSegThreads) {
        const int f = p.seg_free[s];
        n_live += f;
        before += s < seg ? f : 0;
    }
    n_live = block_sum<WAVES>(n_live, sums);
    before = block_sum<WAVES>(before, sums);
    // pages in use among the first n_live: whole segments by their counts, the one that n_live cuts by its refs
    const int cut = n_live / kSegPages;
    int low = 0;
    for (int s = (int)threadIdx.x; s < min(cut, n_seg); s += kSegThreads) low += p.seg_free[s];
    for (int i = cut * kSegPages + (int)threadIdx.x; i < n_live; i += kSegThreads) low += c.refs[i] > 0;
    low = block_sum<WAVES>(low, sums);
    if (seg == 0 && threadIdx.x == 0) {
        p.totals[0] = n_live - low;
        p.totals[1] = n_live;
    }
    for (int i0 = 0; i0 < kSegPages; i0 += kSegThreads) {
        const int page = seg * kSegPages + i0 + (int)threadIdx.x;
        const bool live = page < c.n_pages && c.refs[page] > 0;
        int total;
        const int upto = before + block_scan<WAVES>(live ? 1 : 0, sums, &total);
        list_page(c, p, page, live, upto, n_live, low);
        before += total;
    }
}

// ---- last launch of a fork or a compaction: state that follows the plan by the first workgroups, whole pages (in every pool, 16 KB
// a step) by the others --------------------------------------------------------------------------------------------------
constexpr int kCopyThreads = 256, kCopyBytes = 16384;

__device__ __forceinline__ void copy_piece(const uint8_t* src, uint8_t* dst, int bytes)   // a multiple of 16, at most kCopyBytes
{
    constexpr int N = kCopyBytes / (16 * kCopyThreads);
    u32x4 v[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int at = (k * kCopyThreads + (int)threadIdx.x) * 16;
        if (at < bytes) v[k] = load_once<true>(src + at);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int at = (k * kCopyThreads + (int)threadIdx.x) * 16;
        if (at < bytes) store_once<true>(dst + at, v[k]);
    }
}

// first: workgroup among the copying ones
__device__ __forceinline__ void copy_pages(const CacheView& c, const int* src, const int* dst, int n, void* const* pools, int n_pools, int first, int groups)
{
    const int pieces = (int)((c.page_bytes + kCopyBytes - 1) / kCopyBytes);
    const long long units = (long long)n * n_pools * pieces;
    for (long long u = first; u < units; u += groups) {
        const int piece = (int)(u % pieces);
        const int i = (int)(u / pieces % n), pool = (int)(u / pieces / n);
        const int from = src[i], to = dst[i];
        if (to < 0 || from < 0) continue;
        const long long at = (long long)piece * kCopyBytes;
        uint8_t* base = static_cast<uint8_t*>(pools[pool]);
        copy_piece(base + from * c.page_bytes + at, base + to * c.page_bytes + at, (int)min((long long)kCopyBytes, c.page_bytes - at));
    }
}

// n_state workgroups take the children's table rows, a wave each
__global__ __launch_bounds__(kCopyThreads) void fork_kernel(CacheView c, PagePlan p, int n, int n_state, void* const* pools, int n_pools)
{
    if ((int)blockIdx.x >= n_state) {
        copy_pages(c, p.from, p.page, n, pools, n_pools, (int)blockIdx.x - n_state, (int)gridDim.x - n_state);
        return;
    }
    const int i = (int)blockIdx.x * (kCopyThreads / kWave) + (int)threadIdx.x / kWave;
    if (i >= n || p.slot[i] < 0) return;
    const int32_t* from = c.table + (long long)p.src[i] * c.max_pages;
    int32_t* to = c.table + (long long)p.slot[i] * c.max_pages;
    for (int j = lane_id(); j < p.have[i]; j += kWave) {
        const int page = from[j];
        to[j] = page;
        if (page >= 0 && page < c.n_pages) atomicAdd(c.refs + page, 1);
        else atomicOr(c.err, kErrBadSegment);
    }
    if (lane_id() == 0) c.lens[p.slot[i]] = p.add[i];
}

// the first kRefGroups workgroups move the refs, the next n_slots take a slot's table row each
__global__ __launch_bounds__(kCopyThreads) void compact_kernel(CacheView c, PagePlan p, int32_t* n_live, void* const* pools, int n_pools)
{
    const int moves = p.totals[0], n_state = kRefGroups + c.n_slots;
    if ((int)blockIdx.x >= n_state) {
        if (moves > 0) copy_pages(c, p.list_src, p.list_dst, moves, pools, n_pools, (int)blockIdx.x - n_state, (int)gridDim.x - n_state);
        return;
    }
    if ((int)blockIdx.x < kRefGroups) {
        for (int i = (int)blockIdx.x * kCopyThreads + (int)threadIdx.x; i < moves; i += kRefGroups * kCopyThreads) {
            const int from = p.list_src[i], to = p.list_dst[i];
            c.refs[to] = c.refs[from];
            c.refs[from] = 0;
        }
        if (n_live && blockIdx.x == 0 && threadIdx.x == 0) *n_live = p.totals[1];
        return;
    }
    const int s = (int)blockIdx.x - kRefGroups;
    const int len = c.lens[s];
    if (len < 0 || len > c.max_len) {
        if (threadIdx.x == 0) atomicOr(c.err, kErrBadSegment);
        return;
    }
    const int held = (len + (1 << c.t_log2) - 1) >> c.t_log2;
    int32_t* row = c.table + (long long)s * c.max_pages;
    for (int j = (int)threadIdx.x; j < held; j += kCopyThreads) {
        const int page = row[j];
        if (page < 0 || page >= c.n_pages) {
            atomicOr(c.err, kErrBadSegment);
            continue;
        }
        const int r = p.rank[page];
        if (r >= 0) row[j] = p.list_dst[r];
    }
}

__global__ __launch_bounds__(kSegThreads) void free_kernel(CacheView c, const int32_t* slots)
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
    for (int j = (int)threadIdx.x; j < held; j += kSegThreads) {
        const int page = row[j];
        row[j] = -1;
        const bool ok = page >= 0 && page < c.n_pages;
        if (ok && atomicSub(c.refs + page, 1) > 0) continue;
        if (ok) atomicAdd(c.refs + page, 1);       // it was free already
        atomicOr(c.err, kErrBadSegment);
    }
}

lq_status launched() { return hipGetLastError() == hipSuccess ? LQ_OK : LQ_ERR_HIP; }

// what the page calls share; n = 0 requests is valid for all of them
lq_status page_call(const lq_cache* c, int32_t n, void* workspace, size_t workspace_bytes, CacheView* view)
{
    if (n < 0) return LQ_ERR_INVALID_ARG;
    const lq_status st = cache_view(c, workspace, view);
    if (st != LQ_OK) return st;
    if (n > kMaxSlots) return LQ_ERR_UNSUPPORTED;      // (workgroups of a launch)
    if (!workspace || !aligned16(workspace) || workspace_bytes < lora_cache_workspace_bytes(c, n)) return LQ_ERR_WORKSPACE;
    return LQ_OK;
}

// copying workgroups for at most `pages` pages of every pool
int copy_groups(const CacheView& c, long long pages, int n_pools)
{
    const long long units = pages * n_pools * ((c.page_bytes + kCopyBytes - 1) / kCopyBytes);
    return (int)(units < 4096 ? units : 4096);
}

// plan and hand-out; n > 0
template <bool FORK>
void plan_and_assign(const CacheView& c, const PagePlan& p, const Requests& rq, hipStream_t hs)
{
    if (c.n_pages <= kSmallPages) {
        hipLaunchKernelGGL(plan_small_kernel<FORK>, dim3(1), dim3(kPlanThreads), 0, hs, c, p, rq);
        return;
    }
    const int n_seg = segments_of(c.n_pages);
    hipLaunchKernelGGL(plan_kernel<FORK>, dim3(1 + n_seg), dim3(kPlanThreads), 0, hs, c, p, rq);
    hipLaunchKernelGGL(assign_kernel<FORK>, dim3(n_seg + 1), dim3(kPlanThreads), 0, hs, c, p, rq.n, n_seg);
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
    if (items * host_cache->n_kv_heads > kMaxRowWaves) return LQ_ERR_UNSUPPORTED;
    if (!workspace || !aligned16(workspace) || workspace_bytes < LQ_CACHE_MIN_WORKSPACE) return LQ_ERR_WORKSPACE;
    if (n_seqs == 0 || n_rows == 0) return LQ_OK;
    const Spans sp{slots, row_starts, first, n_seqs, n_rows};
    const dim3 grid((unsigned)((items * host_cache->n_kv_heads + (n_seqs + kWave - 1) / kWave + 3) / 4)), block(256);
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
    plan_and_assign<false>(c, plan_of(workspace, c.n_pages, c.n_slots, n_seqs), Requests{slots, nullptr, add, n_seqs}, static_cast<hipStream_t>(stream));
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
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    plan_and_assign<true>(c, p, Requests{src_slots, dst_slots, keep, n_seqs}, hs);
    const int waves = kCopyThreads / kWave, n_state = (n_seqs + waves - 1) / waves;
    hipLaunchKernelGGL(fork_kernel, dim3(n_state + copy_groups(c, n_seqs, n_pools)), dim3(kCopyThreads), 0, hs, c, p, n_seqs, n_state, pools, n_pools);
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
    hipLaunchKernelGGL(free_kernel, dim3(n_seqs), dim3(kSegThreads), 0, static_cast<hipStream_t>(stream), c, slots);
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
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    if (c.n_pages <= kSmallPages) hipLaunchKernelGGL(list_small_kernel, dim3(1), dim3(kPlanThreads), 0, hs, c, p);
    else {
        const int n_seg = segments_of(c.n_pages);
        hipLaunchKernelGGL(count_live_kernel, dim3(n_seg), dim3(kSegThreads), 0, hs, c, p);
        hipLaunchKernelGGL(list_moves_kernel, dim3(n_seg), dim3(kSegThreads), 0, hs, c, p, n_seg);
    }
    hipLaunchKernelGGL(compact_kernel, dim3(kRefGroups + c.n_slots + copy_groups(c, c.n_pages / 2 + 1, n_pools)), dim3(kCopyThreads), 0, hs, c, p, n_live, pools,
                       n_pools);
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
