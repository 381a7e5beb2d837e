// The paged key/value cache as the kernels see it: geometry, page layout, spans of a step's rows.  (Host checks: lq_cache.hip.)
#pragma once

#include "lq_common.h"

namespace lq {

constexpr int kBlock = LQ_CACHE_BLOCK;
constexpr int kErrNoPages = 4;
constexpr int kMaxPages = 1 << 22, kMaxSlots = 1 << 22;

struct CacheView {
    int n_kv_heads, t_log2, n_pages, n_slots, max_pages;
    int max_len;            // positions that a slot can have
    long long page_bytes;
    int scale_off;          // offset of the exponent bytes within a page
    int32_t* table; int32_t* lens; int32_t* refs;
    int* err;
};

struct Spans {
    const int32_t* slots; const int32_t* row_starts; const int32_t* first;
    int n_seqs, n_rows;
};

// status of a call's cache argument, and its view (err: the workspace's first word)
lq_status cache_view(const lq_cache* c, void* workspace, CacheView* out);
// status of the arguments that the calls on rows share
lq_status check_spans(const lq_cache* c, const void* pages, const int32_t* row_starts, const int32_t* first, int32_t n_seqs, int32_t n_rows);

struct Span { int slot, row0, n, first; };   // n <= 0: nothing to do

// span s; one that is not inside the matrices, the table or its sequence counts as empty and is reported
__device__ __forceinline__ Span load_span(const CacheView& c, const Spans& p, int s)
{
    Span u;
    u.slot = p.slots ? p.slots[s] : s;
    u.row0 = p.row_starts[s];
    const int end = p.row_starts[s + 1];
    u.first = p.first[s];
    const bool slot_ok = u.slot >= 0 && u.slot < c.n_slots;
    const int len = slot_ok ? c.lens[u.slot] : -1;
    const bool rows_ok = u.row0 >= 0 && end >= u.row0 && end <= p.n_rows;
    u.n = rows_ok ? end - u.row0 : 0;
    const bool ok = slot_ok && rows_ok && len >= 0 && len <= c.max_len && u.first >= 0 && u.first <= len && u.n <= len - u.first;
    if (!ok) {
        if (u.n || !rows_ok) atomicOr(c.err, kErrBadSegment);
        u.n = 0;
    }
    return u;
}

// The largest s with key(s) <= i, or -1; key does not decrease over 0 .. n - 1.  Every lane of the wave gets it.  Up to 256 keys are all
// looked at, in one round trip; of more, 64 a round.
template <class Key>
__device__ __forceinline__ int last_not_above(int n, int i, Key&& key)
{
    constexpr int AT_ONCE = 4;
    if (n <= AT_ONCE * kWave) {
        int k[AT_ONCE], found = 0;
#pragma unroll
        for (int r = 0; r < AT_ONCE; ++r) k[r] = key(min(r * kWave + lane_id(), n - 1));      // (no branch: the loads go out together)
#pragma unroll
        for (int r = 0; r < AT_ONCE; ++r) found += __popcll(__ballot(bool(r * kWave + lane_id() < n) & bool(k[r] <= i)));
        return found - 1;
    }
    int at = 0, width = n;      // the answer lies in [at - 1, at + width)
    while (width > 0) {
        const int step = (width + kWave - 1) / kWave;
        const int s = at + lane_id() * step;
        const bool below = s < at + width && key(s) <= i;
        const int found = __popcll(__ballot(below));
        if (found == 0) return at - 1;
        at += (found - 1) * step + 1;                  // key(at - 1) <= i
        width = min(step - 1, n - at);
    }
    return at - 1;
}

// 2^(exponent byte - 127); the bytes that are stored lie in [27, 246]
__device__ __forceinline__ float block_scale(unsigned int e) { return __uint_as_float(e << 23); }

}  // namespace lq
