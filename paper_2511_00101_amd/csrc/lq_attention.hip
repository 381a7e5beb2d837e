// Attention of a step's rows over the paged 8-bit cache.
#include "lq_cache.h"
#include "lq_internal.h"

namespace lq {
namespace {

struct AttnParams {
    CacheView c;
    Spans sp;
    const u16* q; long long ldq;
    u16* out; long long ldo;
    const uint8_t* pages;
    int n_heads, group;
    float scale;
};

// One wave per (row, head): lanes over 64 positions for the scores, over the columns for the sum.
template <int HD>
__global__ __launch_bounds__(64) void attention_kernel(AttnParams p)
{
    __shared__ float qs[HD], ps[kWave];
    const CacheView& c = p.c;
    const int lane = lane_id();
    const int row = (int)(blockIdx.x / p.n_heads), head = (int)(blockIdx.x % p.n_heads), kvh = head / p.group;
    const int s = last_not_above(p.sp.n_seqs, row, [&](int k) { return p.sp.row_starts[k]; });
    if (s < 0) return;
    const Span u = load_span(c, p.sp, s);
    if (row - u.row0 >= u.n) return;
    const int pos = u.first + row - u.row0;
    const int T = 1 << c.t_log2;
    const u16* qr = p.q + row * p.ldq + head * HD;
#pragma unroll
    for (int d = lane; d < HD; d += kWave) qs[d] = __uint_as_float((unsigned)qr[d] << 16) * p.scale;
    __syncthreads();
    float mx = -__builtin_inff(), sum = 0.f, o[HD / kWave] = {};
    const int32_t* table = c.table + (long long)u.slot * c.max_pages;
    for (int j0 = 0; j0 <= pos; j0 += kWave) {
        const int j = j0 + lane;
        float sc = -__builtin_inff();
        if (j <= pos) {
            const int page = table[j >> c.t_log2];
            if (page < 0 || page >= c.n_pages) atomicOr(c.err, kErrBadSegment);
            else {
                const uint8_t* pg = p.pages + page * c.page_bytes;
                const int in = j & (T - 1);
                const unsigned int* kc = reinterpret_cast<const unsigned int*>(pg + (long long)kvh * 2 * T * HD + in * HD);
                const float ks = block_scale(pg[c.scale_off + (kvh * (T / kBlock) + in / kBlock) * 2]);
                sc = 0.f;
                for (int i = 0; i < HD / 4; ++i) {
                    const unsigned int w = kc[i];
                    const unsigned int lo = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, ks, false));
                    const unsigned int hi = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, ks, true));
                    sc += qs[4 * i] * bf16_lo(lo) + qs[4 * i + 1] * bf16_hi(lo) + qs[4 * i + 2] * bf16_lo(hi) + qs[4 * i + 3] * bf16_hi(hi);
                }
            }
        }
        float m = sc;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, kWave));
        m = fmaxf(m, mx);
        if (m == -__builtin_inff()) m = 0.f;                       // nothing seen so far
        const float a = __expf(mx - m), e = sc == -__builtin_inff() ? 0.f : __expf(sc - m);
        mx = m;
        ps[lane] = e;
        float t = e;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) t += __shfl_xor(t, d, kWave);
        sum = sum * a + t;
        __syncthreads();
        for (int i = 0; i < HD / kWave; ++i) {
            const int d = lane + i * kWave;
            float acc = o[i] * a;
            for (int k = 0; k < kWave && j0 + k <= pos; ++k) {
                const int page = table[(j0 + k) >> c.t_log2];
                if (page < 0 || page >= c.n_pages) continue;
                const uint8_t* pg = p.pages + page * c.page_bytes;
                const int in = (j0 + k) & (T - 1);
                const float vs = block_scale(pg[c.scale_off + (kvh * (T / kBlock) + in / kBlock) * 2 + 1]);
                const unsigned int w = pg[(long long)(kvh * 2 + 1) * T * HD + (in >> 2) * 4 * HD + 4 * d + (in & 3)];
                acc += ps[k] * bf16_lo(__builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, vs, false)));
            }
            o[i] = acc;
        }
        __syncthreads();
    }
    u16* orow = p.out + row * p.ldo + head * HD;
    for (int i = 0; i < HD / kWave; ++i) orow[lane + i * kWave] = (u16)f32_to_bf16_bits(sum == 0.f ? 0.f : o[i] / sum);
}

}  // namespace
}  // namespace lq

extern "C" size_t lora_cache_attention_workspace_bytes(const lq_cache* host_cache, int32_t n_heads, int32_t max_rows)
{
    if (!host_cache || n_heads <= 0 || max_rows <= 0) return 0;
    return LQ_CACHE_MIN_WORKSPACE;
}

extern "C" lq_status lora_cache_attention(const void* q, int64_t ldq, void* out, int64_t ldo, int32_t n_rows, int32_t n_heads, float scale,
                                          const lq_cache* host_cache, const void* pages, const int32_t* slots, const int32_t* row_starts,
                                          const int32_t* first, int32_t n_seqs, int32_t max_rows, void* workspace, size_t workspace_bytes,
                                          void* stream)
{
    using namespace lq;
    AttnParams p;
    lq_status st = check_spans(host_cache, pages, row_starts, first, n_seqs, n_rows);
    if (st == LQ_OK) st = cache_view(host_cache, workspace, &p.c);
    if (st != LQ_OK) return st;
    if (n_heads <= 0 || n_heads % host_cache->n_kv_heads || max_rows <= 0) return LQ_ERR_INVALID_ARG;
    if (ldq < (int64_t)n_heads * host_cache->head_dim || ldo < (int64_t)n_heads * host_cache->head_dim) return LQ_ERR_INVALID_ARG;
    if (n_rows > 0 && (!q || !out || q == out)) return LQ_ERR_INVALID_ARG;
    if (!(scale > -__builtin_inff() && scale < __builtin_inff())) return LQ_ERR_INVALID_ARG;
    if (n_heads > LQ_CACHE_MAX_HEADS || n_seqs > LQ_CACHE_MAX_SEQS) return LQ_ERR_UNSUPPORTED;
    if ((ldq % 8) || (ldo % 8) || !aligned16(q) || !aligned16(out)) return LQ_ERR_UNSUPPORTED;
    if (!workspace || !aligned16(workspace) || workspace_bytes < lora_cache_attention_workspace_bytes(host_cache, n_heads, max_rows))
        return LQ_ERR_WORKSPACE;
    if (n_seqs == 0 || n_rows == 0) return LQ_OK;
    p.sp = Spans{slots, row_starts, first, n_seqs, n_rows};
    p.q = static_cast<const u16*>(q); p.ldq = ldq;
    p.out = static_cast<u16*>(out); p.ldo = ldo;
    p.pages = static_cast<const uint8_t*>(pages);
    p.n_heads = n_heads;
    p.group = n_heads / host_cache->n_kv_heads;
    p.scale = scale;
    const auto kernel = host_cache->head_dim == 128 ? attention_kernel<128> : attention_kernel<64>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)n_rows * (unsigned)n_heads), dim3(64), 0, static_cast<hipStream_t>(stream), p);
    return hipGetLastError() == hipSuccess ? LQ_OK : LQ_ERR_HIP;
}
