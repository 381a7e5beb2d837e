// Attention of a step's rows over the paged 8-bit cache: single tokens, drafts and prompts by one kernel.
//
// Mathematics: a row's probabilities are 2^(c s_j - m), c = scale log2(e), with a maximum m that only follows when a score exceeds it by
// more than 8 (in log2), so one pass over the positions suffices and the sums are rescaled rarely; any m gives the same quotient.
//
// Tiles: 16 x NT rows (token-major: row = token * G + query head of the group) stand as the columns of S^T = K Q^T, so the accumulator
// layout of S^T (lane: one row; registers: keys 4 kg + r of a block of 16) IS the B operand layout of O^T = V^T P^T as far as the
// order of the keys inside the k dimension goes, which is free: P never leaves its registers.  K's codes are loaded in the A operand
// layout directly (16 bytes = the lane's share of two k steps), V's layout in the page gives a lane four positions of a
// column in one word.  The codes become bf16 in registers (v_cvt_scalef32: the block's scale costs nothing; K's of head_dim 128 with four
// tiles are the operand as they are, see kCodesQ), so neither K nor V passes through LDS.  The four waves of a workgroup take alternate 32-key
// steps with maxima of their own and are added at the end.
//
// Work: units of (span, row tile, key head, chunk of positions).  Every workgroup works the unit list out from the spans (a prefix
// sum), so no plan is launched or kept; the chunk length is a workgroup's share of the batch's total work, so that long
// sequences are split where there are few rows and not where there are many.  The last chunk of a tile to arrive adds the tile's
// partial sums in chunk order.
//
// Bound and measured (8 key heads of 128 for 32 query heads unless stated):
//   256 single tokens behind up to 4096 positions  132 us, 5.6 TB/s of codes; equally long ones of 2000 161 us, 6.6 TB/s: the rate of reading
//   3 behind up to 32768, 32 key heads             47 us, 5.1 TB/s
//   48 drafts of 5 rows behind up to 3000, d 64    21 us for 51 MB: 4 us until the first unit, 8 of a chunk's steps (a memory latency each), 4 of joins
//   9 of up to 777 rows behind up to 2500          75 us, 0.62 PFLOP/s: three uneven units a workgroup, 6 us outside the steps each
//   2 of 8192 rows                                 1.02 to 1.05 ms (by card), 1.04 to 1.08 PFLOP/s where a large product reaches 1.24 to 1.27: the vector
//                                                  instructions of the softmax (63 % of the SIMDs' cycles) beside the matrix ones (49 %); with
//                                                  head_dim 64 0.72 ms, 0.76 PFLOP/s (69 % and 31 %)
//   4 single tokens of up to 60 positions, d 64    7 us with its launch: round trips (spans, lengths, pages, codes)
#include "lq_cache.h"
#include "lq_internal.h"

namespace lq {
namespace {

constexpr int kAttnThreads = 256, kAttnWaves = kAttnThreads / kWave;
constexpr int kStep = 32;                       // keys of a wave's step: two blocks
constexpr int kRound = kStep * kAttnWaves;      // keys of a workgroup's round
// Bytes of the workspace header that count the arrivals at split tiles: behind the barrier's words (kBarSub and its lines).  A counter is
// four bits where no tile has more than 15 chunks, else eight.
constexpr int kArrivals = kBarSub + kBarFan * kBarLine;
constexpr int kArrivalBytes = kWsHeaderBytes - 4 * kArrivals;
// Partial-sum slots of a call: a split tile has at least two, and its counter's number is its first slot's / 2.
template <int NT> constexpr int kSlots = NT <= 2 ? 4 * kArrivalBytes : 2 * kArrivalBytes;
constexpr int kManyChunksSlots = 2 * kArrivalBytes;    // with counters of eight bits
// Workgroups of a CU: as many as the accumulators, the codes of a step and Q leave registers for in the loop over the steps, where nothing spills.
// (Outside it four tiles of head_dim 128 keep 11 vector registers in memory, and every kernel 51 to 69 scalar ones in lanes of vector registers.)
template <int HD, int NT> constexpr int kResident = HD == 64 ? (NT == 1 ? 4 : NT == 2 ? 3 : 2) : NT == 1 ? 3 : 2;
// (us, half as long and twice as long beside it: 8 drafts of 8 rows behind up to 6000 positions 24.2, 21.0, 22.0; one token behind 3000 11.6, 12.8,
// 14.5, behind 30000 25.7, 23.2, 21.8)
constexpr int kLeastChunk = 4 * kRound;
// Positions that take as long as the stores, arrivals and sums of a split (30 drafts of 8 rows behind 1500 positions: 31 us in two
// chunks each, 25 in one).
template <int NT> constexpr int kSplitCost = NT == 1 ? 4 * kRound : 8 * kRound;
constexpr int kAloneLongest = kLeastChunk;      // (not split, then)
constexpr int kClasses = 5;
__host__ __device__ constexpr int span_at(int n) { return (3 * n + 1 + 3) / 4 * 4; }
// Spans that a workgroup keeps in LDS (16 bytes each, beside the 12 that every span takes there); of more, a unit's is read again.  With one row tile some 690
// spans (head_dim 64: 820) take the room of a workgroup, which costs less than reading them again would (1000 of up to 600 positions 98 us against
// 100 and, with head_dim 64, 57 against 65); with four it would be one of two.
template <int NT> constexpr int kKeptSpans = NT < 4 ? 1024 : 256;
constexpr int kLdsBytes = 160 * 1024, kLdsGranule = 1280;       // of a compute unit; what a workgroup gets is a multiple
constexpr float kNone = -3e38f;                 // a maximum before anything was seen: below every score, and finite (no case of its own anywhere)
constexpr float kLazy = 8.f;                    // log2 of how far a score may exceed the maximum that its exponentials use
constexpr int kAllButOrder = 0x4;              // what the scheduler may move across: scalar arithmetic
constexpr int kRawBuffer = 0x00020000, kSc1 = 16;   // descriptor word 3 (raw 32-bit data); device-scope cache policy

struct AttnParams {
    CacheView c;
    Spans sp;
    const u16* q; long long ldq;
    u16* out; long long ldo;
    const uint8_t* pages;
    int group;
    unsigned int group_magic;   // ceil(2^20 / group): x / group = x * magic >> 20 for x below 2^20 / group
    float c_log2;               // |scale| * log2(e)
    unsigned int q_sign;        // 0x80008000 where the scale is negative
    float* partial;
    unsigned int partial_bytes;
    int* tickets;
    uint8_t* arrivals;
};

template <int HD, int NT> constexpr int slot_floats() { return 16 * NT * (HD + 2); }

// Codes of a step: per block of 16 keys K in the A operand layout, V in words of four positions, and the two exponent bytes.
template <int HD>
struct Step {
    u32x4 k[2][HD / 64], v[2][HD / 64];
    unsigned int e[2];
    bool ok[2];                 // wave uniform: the block's page can be used
};
template <int HD>
struct Where { const uint8_t* k[2]; const uint8_t* e[2]; bool ok[2]; };   // wave uniform

__device__ __forceinline__ unsigned int to_bf16(unsigned int w, float scale, bool high)
{
    return __builtin_bit_cast(unsigned int, high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true)
                                                 : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
}
__device__ __forceinline__ bf16x8 eight_bf16(unsigned int a, float sa, unsigned int b, float sb)
{
    return __builtin_bit_cast(bf16x8, u32x4{to_bf16(a, sa, false), to_bf16(a, sa, true), to_bf16(b, sb, false), to_bf16(b, sb, true)});
}
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Two bf16 values with an infinity made NaN: its row's scores may all be minus infinity, which a sum of exponentials does not tell from
// a row that sees nothing.
__device__ __forceinline__ unsigned int no_infinities(unsigned int w)
{
    return w | (((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 9;
}

// all ones where a row that sees positions up to `limit` does not see `key` (in integers: comparisons would hold a mask
// register pair per element)
__device__ __forceinline__ unsigned int hidden(int limit, int key, bool ok) { return (unsigned int)(((ok ? limit : -1) - key) >> 31); }
// bits of `a` where mask is set, of v elsewhere
__device__ __forceinline__ float select_bits(unsigned int mask, unsigned int a, float v)
{
    return __uint_as_float((mask & a) | (~mask & __float_as_uint(v)));
}

// maximum (sum) over the four lanes that hold one column
__device__ __forceinline__ float column_max(float v)
{
    typedef __attribute__((ext_vector_type(2))) unsigned int pair;
    const unsigned int u = __float_as_uint(v);
    const pair a = __builtin_bit_cast(pair, __builtin_amdgcn_permlane16_swap(u, u, false, false));
    const unsigned int w = __float_as_uint(fmaxf(__uint_as_float(a.x), __uint_as_float(a.y)));
    const pair b = __builtin_bit_cast(pair, __builtin_amdgcn_permlane32_swap(w, w, false, false));
    return fmaxf(__uint_as_float(b.x), __uint_as_float(b.y));
}
__device__ __forceinline__ float column_sum(float v)
{
    v += __shfl_xor(v, 16, kWave);
    return v + __shfl_xor(v, 32, kWave);
}

// page numbers of a slot's row, 64 entries in the lanes and the next 64 behind them
struct PageIds {
    const int32_t* row;
    int held, batch;
    int now, next;
    __device__ __forceinline__ int load(int b) const { return row[min(b * kWave + lane_id(), held - 1)]; }
    __device__ __forceinline__ void start(const int32_t* r, int n, int entry)
    {
        row = r;
        held = n;
        batch = entry / kWave;
        now = load(batch);
        next = load(batch + 1);
    }
    // makes `entry` (wave uniform) one of the lanes'; entries are asked for in order
    __device__ __forceinline__ void reach(int entry)
    {
        if (entry / kWave != batch) {
            now = next;
            batch = entry / kWave;
            next = load(batch + 1);
        }
    }
    __device__ __forceinline__ int get(int entry) const { return lane_value(now, entry % kWave); }
};

struct Unit { int slot, row0, n, first, tile, head, chunk, chunks, slot0, bits; };   // slot0: first partial-sum slot of the tile; bits: of a counter

template <int HD, int NT>
struct Attention {
    static constexpr int D = HD / 16;           // O^T rows of a lane's accumulator register set; also V words of a lane and block
    static constexpr int LD = HD / 64;          // 16-byte loads of a lane for 16 keys
    static constexpr int PITCH = HD + 4;
    static constexpr int kHalfD = 4, kHalves = D / kHalfD;
    // Few rows: the codes are read once and bound the kernel.  Every load takes whole 128-byte lines, past the caches (256 tokens behind up to
    // 4096 positions 130 us, with plain loads 143; prompts, whose tiles read the same codes, the other way round: 1167 and 1097).
    static constexpr bool kStream = NT < 4;
    // head_dim 128: a load of K takes eight whole rows (lanes m < 8 of 16 the lower halves, the others the upper ones)
    static constexpr bool kWholeRows = kStream && LD == 2;
    static constexpr bool kSharedQ = NT >= 4;   // Q's fragments in LDS (the waves have the same rows): 64 registers less, without which the sums spill
    // Prompts with head_dim 128: K's codes are the operand themselves, with their block's exponent as the matrix instruction's scale, and Q is the sum
    // of rows of codes: q = 2^e (high + low 2^-11 + last 2^-22), one e a row, high and last in e4m3, low in e5m2.  Of a bf16 value's
    // eight bits high takes four and low the other three (a nearest one's remainder has a sign); where the row's largest element is more than 2^14
    // times larger, high loses bits, and last has what low cannot hold: the sum is exact down to 2^-31 of the largest element, and off by at most
    // 2^-39 of it below (and of 2^-97 in rows that are smaller).  Last is multiplied only for row tiles that have one (of Gaussian rows one of eleven; 1.7 % of the
    // time of two 8192-row prompts).  Two 16 x 16 x 128 products take what four bf16 ones take, without the conversion of K (two prompts of 8192 rows 1137 us
    // against 1241 when it was brought in).  With head_dim 64 one product of the depth 128 would hold both parts, but K's duplicated halves have to be
    // exchanged between lanes, as many instructions as the conversion.
    static constexpr bool kCodesQ = kSharedQ && HD == 128;
    struct Shared {
        union {
            float acc[NT < kAttnWaves ? kAttnWaves : 1][16][PITCH];
            struct {
                u32x4 q[NT][kCodesQ ? 6 : HD / 32][kWave];      // fragments: of bf16 values; or of codes, high, low and last parts
                uint8_t q_exp[16][4];
                uint8_t q_last[4];              // whether the row tile has last parts that are not zero
            };
            float sums_of_groups[NT < kAttnWaves ? NT * kAttnThreads * (D + 2) : 1];    // of a split tile's rows
            f32x4 part[NT < kAttnWaves ? 1 : kAttnWaves][NT][kHalfD][kWave];     // every wave's sums of 64 columns, as its registers hold them
        };
        float m[kAttnWaves][16 * NT], l[kAttnWaves][16 * NT];
        long long sums[kAttnWaves];
        unsigned int tiles[kAttnWaves];
        int longest[kAttnWaves], scan[kAttnWaves][2], classes[kAttnWaves][kClasses];
        int slot[2], last;
    };

    // The addresses of a step's two blocks (their entries lie in one batch: a step begins at a multiple of 32 positions).  A block that is
    // not there gets page 0's: what is read is not used.  bad: whether a position that a row sees has no usable page.
    struct Head { const uint8_t* k; const uint8_t* e; unsigned int page_bytes, n_pages; int t_log2; };   // of page 0: the unit's key head
    static __device__ __forceinline__ Where<HD> find_step(const Head& hd, PageIds& ids, int key0, int last_key, bool& bad)
    {
        Where<HD> w;
        ids.reach(key0 >> hd.t_log2);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int key = key0 + b * kBlock;
            const unsigned int in = (unsigned)key & ((1u << hd.t_log2) - 1u);
            const unsigned int page = (unsigned)ids.get(min(key, last_key) >> hd.t_log2);
            const bool usable = page < hd.n_pages;
            bad = bad || !usable;
            w.ok[b] = usable && key <= last_key;
            const unsigned long long at = (unsigned long long)(usable ? page : 0u) * hd.page_bytes;
            w.k[b] = hd.k + (at + in * HD);
            w.e[b] = hd.e + (at + in / kBlock * 2);
        }
        return w;
    }
    static __device__ __forceinline__ void load_k(const Where<HD>& w, Step<HD>& s)
    {
        const unsigned int lane = lane_id();
        const unsigned int off = kWholeRows ? (lane & 7) * HD + (lane >> 3 & 1) * 64 + (lane >> 4) * 16 : (lane & 15) * HD + (lane >> 4) * 16;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            s.ok[b] = w.ok[b];
            s.e[b] = *reinterpret_cast<const u16*>(w.e[b]);
#pragma unroll
            for (int j = 0; j < LD; ++j) s.k[b][j] = load_once<kStream>(w.k[b] + off + (kWholeRows ? 8 * HD : 64) * j);
        }
    }
    // K of a block in the A operand layout: lane (m, kg), key m, word group j its codes 64 j + 16 kg .. + 15.  Lanes m and m + 8 swap what
    // they loaded for each other where a load took eight whole rows.
    static __device__ __forceinline__ void operand_k(const u32x4 (&loaded)[LD], u32x4 (&k)[LD])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (kWholeRows) {
                k[0][i] = __builtin_amdgcn_update_dpp((int)loaded[0][i], (int)loaded[1][i], 0x128, 0xf, 0xc, false);   // row_ror:8
                k[1][i] = __builtin_amdgcn_update_dpp((int)loaded[1][i], (int)loaded[0][i], 0x128, 0xf, 0x3, false);
            } else {
#pragma unroll
                for (int j = 0; j < LD; ++j) k[j][i] = loaded[j][i];
            }
        }
    }
    static __device__ __forceinline__ void load_v(const AttnParams& p, const Where<HD>& w, Step<HD>& s)
    {
        const unsigned int lane = lane_id(), off = (lane >> 4) * 4 * HD + (lane & 15) * 16;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < LD; ++j) s.v[b][j] = load_once<kStream>(w.k[b] + ((unsigned)HD << p.c.t_log2) + off + 256 * j);
    }

    // One unit's chunk: the wave's share of the positions [begin, end).
    struct State { f32x4 o[NT][D]; float m[NT], l[NT]; };

    struct Scores { f32x4 s[2][NT]; };
    static constexpr bool kAlone = NT == 1;     // a unit per wave is offered
    typedef __attribute__((ext_vector_type(8))) int i32x8;
    static constexpr int kAhead = 3;
    static constexpr int kLowExp = 11, kLastExp = 22;

    // two values' high parts, low parts, and what those leave (times 2^kLastExp)
    static __device__ __forceinline__ unsigned int split2(const float* x, float r, unsigned int& low, float (&left)[2])
    {
        const float a[2] = {x[0] * r, x[1] * r};
        const unsigned int high = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(a[0], a[1], 0, false) & 0xffffu;
        const f32x2 back = __builtin_amdgcn_cvt_pk_f32_fp8((int)high, false);
#pragma unroll
        for (int k = 0; k < 2; ++k) left[k] = (a[k] - back[k]) * (1 << kLowExp);
        low = (unsigned)__builtin_amdgcn_cvt_pk_bf8_f32(left[0], left[1], 0, false) & 0xffffu;
        const f32x2 low_back = __builtin_amdgcn_cvt_pk_f32_bf8((int)low, false);
#pragma unroll
        for (int k = 0; k < 2; ++k) left[k] = (left[k] - low_back[k]) * (1 << (kLastExp - kLowExp));
        return high;
    }
    // The row tile's fragments into LDS; w: the lane's share of its row
    static __device__ __forceinline__ void split_q(const u32x4 (&w)[4], Shared& sh, int n)
    {
        const int lane = lane_id();
        float x[32], amax = 0.f, any = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack8(w[i], x + 8 * i);
#pragma unroll
        for (int i = 0; i < 32; ++i) amax = fmaxf(amax, fabsf(x[i]));
        amax = column_max(amax);
        const unsigned int u = __float_as_uint(fminf(amax, 3.4e38f));
        const int e = max((int)(u >> 23) - 127 - ((u & 0x7fffffu) <= 0x600000u ? 8 : 7), kLastExp - 127);     // least with amax <= 448 * 2^e
        const float r = __uint_as_float((unsigned)(127 - e) << 23);
        if (lane < 16) sh.q_exp[lane][n] = (uint8_t)(e + 127);         // E8M0, of the high parts; the others' are kLowExp and kLastExp less
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            u32x4 high, low;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                unsigned int lo[2], hi[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float left[2];
                    hi[h] = split2(x + 16 * g + 4 * i + 2 * h, r, lo[h], left);
                    any = fmaxf(any, fmaxf(fabsf(left[0]), fabsf(left[1])));       // (a NaN's high and low parts are NaN: the last one may be anything)
                }
                high[i] = hi[0] | hi[1] << 16;
                low[i] = lo[0] | lo[1] << 16;
            }
            sh.q[n][g][lane] = high;
            sh.q[n][2 + g][lane] = low;
        }
        const bool last = __any(any > 0.f);
        if (lane == 0) sh.q_last[n] = last;
        if (!last) return;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            u32x4 part;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                unsigned int la[2], lo;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float left[2];
                    split2(x + 16 * g + 4 * i + 2 * h, r, lo, left);
                    la[h] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(left[0], left[1], 0, false) & 0xffffu;
                }
                part[i] = la[0] | la[1] << 16;
            }
            sh.q[n][4 + g][lane] = part;
        }
    }

    // n: the byte of qe that holds the exponents of row tile n (a constant once the loops are unrolled); FORMAT of b: 0 e4m3, 1 e5m2
    template <int FORMAT>
    static __device__ __forceinline__ f32x4 mfma_codes(int n, i32x8 a, i32x8 b, f32x4 c, int ke, int qe)
    {
        return n == 0   ? __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, FORMAT, 0, ke, 0, qe)
               : n == 1 ? __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, FORMAT, 0, ke, 1, qe)
               : n == 2 ? __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, FORMAT, 0, ke, 2, qe)
                        : __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, FORMAT, 0, ke, 3, qe);
    }

    // with kCodesQ: q_exp the exponents of the lane's row in the row tiles, a byte each; q_last a byte of 1 for each tile with last parts
    static __device__ __forceinline__ void scores(const Step<HD>& s, const bf16x8 (&q)[kSharedQ ? 1 : NT][HD / 32], int q_exp, int q_last, const Shared& sh,
                                                  Scores& sc)
    {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int n = 0; n < NT; ++n) sc.s[b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (kSharedQ) asm volatile("" ::: "memory");   // (read again every step: kept in registers, Q would displace the sums)
        const float k0 = block_scale(uniform((int)s.e[0]) & 0xffu), k1 = block_scale(uniform((int)s.e[1]) & 0xffu);
        u32x4 k[2][LD];
        operand_k(s.k[0], k[0]);
        operand_k(s.k[1], k[1]);
        if constexpr (kCodesQ) {
            i32x8 a[2];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 8; ++i) a[b][i] = (int)k[b][i / 4][i % 4];
            const int e0 = uniform((int)s.e[0]) & 0xff, e1 = uniform((int)s.e[1]) & 0xff;
            const int low_exp = q_exp - 0x01010101 * kLowExp;
            const auto parts = [&](int n, int which) {      // of row tile n: its high parts, its low parts, its last ones
                const u32x4 x = sh.q[n][which * 2][lane_id()], y = sh.q[n][which * 2 + 1][lane_id()];
                return i32x8{(int)x.x, (int)x.y, (int)x.z, (int)x.w, (int)y.x, (int)y.y, (int)y.z, (int)y.w};
            };
            const auto fragment = [&](int i) { return parts(i / 2, i % 2); };
            // kAhead fragments on their way while a pair of products runs (in this order: left to the scheduler, the reads are either all in
            // front, which takes registers that spill, or each is waited for)
            i32x8 f[kAhead + 1];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) f[i] = fragment(i);
#pragma unroll
            for (int i = 0; i < 2 * NT; ++i) {
                if (i + kAhead < 2 * NT) f[(i + kAhead) % (kAhead + 1)] = fragment(i + kAhead);
                __builtin_amdgcn_sched_barrier(0);
                if (i % 2 == 0) {
                    sc.s[0][i / 2] = mfma_codes<0>(i / 2, a[0], f[i % (kAhead + 1)], sc.s[0][i / 2], e0, q_exp);
                    sc.s[1][i / 2] = mfma_codes<0>(i / 2, a[1], f[i % (kAhead + 1)], sc.s[1][i / 2], e1, q_exp);
                } else {
                    sc.s[0][i / 2] = mfma_codes<1>(i / 2, a[0], f[i % (kAhead + 1)], sc.s[0][i / 2], e0, low_exp);
                    sc.s[1][i / 2] = mfma_codes<1>(i / 2, a[1], f[i % (kAhead + 1)], sc.s[1][i / 2], e1, low_exp);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // (a loop over the marked tiles, not a test for each: 2 prompts of 8192 rows 1018 us against 1023, 32 of 512 behind 2560 773 against 789)
            const int last_exp = q_exp - 0x01010101 * kLastExp;
            for (int left = q_last; left; left &= left - 1) {
                const int tile = __builtin_ctz(left) / 8;
                const i32x8 part = parts(tile, 2);
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    if (n == tile) {
                        sc.s[0][n] = mfma_codes<0>(n, a[0], part, sc.s[0][n], e0, last_exp);
                        sc.s[1][n] = mfma_codes<0>(n, a[1], part, sc.s[1][n], e1, last_exp);
                    }
            }
            return;
        }
        bf16x8 a[2][HD / 32];
#pragma unroll
        for (int j = 0; j < LD; ++j) {
            a[0][2 * j] = eight_bf16(k[0][j].x, k0, k[0][j].y, k0);
            a[1][2 * j] = eight_bf16(k[1][j].x, k1, k[1][j].y, k1);
            a[0][2 * j + 1] = eight_bf16(k[0][j].z, k0, k[0][j].w, k0);
            a[1][2 * j + 1] = eight_bf16(k[1][j].z, k1, k[1][j].w, k1);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int g = 0; g < HD / 32; ++g) {
                bf16x8 qf;
                if constexpr (kSharedQ) qf = __builtin_bit_cast(bf16x8, sh.q[n][g][lane_id()]);
                else qf = q[n][g];
                sc.s[0][n] = mfma(a[0][g], qf, sc.s[0][n]);
                sc.s[1][n] = mfma(a[1][g], qf, sc.s[1][n]);
            }
        pace<3>();
    }

    // Fragments of Q from LDS: the first AHEAD on their way before the first products, then as many reads as a pair of products needs behind it
    // (left alone, the reads are either all in front, which takes registers that spill, or each waited for).
    template <int AHEAD>
    static __device__ __forceinline__ void pace()
    {
        if constexpr (kSharedQ) {
            constexpr int PAIRS = NT * HD / 32;                                     // pairs of products
            __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);                  // LDS reads
#pragma unroll
            for (int i = 0; i < PAIRS - AHEAD; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);                    // matrix products
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x8, 2 * AHEAD, 0);
        }
    }

    // The rows of a tile: row row_base + x is query head y % group of token token0 + y / group, y = within0 + x.
    struct Rows {
        int token0, within0, left, first, group;    // left: rows from row_base on
        unsigned int magic;
        __device__ __forceinline__ int token(int x) const { return token0 + (int)(((unsigned)(within0 + x) * magic) >> 20); }
        __device__ __forceinline__ int query(int x) const { return within0 + x - (token(x) - token0) * group; }
        // the last position that the lane's rows see; -1: no row
        __device__ __forceinline__ void limits(int (&limit)[NT]) const
        {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int x = 16 * n + (lane_id() & 15);
                limit[n] = x < left ? first + token(x) : -1;
            }
        }
    };

    // probabilities of a step, and its share of O^T
    // request() is called halfway, when half of the scores' registers are free; with one row tile at once
    template <class Request>
    static __device__ __forceinline__ void accumulate(Request&& request, const u32x4 (&v)[2][LD], bool ok0, bool ok1, Scores& scores, const unsigned int (&e)[2],
                                                      const Rows& rows, int key0, int last_key, bool masked, float c_log2, State& st)
    {
        if (NT == 1) request();
        const bool ok[2] = {ok0, ok1};
        const int kg = lane_id() >> 4;
        f32x4 (&sc)[2][NT] = scores.s;
        unsigned int vw[2][D];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < D; ++i) vw[b][i] = v[b][i / 4][i % 4];
        if (masked) {
            asm volatile("" ::: "memory");      // (a branch: selected without one, every step would pay for it)
            int limit[NT];
            rows.limits(limit);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int key = key0 + b * kBlock + 4 * kg;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        sc[b][n][r] = select_bits(hidden(limit[n], key + r, ok[b]), 0xff800000u, sc[b][n][r]);   // -infinity
                // what lies in the page behind the last position that any row sees is nobody's
                const int live = last_key + 1 - key;
                const unsigned int keep = !ok[b] || live <= 0 ? 0u : live >= 4 ? ~0u : (1u << (8 * live)) - 1u;
#pragma unroll
                for (int i = 0; i < D; ++i) vw[b][i] &= keep;
            }
        }
        // Only a score that exceeds its row's maximum by more than kLazy changes the maximum: every lane looks at its own, and the
        // columns' maxima are worked out when one does.
        float top[NT];
        bool grows = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            top[n] = sc[0][n][0];
#pragma unroll
            for (int r = 1; r < 8; ++r) top[n] = fmaxf(top[n], sc[r / 4][n][r % 4]);
            grows = grows || __builtin_fmaf(top[n], c_log2, -kLazy) > st.m[n];
        }
        if (__any(grows)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float m = fmaxf(st.m[n], column_max(top[n]) * c_log2);
                const float a = __builtin_amdgcn_exp2f(st.m[n] - m);
                st.m[n] = m;
                st.l[n] *= a;
#pragma unroll
                for (int i = 0; i < D; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) st.o[n][i][r] *= a;
            }
        }
        if (masked) {
            asm volatile("" ::: "memory");
            // 0 x NaN is NaN: a NaN value must reach the rows that see its position and no others
            unsigned int nan = 0;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < D; ++i) nan |= ((vw[b][i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            if (__any(nan != 0)) {
                unsigned int seen[NT][4];
                int limit[NT];
                rows.limits(limit);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int key = key0 + (r / 2) * kBlock + 4 * kg + 2 * (r % 2);
                        seen[n][r] = (~hidden(limit[n], key, ok[r / 2]) & 0x3f80u) | (~hidden(limit[n], key + 1, ok[r / 2]) & 0x3f800000u);
                    }
#pragma unroll
                for (int i = 0; i < D; ++i) {
                    unsigned int one[2];
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const unsigned int bad = (((vw[b][i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;   // 1 per NaN byte
                        one[b] = bad * 0x38u;                                                                      // e4m3 1.0
                        vw[b][i] &= ~(bad * 0xffu);
                    }
                    const bf16x8 a = eight_bf16(one[0], 1.f, one[1], 1.f);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const f32x4 hit = mfma(a, __builtin_bit_cast(bf16x8, u32x4{seen[n][0], seen[n][1], seen[n][2], seen[n][3]}), f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            st.o[n][i][r] = select_bits((unsigned int)(-(int)__float_as_uint(hit[r]) >> 31), 0x7fc00000u, st.o[n][i][r]);   // a count
                    }
                }
            }
        }
        const float v0 = ok[0] ? block_scale((unsigned)uniform((int)e[0]) >> 8) : 1.f, v1 = ok[1] ? block_scale((unsigned)uniform((int)e[1]) >> 8) : 1.f;
        bf16x8 vt[D];
#pragma unroll
        for (int i = 0; i < D; ++i) vt[i] = eight_bf16(vw[0][i], v0, vw[1][i], v1);
        // Row tile by row tile, the products of one between the exponentials of the next, in this order: a product occupies its unit
        // for four vector instructions' time, and left alone the scheduler puts the products, and the exponentials, in a row.
        constexpr int PER = 8 / D;                  // exponentials between two products
        float x[2][8], sum[2];
        u32x4 pt[2];
        const auto exponential = [&](int n, int r) { x[n % 2][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r / 4][n][r % 4], c_log2, -st.m[n])); };
        // (bf16 probabilities: rounded, 2^-9 of a term on average in the sum of p v, below the output's own rounding)
        const auto pack = [&](int n, int r) { pt[n % 2][r / 2] = pack_bf16x2(x[n % 2][r], x[n % 2][r + 1]); };
        const auto add = [&](int n, int r) { sum[n % 2] = r == 0 ? x[n % 2][0] : sum[n % 2] + x[n % 2][r]; };
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            exponential(0, r);
            if (r % 2) pack(0, r - 1);
            add(0, r);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            st.l[n] += sum[n % 2];
            const bf16x8 p = __builtin_bit_cast(bf16x8, pt[n % 2]);
#pragma unroll
            for (int i = 0; i < D; ++i) {
                st.o[n][i] = mfma(vt[i], p, st.o[n][i]);
                if (n + 1 < NT) {
#pragma unroll
                    for (int r = i * PER; r < (i + 1) * PER; ++r) {
                        exponential(n + 1, r);
                        if (r > 0) add(n + 1, r - 1);
                        if (r > 1 && r % 2 == 0) pack(n + 1, r - 2);
                    }
                    __builtin_amdgcn_sched_barrier(kAllButOrder);
                }
            }
            if (n + 1 < NT) {
                add(n + 1, 7);
                pack(n + 1, 6);
            }
            if (NT > 1 && n == NT / 2 - 1) request();
        }
    }

    // Sums of D columns of a row over some of its positions, the maximum that they were taken with, and the exponentials' sum.
    struct Sums {
        float m = kNone, l = 0.f, o[D] = {};
        __device__ __forceinline__ void add(const Sums& x)
        {
            const float top = fmaxf(m, x.m), a = __builtin_amdgcn_exp2f(m - top), b = __builtin_amdgcn_exp2f(x.m - top);
            m = top;
            l = l * a + x.l * b;
#pragma unroll
            for (int i = 0; i < D; ++i) o[i] = o[i] * a + x.o[i] * b;
        }
    };

    // whether all other chunks of the unit's tile have left their sums
    static __device__ __forceinline__ bool last_to_arrive(const AttnParams& p, const Unit& u, Shared& sh)
    {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) {
            const int i = u.slot0 / 2 * u.bits, shift = i % 32;
            int* word = reinterpret_cast<int*>(p.arrivals) + i / 32;
            const int old = __hip_atomic_fetch_add(word, 1 << shift, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const bool last = ((old >> shift) & ((1 << u.bits) - 1)) == u.chunks - 1;
            if (last) __hip_atomic_fetch_sub(word, (int)((unsigned)u.chunks << shift), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            sh.last = last;
        }
        __syncthreads();
        const bool last = sh.last;
        asm volatile("" ::: "memory");
        return last;
    }

    // As many row tiles as waves: wave n adds up tile n, 64 columns at a time, in the layout of the accumulators (whole 1 KB accesses, also of a
    // split tile's partial sums), and writes it from its registers.  (Maxima and sums of the rows are in LDS, behind a barrier.)  Tile after
    // tile by all waves, with every row's columns dealt to 16 threads, took twice the barriers and read a split tile's sums one tile after
    // the other: 8 prompts of 512 rows 61 us against 57, 64 rows behind 3000 positions 35 against 24.
    static __device__ __forceinline__ void join_by_tiles(const AttnParams& p, const Unit& u, const Rows& tr, int wave, bool split, const State& st, Shared& sh)
    {
        const int lane = lane_id(), col = lane & 15, kg = lane >> 4, row = 16 * wave + col;
        const __amdgpu_buffer_rsrc_t part = __builtin_amdgcn_make_buffer_rsrc(p.partial, 0, (int)p.partial_bytes, kRawBuffer);
        const int slot_bytes = slot_floats<HD, NT>() * 4, stat_at = 16 * NT * HD * 4 + row * 8;
        float a[NT], m = sh.m[0][row], l = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float top = sh.m[0][16 * n + col];
#pragma unroll
            for (int w = 1; w < kAttnWaves; ++w) top = fmaxf(top, sh.m[w][16 * n + col]);
            a[n] = __builtin_amdgcn_exp2f(st.m[n] - top);
        }
#pragma unroll
        for (int w = 1; w < kAttnWaves; ++w) m = fmaxf(m, sh.m[w][row]);
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) l += sh.l[w][row] * __builtin_amdgcn_exp2f(sh.m[w][row] - m);
        float inv = l == 0.f ? 0.f : 1.f / l;
        const bool live = row < tr.left;
        const int token = tr.token(row), h = u.head * p.group + tr.query(row);
        u16* dst = p.out + (long long)(u.row0 + token) * p.ldo + h * HD + 16 * kg;
        const auto write = [&](int half, const f32x4 (&o)[kHalfD]) {
#pragma unroll
            for (int i = 0; i < kHalfD; i += 4)      // 16 columns of the lane
#pragma unroll
                for (int r = 0; r < 4; r += 2)
                    *reinterpret_cast<u32x4*>(dst + 16 * (half * kHalfD + i) + 4 * r) =
                        u32x4{pack_bf16x2(o[i][r] * inv, o[i + 1][r] * inv), pack_bf16x2(o[i + 2][r] * inv, o[i + 3][r] * inv),
                              pack_bf16x2(o[i][r + 1] * inv, o[i + 1][r + 1] * inv), pack_bf16x2(o[i + 2][r + 1] * inv, o[i + 3][r + 1] * inv)};
        };
#pragma unroll
        for (int half = 0; half < kHalves; ++half) {
            if (half) __syncthreads();
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < kHalfD; ++i) sh.part[wave][n][i][lane] = st.o[n][half * kHalfD + i] * a[n];
            __syncthreads();
            f32x4 o[kHalfD];
#pragma unroll
            for (int i = 0; i < kHalfD; ++i) {
                o[i] = sh.part[0][wave][i][lane];
#pragma unroll
                for (int w = 1; w < kAttnWaves; ++w) o[i] += sh.part[w][wave][i][lane];
            }
            if (!split) {
                if (live) write(half, o);
            } else {
#pragma unroll
                for (int i = 0; i < kHalfD; ++i)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o[i]), part, ((wave * D + half * kHalfD + i) * kWave + lane) * 16,
                                                           (u.slot0 + u.chunk) * slot_bytes, kSc1);
            }
        }
        if (!split) return;
        if (kg == 0) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, f32x2{m, l}), part, stat_at, (u.slot0 + u.chunk) * slot_bytes, kSc1);
        if (!last_to_arrive(p, u, sh)) return;
        if (16 * wave >= tr.left) return;
        const auto stat = [&](int k) { return __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(part, stat_at, (u.slot0 + k) * slot_bytes, kSc1)); };
        m = kNone;
#pragma unroll 4
        for (int k = 0; k < u.chunks; ++k) m = fmaxf(m, stat(k).x);
        l = 0.f;
        f32x4 o[D];
#pragma unroll
        for (int i = 0; i < D; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
        for (int k = 0; k < u.chunks; ++k) {
            const f32x2 ml = stat(k);
            f32x4 v[D];
#pragma unroll
            for (int i = 0; i < D; ++i)
                v[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(part, ((wave * D + i) * kWave + lane) * 16, (u.slot0 + k) * slot_bytes, kSc1));
            const float f = __builtin_amdgcn_exp2f(ml.x - m);
            l += ml.y * f;
#pragma unroll
            for (int i = 0; i < D; ++i) o[i] += v[i] * f;
        }
        inv = l == 0.f ? 0.f : 1.f / l;
        if (!live) return;
#pragma unroll
        for (int half = 0; half < kHalves; ++half) {
            f32x4 x[kHalfD];
#pragma unroll
            for (int i = 0; i < kHalfD; ++i) x[i] = o[half * kHalfD + i];
            write(half, x);
        }
    }

    // ALONE: the wave has the unit to itself (no other wave of the workgroup may be waited for)
    template <bool ALONE>
    static __device__ __forceinline__ void run_unit(const AttnParams& p, const Unit& u, int chunk_len, Shared& sh)
    {
        const CacheView& c = p.c;
        const int lane = lane_id(), wave = uniform((int)threadIdx.x / kWave), col = lane & 15, kg = lane >> 4;
        const int rows = u.n * p.group, row_base = u.tile * 16 * NT;
        const int last_row = min(row_base + 16 * NT, rows) - 1;
        const int last_key = u.first + last_row / p.group;                        // the last position that a row of the tile sees
        const int begin = u.chunk * chunk_len, end = min(begin + chunk_len, last_key + 1);
        Rows tr;
        tr.token0 = row_base / p.group;
        tr.within0 = row_base - tr.token0 * p.group;
        tr.left = rows - row_base;
        tr.first = u.first;
        tr.group = p.group;
        tr.magic = p.group_magic;
        const int first_pos = u.first + tr.token0;                                // the first row's
        const auto row_of = [&](int x, int& token, int& h) {
            token = tr.token(x);
            h = u.head * p.group + tr.query(x);
        };
        bf16x8 q[kSharedQ ? 1 : NT][HD / 32];
        const auto load_q = [&](int n, u32x4 (&w)[HD / 32]) {
            const int r = row_base + 16 * n + col;
            int token, h;
            row_of(16 * n + col, token, h);
            const u16* src = p.q + (long long)(u.row0 + token) * p.ldq + h * HD + kg * 16;
#pragma unroll
            for (int j = 0; j < HD / 32; ++j) {
                w[j] = u32x4{0, 0, 0, 0};
                if (r < rows) w[j] = *reinterpret_cast<const u32x4*>(src + (j / 2) * 64 + (j % 2) * 8);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[j][i] = no_infinities(w[j][i] ^ p.q_sign);
            }
        };
        if constexpr (kSharedQ) {
            static_assert(NT == kAttnWaves, "a wave prepares one row tile (by its number: unrolled, this would be a copy of cold code for every wave)");
            u32x4 w[HD / 32];
            load_q(wave, w);
            if constexpr (kCodesQ) {
                split_q(w, sh, wave);
            } else {
#pragma unroll
                for (int j = 0; j < HD / 32; ++j) sh.q[wave][j][lane] = w[j];
            }
        } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                u32x4 w[HD / 32];
                load_q(n, w);
#pragma unroll
                for (int j = 0; j < HD / 32; ++j) q[n][j] = __builtin_bit_cast(bf16x8, w[j]);
            }
        }
        if (kSharedQ) __syncthreads();
        const int q_exp = kCodesQ ? *reinterpret_cast<const int*>(sh.q_exp[col]) : 0, q_last = kCodesQ ? uniform(*reinterpret_cast<const int*>(sh.q_last)) : 0;
        State st;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            st.m[n] = kNone;
            st.l[n] = 0.f;
#pragma unroll
            for (int i = 0; i < D; ++i) st.o[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        constexpr int stride = ALONE ? kStep : kRound;
        int key = begin + (ALONE ? 0 : wave * kStep);
        if (key < end) {
            PageIds ids;
            ids.start(c.table + (long long)u.slot * c.max_pages, (last_key >> c.t_log2) + 1, key >> c.t_log2);
            Step<HD> s;
            bool bad = false;
            const int T = 1 << c.t_log2;
            const Head hd{p.pages + (long long)u.head * 2 * T * HD, p.pages + c.scale_off + u.head * (T / kBlock) * 2, (unsigned)c.page_bytes,
                          (unsigned)c.n_pages, c.t_log2};
            Where<HD> w = find_step(hd, ids, key, last_key, bad);
            load_k(w, s);
            load_v(p, w, s);
            const auto is_masked = [&](const Step<HD>& t) { return key + kStep - 1 > first_pos || !t.ok[0] || !t.ok[1]; };
            // K's registers are free for the next step's codes once the scores are there, V's at the step's end.  A second set of registers,
            // requested a whole step ahead, was slower: what it spilled cost more (decode of 256 requests 145 us against 138).  Behind
            // the last step long row tiles request the same codes again, which spares their loop the branches.
            for (; key < end; key += stride) {
                const int next = key + stride;
                const bool more = NT >= 4 || next < end;
                const bool masked = is_masked(s), ok0 = s.ok[0], ok1 = s.ok[1];
                const unsigned int e[2] = {(unsigned)uniform((int)s.e[0]), (unsigned)uniform((int)s.e[1])};
                if (more) w = find_step(hd, ids, next < end ? next : key, last_key, bad);
                Scores sc;
                __builtin_amdgcn_s_setprio(1);      // (the other waves of the SIMD have exponentials to do)
                scores(s, q, q_exp, q_last, sh, sc);
                __builtin_amdgcn_s_setprio(0);
                accumulate([&] { if (more) load_k(w, s); }, s.v, ok0, ok1, sc, e, tr, key, last_key, masked, p.c_log2, st);
                if (more) load_v(p, w, s);
            }
            if (bad && lane == 0) atomicOr(c.err, kErrBadSegment);
        }
        if (kSharedQ) __syncthreads();          // acc takes q's place

        if constexpr (ALONE) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int x = 16 * n + col;
                const float l = column_sum(st.l[n]), inv = l == 0.f ? 0.f : 1.f / l;
                if (x >= tr.left) continue;
                int token, h;
                row_of(x, token, h);
                u16* dst = p.out + (long long)(u.row0 + token) * p.ldo + h * HD + 16 * kg;
#pragma unroll
                for (int i = 0; i < D; i += 4)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        *reinterpret_cast<u32x2*>(dst + 16 * i + 4 * r) = u32x2{pack_bf16x2(st.o[n][i][r] * inv, st.o[n][i + 1][r] * inv),
                                                                                pack_bf16x2(st.o[n][i + 2][r] * inv, st.o[n][i + 3][r] * inv)};
            }
            return;
        }

        // the waves' maxima and sums
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float l = column_sum(st.l[n]);
            if (kg == 0) {
                sh.m[wave][16 * n + col] = st.m[n];
                sh.l[wave][16 * n + col] = l;
            }
        }
        __syncthreads();
        const bool split = u.chunks > 1;
        if constexpr (NT == kAttnWaves) {
            join_by_tiles(p, u, tr, wave, split, st, sh);
            return;
        }
        const int out_row = (int)threadIdx.x / 16, out_col = (int)threadIdx.x % 16 * D;
        const __amdgpu_buffer_rsrc_t part = __builtin_amdgcn_make_buffer_rsrc(p.partial, 0, (int)p.partial_bytes, kRawBuffer);
        const int slot_bytes = slot_floats<HD, NT>() * 4, stat_at = 16 * NT * HD * 4;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float top = sh.m[0][16 * n + col];
#pragma unroll
            for (int w = 1; w < kAttnWaves; ++w) top = fmaxf(top, sh.m[w][16 * n + col]);
            const float a = __builtin_amdgcn_exp2f(st.m[n] - top);
#pragma unroll
            for (int i4 = 0; i4 < D / 4; ++i4)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const f32x4 v{st.o[n][4 * i4][r] * a, st.o[n][4 * i4 + 1][r] * a, st.o[n][4 * i4 + 2][r] * a, st.o[n][4 * i4 + 3][r] * a};
                    *reinterpret_cast<f32x4*>(&sh.acc[wave][col][64 * i4 + 16 * kg + 4 * r]) = v;
                }
            __syncthreads();
            const int r = row_base + 16 * n + out_row;
            if (r < rows) {
                float mt = sh.m[0][16 * n + out_row], l = 0.f;
#pragma unroll
                for (int w = 1; w < kAttnWaves; ++w) mt = fmaxf(mt, sh.m[w][16 * n + out_row]);
#pragma unroll
                for (int w = 0; w < kAttnWaves; ++w) {
                    const float mw = sh.m[w][16 * n + out_row];
                    l += sh.l[w][16 * n + out_row] * __builtin_amdgcn_exp2f(mw - mt);
                }
                float o[D];
#pragma unroll
                for (int i = 0; i < D; ++i) {
                    o[i] = 0.f;
#pragma unroll
                    for (int w = 0; w < kAttnWaves; ++w) o[i] += sh.acc[w][out_row][out_col + i];
                }
                if (!split) {
                    int token, h;
                    row_of(16 * n + out_row, token, h);
                    write_out(p, u.row0 + token, h, out_col, o, l);
                }
                else {
                    const int at = (u.slot0 + u.chunk) * slot_bytes;
                    const int row = 16 * n + out_row;
#pragma unroll
                    for (int i = 0; i < D; i += 4)
                        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]}), part, (row * HD + out_col + i) * 4, at, kSc1);
                    if (out_col == 0)
                        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, f32x2{mt, l}), part, stat_at + row * 8, at, kSc1);
                }
            }
            __syncthreads();
        }
        if (!split) return;

        // the last chunk of the tile adds them up
        if (!last_to_arrive(p, u, sh)) return;
        // Sixteen threads a row, and of few rows as many groups of threads as fit, to which the chunks are dealt: a chunk's sums and its maximum come
        // in one round trip and are added to what the group has; then the groups' sums in order.
        const int left = rows - row_base, live = min(left, 16);
        const int row_log2 = live <= 1 ? 0 : 32 - __builtin_clz(live - 1);       // the power of two above
        const int r = out_row & ((1 << row_log2) - 1), group = out_row >> row_log2, groups = 16 >> row_log2;
        Sums own[NT];
        if (r < live) {
#pragma unroll 2
            for (int k = group; k < u.chunks; k += groups)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int row = min(16 * n + r, left - 1), at = (u.slot0 + k) * slot_bytes;
                    Sums x;
                    const f32x2 ml = __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(part, at + stat_at + row * 8, 0, kSc1));
                    x.m = ml.x;
                    x.l = ml.y;
#pragma unroll
                    for (int i = 0; i < D; i += 4) {
                        const f32x4 v = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(part, at + (row * HD + out_col + i) * 4, 0, kSc1));
#pragma unroll
                        for (int c = 0; c < 4; ++c) x.o[i + c] = v[c];
                    }
                    own[n].add(x);
                }
        }
        Sums* all = reinterpret_cast<Sums*>(sh.sums_of_groups);
#pragma unroll
        for (int n = 0; n < NT; ++n) all[n * kAttnThreads + (int)threadIdx.x] = own[n];
        __syncthreads();
        if (group == 0 && r < live) {
            for (int g = 1; g < groups; ++g)
#pragma unroll
                for (int n = 0; n < NT; ++n) own[n].add(all[n * kAttnThreads + (int)threadIdx.x + (g << row_log2) * 16]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (16 * n + r >= left) continue;
                int token, h;
                row_of(16 * n + r, token, h);
                write_out(p, u.row0 + token, h, out_col, own[n].o, own[n].l);
            }
        }
    }

    static __device__ __forceinline__ void write_out(const AttnParams& p, int row, int h, int col, const float* o, float l)
    {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        unsigned int w[D / 2];
#pragma unroll
        for (int i = 0; i < D / 2; ++i) w[i] = pack_bf16x2(o[2 * i] * inv, o[2 * i + 1] * inv);
        u16* dst = p.out + (long long)row * p.ldo + h * HD + col;
        if constexpr (D == 8) *reinterpret_cast<u32x4*>(dst) = u32x4{w[0], w[1], w[2], w[3]};
        else *reinterpret_cast<u32x2*>(dst) = u32x2{w[0], w[1]};
    }
};

template <int HD, int NT>
__global__ __launch_bounds__(kAttnThreads, (kResident<HD, NT>)) void attention_kernel(AttnParams p)
{
    using A = Attention<HD, NT>;
    __shared__ typename A::Shared sh;
    extern __shared__ int prefix[];             // in the order of work: units before a span, partial-sum slots before it (both without the heads), its number
    const int n = p.sp.n_seqs, heads = p.c.n_kv_heads;
    int* units = prefix;
    int* slots = units + n + 1;
    int* order = slots + n;
    Span* spans = reinterpret_cast<Span*>(prefix + span_at(n));      // the spans, where they are few enough to be kept

    // the batch's work in (row tile) x (positions), and from it the chunk length
    const auto tiles_of = [&](const Span& s) { return (int)(((long long)s.n * p.group + 16 * NT - 1) / (16 * NT)); };
    long long work = 0;
    int longest = 0;
    unsigned int all_tiles = 0;                 // (stays at 2^30)
    for (int s = (int)threadIdx.x; s < n; s += kAttnThreads) {
        const Span u = load_span(p.c, p.sp, s);
        const int keys = u.n > 0 ? u.first + u.n : 0;
        const int tiles = u.n > 0 ? tiles_of(u) : 0;
        units[s] = tiles;
        slots[s] = keys;
        if (n <= kKeptSpans<NT>) spans[s] = u;
        work += (long long)tiles * keys;
        longest = max(longest, keys);
        all_tiles = min(all_tiles + (unsigned)tiles, 1u << 30);
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        all_tiles = min(all_tiles + (unsigned)__shfl_xor((int)all_tiles, d, kWave), 1u << 30);
        longest = max(longest, __shfl_xor(longest, d, kWave));
        work += __shfl_xor(work, d, kWave);
    }
    if (lane_id() == 0) {
        sh.sums[threadIdx.x / kWave] = work;
        sh.longest[threadIdx.x / kWave] = longest;
        sh.tiles[threadIdx.x / kWave] = all_tiles;
    }
    __syncthreads();
    work = 0;
    all_tiles = 0;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
        work += sh.sums[w];
        longest = max(longest, sh.longest[w]);
        all_tiles = min(all_tiles + sh.tiles[w], 1u << 30);
    }
    // Spans that share rows (row_starts that decrease) may have more tiles than the rows there are: the sums below would not fit.
    if (all_tiles > (unsigned)((long long)p.sp.n_rows * p.group / (16 * NT) + n)) {
        if (threadIdx.x == 0) atomicOr(p.c.err, kErrBadSegment);
        return;
    }
    work *= heads;
    // Tiles with more positions than the chunk length are fewer than work / length and have fewer than 2 work / length chunks in all.
    const auto length = [&](int n_slots, int most) { return max((work + n_slots / 2 - 1) / (n_slots / 2), (long long)((longest + most - 1) / most)); };
    const long long few = length(kSlots<NT>, 15), many = length(kManyChunksSlots, 255);
    const int bits = uniform(few <= many ? 4 : 8);
    // A tile has half a chunk more than its share of the work on average, so this is the length with which every workgroup gets a unit; with
    // more than half as many tiles as workgroups, half a unit.  Nothing is split that is not longer by kSplitCost.
    const int grid = (int)gridDim.x;
    const long long share = work / (grid - (int)min((long long)all_tiles * heads, (long long)grid) / 2) + 1;
    const long long split = max(max(min(few, many), share), (long long)kLeastChunk);
    const long long len = longest <= split + kSplitCost<NT> ? max((long long)longest, split) : split;
    const int chunk_len = uniform((int)min((len + kRound - 1) / kRound * kRound, 1ll << 30));

    // Prefix sums, 256 spans a round; within a round the longest spans first (by powers of two below the longest of all), so that the
    // tickets end evenly.
    int unit_base = 0, slot_base = 0;
    for (int s0 = 0; s0 < n; s0 += kAttnThreads) {
        const int s = s0 + (int)threadIdx.x, wave = (int)threadIdx.x / kWave;
        int tiles = s < n ? units[s] : 0, keys = s < n ? slots[s] : 0;
        const int shorter = s < n ? min(__builtin_clz(max(keys, 1)) - __builtin_clz(max(longest, 1)), kClasses - 1) : kClasses;
        int same = 0, rank = 0;
#pragma unroll
        for (int k = 0; k < kClasses; ++k) {
            const unsigned long long in = __ballot(shorter == k);
            if (shorter == k) same = __popcll(in & ((1ull << lane_id()) - 1));
            if (lane_id() == 0) sh.classes[wave][k] = __popcll(in);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kClasses; ++k)
#pragma unroll
            for (int w = 0; w < kAttnWaves; ++w)
                if (k < shorter || (k == shorter && w < wave)) rank += sh.classes[w][k];
        if (s < n) {
            order[s0 + rank + same] = s;
            units[s0 + rank + same] = tiles;
            slots[s0 + rank + same] = keys;
        }
        __syncthreads();
        tiles = s < n ? units[s] : 0;
        keys = s < n ? slots[s] : 0;
        const int chunks = max((keys + chunk_len - 1) / chunk_len, 1);
        const int mine = tiles * chunks, split = chunks > 1 ? mine : 0;
        const int units_upto = wave_inclusive_scan(mine), slots_upto = wave_inclusive_scan(split);
        if (lane_id() == kWave - 1) {
            sh.scan[wave][0] = units_upto;
            sh.scan[wave][1] = slots_upto;
        }
        __syncthreads();
        int units_at = unit_base + units_upto - mine, slots_at = slot_base + slots_upto - split;
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) {
            if (w < wave) {
                units_at += sh.scan[w][0];
                slots_at += sh.scan[w][1];
            }
            unit_base += sh.scan[w][0];
            slot_base += sh.scan[w][1];
        }
        if (s < n) {
            units[s] = units_at;
            slots[s] = slots_at;
        }
    }
    if (threadIdx.x == 0) units[n] = unit_base;
    __syncthreads();

    // Many sequences that are short, or about equally long: a unit per wave.  (A unit's instructions outside its steps, some 1000 a wave, are then
    // spent by one wave and not by four, and nothing is exchanged: 300 requests of up to 100 positions 39 us by workgroups, 16 by waves, 256
    // of 2000 181 and 160; but 256 of up to 2000, the longest eight times the mean of a wave, 68 and 89.)
    const int n_units = uniform(unit_base) * heads;
    const bool even = chunk_len >= longest && (long long)longest * (2 * grid) <= work;       // (a wave's share is half the longest or more)
    const bool alone = A::kAlone && n_units > grid && uniform(even || longest <= kAloneLongest);
    // Prompts: a key head's units in one XCD, where the heads fall evenly on them (32 of 512 rows behind 2560 positions, 8 key heads: 786 us
    // with one counter, 756 so; 4 of 3000 rows, 5 key heads: 115 and 117).
    const bool by_heads = NT >= 4 && (heads % 8 == 0 || 8 % heads == 0) && gridDim.x % 8 == 0;
    for_each_unit(p.tickets, alone ? (n_units + kAttnWaves - 1) / kAttnWaves : n_units, sh.slot, [&](int group, int) {
        // Where every workgroup has one unit or two, the workgroups with the longest first unit have no second.
        const int id = alone                                                     ? group * kAttnWaves + uniform((int)threadIdx.x / kWave)
                       : group < grid && n_units > grid && n_units <= 2 * grid ? grid - 1 - group
                                                                                 : group;
        if (id >= n_units) return;
        Unit u;
        const int v = id / heads;
        u.head = id - v * heads;
        const int at = uniform(last_not_above(n, v, [&](int k) { return units[k]; })), s = uniform(order[at]);
        const Span span = n <= kKeptSpans<NT> ? spans[s] : load_span(p.c, p.sp, s);
        u.slot = uniform(span.slot);
        u.row0 = uniform(span.row0);
        u.n = uniform(span.n);
        u.first = uniform(span.first);
        if (u.n <= 0) return;
        u.chunks = max((u.first + u.n + chunk_len - 1) / chunk_len, 1);
        u.bits = bits;
        // (the chunks of a tile equally long)
        const int equal = ((u.first + u.n + u.chunks - 1) / u.chunks + kRound - 1) / kRound * kRound;
        const int local = v - uniform(units[at]);
        const int back = local / u.chunks;
        u.chunk = local - back * u.chunks;
        u.tile = tiles_of(Span{u.slot, u.row0, u.n, u.first}) - 1 - back;      // the tiles with the most positions first
        u.slot0 = ((uniform(slots[at]) + back * u.chunks) * heads + u.head * u.chunks);
        if constexpr (A::kAlone) {
            if (alone) {
                A::template run_unit<true>(p, u, equal, sh);
                return;
            }
        }
        A::template run_unit<false>(p, u, equal, sh);
    }, 0, by_heads ? 8 : 1);
}

template <int HD, int NT>
constexpr int prefix_bytes(int n_seqs) { return span_at(n_seqs) * (int)sizeof(int) + (n_seqs <= kKeptSpans<NT> ? n_seqs * (int)sizeof(Span) : 0); }

// Workgroups of a CU that the LDS has room for: the grid is no larger.  (A workgroup's first two units are its own, the longest first: one that only
// starts when others are done ends last.  With kResident whatever the LDS holds: 1000 sequences of 600 positions 228 us, so 208; 2000 of up
// to 60 87 and 72; but 700 of up to 4000, about as many units as the larger grid has places for, 369 and 410.)
template <int HD, int NT>
constexpr int resident(int n_seqs)
{
    const int bytes = (int)sizeof(typename Attention<HD, NT>::Shared) + prefix_bytes<HD, NT>(n_seqs);
    const int room = kLdsBytes / ((bytes + kLdsGranule - 1) / kLdsGranule * kLdsGranule);
    return room < kResident<HD, NT> ? room : kResident<HD, NT>;
}

template <int HD, int NT>
hipError_t launch_attention(AttnParams p, int max_units, void* workspace, hipStream_t stream)
{
    static_assert(resident<HD, NT>(NT < 4 ? 512 : kKeptSpans<NT>) == kResident<HD, NT>, "no workgroup's room is taken by few spans");
    static_assert(resident<HD, NT>(kKeptSpans<NT>) >= 1 && resident<HD, NT>(LQ_CACHE_MAX_SEQS) >= 1, "every call fits");
    static DeviceGrid cus;
    const int n_cu = cus.get([] {
        int dev = 0, n = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(attention_kernel<HD, NT>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                  max(prefix_bytes<HD, NT>(LQ_CACHE_MAX_SEQS), prefix_bytes<HD, NT>(kKeptSpans<NT>)));
        return n;
    });
    const int grid = min(max_units, n_cu * resident<HD, NT>(p.sp.n_seqs)), lds = prefix_bytes<HD, NT>(p.sp.n_seqs);
    p.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + kWsHeaderBytes);
    p.partial_bytes = (unsigned)kSlots<NT> * slot_floats<HD, NT>() * 4;
    p.tickets = static_cast<int*>(workspace) + 4;
    p.arrivals = static_cast<uint8_t*>(workspace) + 4 * kArrivals;
    hipLaunchKernelGGL((attention_kernel<HD, NT>), dim3(grid), dim3(kAttnThreads), lds, stream, p);
    return hipGetLastError();
}

// Row tiles of 16 of a unit: a group of query heads of one token, a draft, or a prompt.  Four tiles widen every code for 64 rows and
// cost 3 us more to set up and to join: where units of two tiles do not fill the compute units, those are faster by that behind few
// positions, and lose it only behind thousands (us, two tiles against four: 16 spans of 16 rows of 4 heads behind 300 positions 12.0 and
// 15.4, behind 2000 28.6 and 29.5; one of 64 rows behind 1000 16.6 and 22.0, behind 12000 37.4 and 37.5, behind 30000 62 and 54; but 20 spans of
// 16 rows, 320 units, behind 2000 34.1 and 30.5; 60 of 14 x 3 rows for 16 key heads, 1920 units, 38 and 27).
int row_tiles(int group, int max_rows, int n_seqs, int kv_heads)
{
    const long long rows = (long long)group * max_rows;
    if (rows <= 16) return 1;
    if (rows <= 32) return 2;
    return (rows + 31) / 32 * n_seqs * kv_heads <= (rows <= 128 ? 256 : rows <= 256 ? 128 : 0) ? 2 : 4;
}

}  // namespace
}  // namespace lq

extern "C" size_t lora_cache_attention_workspace_bytes(const lq_cache* host_cache, int32_t n_heads, int32_t max_rows)
{
    using namespace lq;
    if (!host_cache || host_cache->n_kv_heads <= 0 || n_heads <= 0 || n_heads % host_cache->n_kv_heads || max_rows <= 0) return 0;
    // (two row tiles and four need the same)
    static_assert(kSlots<2> * 2 == kSlots<4> * 4, "one size for both");
    const int nt = row_tiles(n_heads / host_cache->n_kv_heads, max_rows, 1, 1);
    const size_t slots = nt == 1 ? kSlots<1> : nt == 2 ? kSlots<2> : kSlots<4>;
    return kWsHeaderBytes + slots * 16 * nt * ((size_t)host_cache->head_dim + 2) * 4;
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
    const int hd = host_cache->head_dim, kv = host_cache->n_kv_heads;
    if (n_heads <= 0 || n_heads % kv || max_rows <= 0) return LQ_ERR_INVALID_ARG;
    if (ldq < (int64_t)n_heads * hd || ldo < (int64_t)n_heads * hd) return LQ_ERR_INVALID_ARG;
    if (n_rows > 0 && (!q || !out || q == out)) return LQ_ERR_INVALID_ARG;
    if (!(scale > -__builtin_inff() && scale < __builtin_inff())) return LQ_ERR_INVALID_ARG;
    if (n_heads > LQ_CACHE_MAX_HEADS || n_seqs > LQ_CACHE_MAX_SEQS || n_rows > LQ_CACHE_MAX_ROWS) return LQ_ERR_UNSUPPORTED;
    if ((ldq % 8) || (ldo % 8) || !aligned16(q) || !aligned16(out)) return LQ_ERR_UNSUPPORTED;
    if (!workspace || !aligned16(workspace) || workspace_bytes < lora_cache_attention_workspace_bytes(host_cache, n_heads, max_rows))
        return LQ_ERR_WORKSPACE;
    if (n_seqs == 0 || n_rows == 0) return LQ_OK;
    p.sp = Spans{slots, row_starts, first, n_seqs, n_rows};
    p.q = static_cast<const u16*>(q);
    p.ldq = ldq;
    p.out = static_cast<u16*>(out);
    p.ldo = ldo;
    p.pages = static_cast<const uint8_t*>(pages);
    p.group = n_heads / kv;
    // (not zero: a masked score is -infinity times this; the least number above it times the largest score is below 2^-20)
    p.c_log2 = __builtin_fmaxf(__builtin_fabsf(scale) * 1.44269504f, 1e-45f);
    p.group_magic = (unsigned)(((1 << 20) + p.group - 1) / p.group);
    p.q_sign = scale < 0.f ? 0x80008000u : 0u;
    const int nt = row_tiles(p.group, max_rows, n_seqs, kv);
    // no more workgroups than there can be units
    const int64_t tiles = (int64_t)n_rows * p.group / (16 * nt) + n_seqs;
    const int64_t chunks = (p.c.max_len + kLeastChunk - 1) / kLeastChunk;
    const int64_t units = tiles * kv * (chunks < 255 ? chunks : 255);
    const int max_units = (int)(units < (1 << 20) ? units : 1 << 20);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (hd == 128) e = nt == 1 ? launch_attention<128, 1>(p, max_units, workspace, hs) : nt == 2 ? launch_attention<128, 2>(p, max_units, workspace, hs)
                                                                                            : launch_attention<128, 4>(p, max_units, workspace, hs);
    else e = nt == 1 ? launch_attention<64, 1>(p, max_units, workspace, hs) : nt == 2 ? launch_attention<64, 2>(p, max_units, workspace, hs)
                                                                                       : launch_attention<64, 4>(p, max_units, workspace, hs);
    return e == hipSuccess ? LQ_OK : LQ_ERR_HIP;
}
