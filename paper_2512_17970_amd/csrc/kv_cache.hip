// The paged cache: new keys and values go in, rotated and normalised on the way, and come out again as contiguous fp16.
//
// Append: a team of 128 threads takes the queries of a token, a workgroup the keys (or values) of one head for the tokens that share a scale, so
// that their largest |x| stays within it; a lane has 16 elements of a row, those that turn with each other, so that rotation needs no exchange and the norm a few.
// Bound by the bytes: 8446 tokens, 64 and 8 heads of 128, 8 bits: 73 us for 346 MB, 4.7 TB/s; by the launch and loads one after the other where there are few: one
// token of 32 heads 3.7 us, 32 sequences' 5.8 (lengths, page, old scale; tokens too are asked for after those, which they do not depend on), 7.0 where
// blocks get larger scales and the codes in them are converted.
// Gather: a workgroup takes 16 tokens of one head, values by way of LDS, which turns them.  30087 tokens of 8 heads, 8 bits: 30 to 33 us for
// 185 MB, 5.6 to 6.2 TB/s.
#include "attn_common.h"

namespace cg {

constexpr int kAppendThreads = 128;         // that take 16 tokens of a head, or the queries of a token
constexpr int kMostTeams = 8;               // of them in a workgroup
constexpr int kTeamsAtOnce = 2048;          // 16 wavefronts on each of 256 compute units
constexpr int kLastEnd = 0x7ffffe00;        // a length past every table, from which counting on by a unit stays within 32 bits

struct AppendParams {
    CacheView c;
    const int32_t* cu;
    const _Float16 *q, *k, *v, *q_norm, *k_norm;
    const float* rope;
    _Float16 *q_out, *k_out;
    int T, Hq, R, positions;
    int q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
    int interleaved;
    float eps;
    int row_lanes;      // lanes of a row of D: the power of two from D / 16 on
    int group;          // tokens of a unit: those that share a scale, at least kTokenGroup
    int units;          // of keys, and of values
    int teams;          // of a workgroup
    int token_blocks;   // workgroups that work on queries, ahead of those of keys and values
    int token_split;    // teams of one token
};

__device__ __forceinline__ int new_tokens(const AppendParams& p, int seq, int* row0)
{
    int lo = p.cu ? p.cu[seq] : seq, hi = p.cu ? p.cu[seq + 1] : seq + 1;
    lo = lo < 0 ? 0 : lo > p.T ? p.T : lo;
    hi = hi < lo ? lo : hi > p.T ? p.T : hi;
    *row0 = lo;
    return hi - lo;
}

// 16 elements of a row, as two runs of 8: where the lane's pairs lie.  Lanes in front of R / 16 hold pairs 8 c .. 8 c + 7.
struct Runs {
    int a, b;
    bool turns;
};
__device__ __forceinline__ Runs runs_of(int c, int R, bool interleaved)
{
    Runs r;
    r.turns = c < R / 16;
    const bool half = r.turns && !interleaved;
    r.a = half ? 8 * c : 16 * c;
    r.b = half ? R / 2 + 8 * c : 16 * c + 8;
    return r;
}

// The lane's 16 values of one head, normalised and rotated in fp32.  x is clear where the lane has none (D / 16 <= c).
__device__ __forceinline__ void load_row(float (&x)[16], const _Float16* row, const Runs& r, bool live)
{
    half8_t a = {0, 0, 0, 0, 0, 0, 0, 0}, b = a;
    if (live) {
        a = *reinterpret_cast<const half8_t*>(row + r.a);
        b = *reinterpret_cast<const half8_t*>(row + r.b);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) { x[e] = (float)a[e]; x[8 + e] = (float)b[e]; }
}

__device__ __forceinline__ void norm_row(float (&x)[16], const _Float16* weight, const Runs& r, bool live, int row_lanes, int D, float eps)
{
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
    for (int o = row_lanes >> 1; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    const float by = 1.0f / sqrtf(sum / (float)D + eps);
    if (!live) return;
    const half8_t a = *reinterpret_cast<const half8_t*>(weight + r.a), b = *reinterpret_cast<const half8_t*>(weight + r.b);
#pragma unroll
    for (int e = 0; e < 8; ++e) { x[e] = x[e] * by * (float)a[e]; x[8 + e] = x[8 + e] * by * (float)b[e]; }
}

struct Turn {
    float cs[16];       // cos and sin of the lane's 8 pairs
};

__device__ __forceinline__ Turn load_turn(const AppendParams& p, int position, int c)
{
    const int at = position < p.positions ? position : p.positions - 1;
    const float4_t* t = reinterpret_cast<const float4_t*>(p.rope + ((size_t)at * (p.R / 2) + 8 * c) * 2);
    Turn r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float4_t w = t[e];
#pragma unroll
        for (int i = 0; i < 4; ++i) r.cs[4 * e + i] = w[i];
    }
    return r;
}

// (a, b) -> (a cos - b sin, b cos + a sin); products and sums each rounded, as elementary operations give them
__device__ __forceinline__ void rotate_row(float (&x)[16], const Turn& t, bool interleaved)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float co = t.cs[2 * e], si = t.cs[2 * e + 1];
        float a = interleaved ? x[2 * e] : x[e], b = interleaved ? x[2 * e + 1] : x[8 + e];
        const float ra = a * co - b * si, rb = b * co + a * si;
        if (interleaved) { x[2 * e] = ra; x[2 * e + 1] = rb; }
        else { x[e] = ra; x[8 + e] = rb; }
    }
}

__device__ __forceinline__ void store_row(_Float16* row, const float (&x)[16], const Runs& r)
{
    half8_t a, b;
#pragma unroll
    for (int e = 0; e < 8; ++e) { a[e] = (_Float16)x[e]; b[e] = (_Float16)x[8 + e]; }
    *reinterpret_cast<half8_t*>(row + r.a) = a;
    *reinterpret_cast<half8_t*>(row + r.b) = b;
}

template <int TYPE> struct KvType;
template <> struct KvType<CODEGEMM_KV_FP16> { typedef _Float16 elem; static constexpr float kMax = 0.0f; };
template <> struct KvType<CODEGEMM_KV_INT8> { typedef uint8_t elem; static constexpr float kMax = 127.0f; };
template <> struct KvType<CODEGEMM_KV_FP8> { typedef uint8_t elem; static constexpr float kMax = 448.0f; };

// x / scale as the cache holds it, ties to even; |x / scale| <= kMax but for the rounding of the scale's reciprocal.
template <int TYPE>
__device__ __forceinline__ uint8_t code_of(float x)
{
    x = __builtin_amdgcn_fmed3f(x, -KvType<TYPE>::kMax, KvType<TYPE>::kMax);
    if constexpr (TYPE == CODEGEMM_KV_INT8) return (uint8_t)(int8_t)(int)rintf(x);
    else return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 255);
}
template <int TYPE>
__device__ __forceinline__ float value_of(uint8_t c)
{
    if constexpr (TYPE == CODEGEMM_KV_INT8) return (float)(int8_t)c;
    else return (float)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)c, 1.0f, false)[0];
}

// Queries of one token: a team, or token_split of them.
__device__ void append_queries(const AppendParams& p, int team)
{
    const int token = team / p.token_split, part = team % p.token_split;
    if (token >= p.T) return;
    const int tid = threadIdx.x % kAppendThreads, lanes = p.row_lanes, c = tid & (lanes - 1), rows = kAppendThreads / lanes;
    const bool live = c < p.c.D / 16;
    const Runs r = runs_of(c, p.R, p.interleaved != 0);
    // the first rows are on their way while the token's position is looked up
    float x[16];
    auto load = [&](int h) { load_row(x, p.q + (size_t)token * p.q_stride + (h < p.Hq ? h : 0) * p.c.D, r, live && h < p.Hq); };
    if (p.Hq > 0) load(part * rows + tid / lanes);
    const int seq = p.cu ? last_at_most(p.c.seqs, token, [&](int i) { return p.cu[i]; }) : token;
    int row0;
    const int n = new_tokens(p, seq, &row0);
    const int len = p.c.lens[seq], position = (len < 0 ? 0 : len) - n + token - row0;
    const float zeros[16] = {0};
    if (position < 0) {                              // no place in the sequence
        for (int h = part * rows + tid / lanes; h < p.Hq; h += rows * p.token_split)
            if (live) store_row(p.q_out + (size_t)token * p.q_out_stride + h * p.c.D, zeros, r);
        if (part == 0 && p.k_out)
            for (int h = tid / lanes; h < p.c.Hk; h += rows)
                if (live) store_row(p.k_out + (size_t)token * p.k_out_stride + h * p.c.D, zeros, r);
        return;
    }
    Turn t;
    if (live && r.turns) t = load_turn(p, position, c);
    for (int h0 = part * rows; h0 < p.Hq; h0 += rows * p.token_split) {          // uniform: the norm's exchanges need whole rows
        const int h = h0 + tid / lanes;
        const bool mine = live && h < p.Hq;
        if (h0 > part * rows) load(h);
        if (p.q_norm) norm_row(x, p.q_norm, r, mine, lanes, p.c.D, p.eps);
        if (!mine) continue;
        if (r.turns) rotate_row(x, t, p.interleaved != 0);
        store_row(p.q_out + (size_t)token * p.q_out_stride + h * p.c.D, x, r);
    }
}

// Keys or values of one unit: up to `group` new tokens of one sequence and head that share a page, and their scales.
template <int TYPE, bool TEAMS>
__device__ void append_unit(const AppendParams& p, int unit, int head, bool values, unsigned char* lds)
{
    typedef typename KvType<TYPE>::elem elem;
    const CacheView& cv = p.c;
    const int D = cv.D, G = p.group, lanes = p.row_lanes, teams = TEAMS ? p.teams : 1, threads = teams * kAppendThreads, tid = threadIdx.x;
    const int team = TEAMS ? __builtin_amdgcn_readfirstlane(tid / kAppendThreads) : 0, member = TEAMS ? tid % kAppendThreads : tid, c = member & (lanes - 1), rows = kAppendThreads / lanes;
    int seq = unit;
    if (p.cu) seq = last_at_most(cv.seqs, unit, [&](int i) { return p.cu[i] / G + 2 * i; });
    int row0;
    const int n = new_tokens(p, seq, &row0);
    const int len = cv.lens[seq], end = len < 0 ? 0 : len < kLastEnd ? len : kLastEnd, start = end - n;         // positions of the new tokens: start .. end - 1
    const int from = start < 0 ? 0 : start;
    const int skip = p.cu ? unit - (p.cu[seq] / G + 2 * seq) : 0;
    if (skip < 0 || from >= end || from / G + skip > (end - 1) / G) return;
    const int pos0 = (from / G + skip) * G;                                                // of the unit
    const int lo = pos0 > from ? pos0 : from, hi = end - pos0 > G ? pos0 + G : end;        // its new tokens
    const int page = page_of(cv, seq, pos0 >> cv.page_shift);
    if (page < 0 && (values || !p.k_out)) return;
    const int slot0 = pos0 & ((1 << cv.page_shift) - 1);
    const bool live = c < D / 16;
    const Runs r = values ? runs_of(c, 0, false) : runs_of(c, p.R, p.interleaved != 0);
    const _Float16* src = (values ? p.v + head * D : p.k + head * D);
    const size_t stride = values ? p.v_stride : p.k_stride;
    unsigned char* pool = values ? cv.v : cv.k;
    const size_t at = page < 0 ? 0 : page_at(cv, page, head);

    auto load = [&](float (&x)[16], int pos, bool mine) {
        const int row = mine ? row0 + pos - start : 0;
        load_row(x, src + row * stride, r, mine);
        if (values) return;
        if (p.k_norm) norm_row(x, p.k_norm, r, mine, lanes, D, p.eps);
        if (mine && r.turns) rotate_row(x, load_turn(p, pos, c), p.interleaved != 0);
    };

    // The unit's groups of 16 tokens go round the teams; where each team has one at most and takes it at once, tokens stay in registers from the search
    // for the largest to their conversion.
    const int group0 = lo & ~(kTokenGroup - 1), groups = (hi - 1 - group0) / kTokenGroup + 1, rounds = (groups + teams - 1) / teams;
    const bool kept = rounds == 1 && (rows >= kTokenGroup || (groups == 1 && hi - lo <= rows));
    float x[16];
    uint32_t* of_block = reinterpret_cast<uint32_t*>(lds);                                 // [G / block <= 16]: the bits of the largest |x|, then of the scale
    auto scale_of_block = [&](int b) { return __builtin_bit_cast(float, of_block[b]); };
    if constexpr (TYPE != CODEGEMM_KV_FP16) {
        // The largest |x| of every block.  As bits: they order as the values do, with infinities and NaN above all numbers.
        const int blocks = G >> cv.block_shift;
        for (int b = tid; b < blocks; b += threads) of_block[b] = 0;
        float* scales = (values ? cv.v_scales : cv.k_scales) + (page < 0 ? 0 : scales_at(cv, page, head) + (slot0 >> cv.block_shift));
        const int b_lo = (lo - pos0) >> cv.block_shift, first_lo = pos0 + (b_lo << cv.block_shift);
        const bool earlier = page >= 0 && first_lo < lo;                                   // the block of the first new token holds tokens already
        const float old = earlier ? scales[b_lo] : 0.0f;
        __syncthreads();
        // tokens that stay: those of the team's group; else as they come
        const int g0 = group0 + team * kTokenGroup, t_lo = !kept ? lo + team * rows : g0 > lo ? g0 : lo, t_hi = kept && g0 + kTokenGroup < hi ? g0 + kTokenGroup : hi;
        for (int t0 = t_lo; t0 < t_hi; t0 += teams * rows) {
            const int pos = t0 + member / lanes;
            const bool mine = live && pos < t_hi;
            load(x, pos, mine);
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t w = __builtin_bit_cast(uint32_t, x[e]) & 0x7fffffffu;
                m = w > m ? w : m;
            }
            for (int o = lanes >> 1; o > 0; o >>= 1) {
                const uint32_t w = (uint32_t)__shfl_xor((int)m, o);
                m = w > m ? w : m;
            }
            if (mine && c == 0) atomicMax(&of_block[(pos - pos0) >> cv.block_shift], m);
        }
        __syncthreads();
        for (int b = tid; b < blocks; b += threads) {
            const int first = pos0 + (b << cv.block_shift), past = first + (1 << cv.block_shift);
            if (page < 0 || past <= lo || first >= hi) continue;
            const uint32_t m = of_block[b];
            float s = __builtin_bit_cast(float, m) / KvType<TYPE>::kMax;
            if (earlier && b == b_lo) s = old <= s ? s : old;                              // a NaN stays
            if (m >= 0x7f800000u || !(s <= 3.402823466e38f)) s = __builtin_nanf("");
            of_block[b] = __builtin_bit_cast(uint32_t, s);
            scales[b] = s;
        }
        __syncthreads();
        const float now = earlier ? scale_of_block(b_lo) : 0.0f;
        if (earlier && old < now) {                                                        // the earlier tokens in the larger scale, 16 bytes at a time
            const float ratio = old > 0.0f ? old / now : 0.0f;
            const int slot_lo = slot0 + first_lo - pos0, slot_hi = slot0 + lo - pos0;
            // of keys, 16 dimensions of a token; of values, a dimension's group of 16 tokens, of which the block may have a part
            const int piece0 = values ? slot_lo / kTokenGroup * D : slot_lo * D / 16, pieces = (values ? ceil_div(slot_hi, kTokenGroup) * D : slot_hi * D / 16) - piece0;
            for (int i = tid; i < pieces; i += threads) {
                u32x4_t* at16 = reinterpret_cast<u32x4_t*>(pool + at) + piece0 + i;
                const int t0 = values ? (piece0 + i) / D * kTokenGroup : slot_lo;
                const u32x4_t in = *at16;
                alignas(16) uint8_t w[16];
                __builtin_memcpy(w, &in, 16);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int slot = values ? t0 + e : t0;
                    const uint8_t c2 = code_of<TYPE>(value_of<TYPE>(w[e]) * ratio);
                    w[e] = slot >= slot_lo && slot < slot_hi ? c2 : w[e];
                }
                u32x4_t out;
                __builtin_memcpy(&out, w, 16);
                *at16 = out;
            }
            __syncthreads();                                                               // before the new tokens go beside them
        }
    }

    constexpr int kPad = 16 / (int)sizeof(elem);
    elem* stage = reinterpret_cast<elem*>(lds + 64) + team * (D * kTokenGroup + D / 16 * kPad);      // [D][16] of a group of 16 tokens, 16 bytes more every 16 rows
    for (int round = 0; round < rounds; ++round) {                                         // a team may have none in the last
        const int g0 = group0 + (round * teams + team) * kTokenGroup, glo = g0 > lo ? g0 : lo, ghi = g0 + kTokenGroup < hi ? g0 + kTokenGroup : hi;
        for (int t0 = glo; t0 < ghi; t0 += rows) {
            const int pos = t0 + member / lanes;
            const bool mine = live && pos < ghi;
            if (TYPE == CODEGEMM_KV_FP16 || !kept) load(x, pos, mine);
            if (!mine) continue;
            if (!values && p.k_out) store_row(p.k_out + (size_t)(row0 + pos - start) * p.k_out_stride + head * D, x, r);
            if (page < 0) continue;
            const int slot = slot0 + pos - pos0;
            alignas(16) elem w[16];
            if constexpr (TYPE == CODEGEMM_KV_FP16) {
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = (_Float16)x[e];
            } else {
                const float s = scale_of_block((pos - pos0) >> cv.block_shift);
                const float by = s >= 1.17549435e-38f ? 1.0f / s : 0.0f;                   // a NaN scale: zeros
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = code_of<TYPE>(by != 0.0f ? x[e] * by : 0.0f);
            }
            if (!values) {
                elem* dst = reinterpret_cast<elem*>(pool) + at + (size_t)slot * D;
                typedef elem run __attribute__((ext_vector_type(8)));
                run a, b;
#pragma unroll
                for (int e = 0; e < 8; ++e) { a[e] = w[e]; b[e] = w[8 + e]; }
                *reinterpret_cast<run*>(dst + r.a) = a;
                *reinterpret_cast<run*>(dst + r.b) = b;
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) stage[(16 * c + e) * kTokenGroup + c * kPad + slot % kTokenGroup] = w[e];
            }
        }
        if (values && page >= 0) {                                                         // uniform
            __syncthreads();
            elem* dst = reinterpret_cast<elem*>(pool) + at + (size_t)((slot0 + g0 - pos0) / kTokenGroup) * D * kTokenGroup;
            if (ghi - glo == kTokenGroup) {
                constexpr int kVec = 16 / (int)sizeof(elem);                               // elements of 16 bytes
                for (int i = member; i < D * kTokenGroup / kVec; i += kAppendThreads) {
                    const int d = i * kVec / kTokenGroup;
                    *reinterpret_cast<u32x4_t*>(dst + i * kVec) = *reinterpret_cast<const u32x4_t*>(stage + i * kVec + d / 16 * kPad);
                }
            } else {
                const int tokens = ghi - glo;
                for (int i = member; i < D * tokens; i += kAppendThreads) {
                    const int d = i / tokens, t = (glo & (kTokenGroup - 1)) + i % tokens;
                    dst[d * kTokenGroup + t] = stage[d * kTokenGroup + d / 16 * kPad + t];
                }
            }
            __syncthreads();
        }
    }
}

// Bytes of LDS of a workgroup.
template <int TYPE>
constexpr size_t append_lds(int teams, int D) { return 64 + (size_t)teams * (D * kTokenGroup * sizeof(typename KvType<TYPE>::elem) + D); }

template <int TYPE, bool TEAMS>
__global__ void __launch_bounds__(TEAMS ? kMostTeams * kAppendThreads : kAppendThreads) kv_append_kernel(const AppendParams p)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const int blk = blockIdx.x;
    if (blk < p.token_blocks) {
        append_queries(p, TEAMS ? blk * p.teams + __builtin_amdgcn_readfirstlane(threadIdx.x / kAppendThreads) : blk);
        return;
    }
    const int i = blk - p.token_blocks, half = p.units * p.c.Hk;
    const bool values = i >= half;
    const int j = values ? i - half : i;
    append_unit<TYPE, TEAMS>(p, j / p.c.Hk, j % p.c.Hk, values, lds);
}

template <int TYPE>
static void launch_append(const AppendParams& p, unsigned blocks, hipStream_t s)
{
    const dim3 grid(blocks), threads(p.teams * kAppendThreads);
    const size_t lds = append_lds<TYPE>(p.teams, p.c.D);
    if constexpr (TYPE != CODEGEMM_KV_FP16) {
        if (p.teams > 1) {
            hipLaunchKernelGGL((kv_append_kernel<TYPE, true>), grid, threads, lds, s, p);
            return;
        }
    }
    hipLaunchKernelGGL((kv_append_kernel<TYPE, false>), grid, threads, lds, s, p);
}

struct GatherParams {
    CacheView c;
    const int32_t *cu, *first;
    _Float16 *k_out, *v_out;
    int rows, row_lanes;
};

// One group of 16 positions of a sequence and head: blockIdx.y 0 keys, 1 values.
template <int TYPE>
__global__ void __launch_bounds__(kAppendThreads) kv_gather_kernel(const GatherParams p)
{
    typedef typename KvType<TYPE>::elem elem;
    __shared__ __align__(16) unsigned char lds[(kMaxHeadDim * kTokenGroup + 256) * sizeof(elem)];
    const CacheView& cv = p.c;
    const bool values = blockIdx.y != 0;
    _Float16* out = values ? p.v_out : p.k_out;
    if (!out) return;
    const int D = cv.D, lanes = p.row_lanes, tid = threadIdx.x, c = tid & (lanes - 1), per = kAppendThreads / lanes;
    const int unit = blockIdx.x / cv.Hk, head = blockIdx.x % cv.Hk;
    const int seq = last_at_most(cv.seqs, unit, [&](int i) { return p.cu[i] / kTokenGroup + 2 * i; });
    int lo = p.cu[seq], hi = p.cu[seq + 1];
    const int skip = unit - (lo / kTokenGroup + 2 * seq);
    lo = lo < 0 ? 0 : lo > p.rows ? p.rows : lo;
    hi = hi < lo ? lo : hi > p.rows ? p.rows : hi;
    const long long start = p.first ? p.first[seq] : 0, end = start + hi - lo;               // positions of the rows
    const long long pos0 = ((start >> 4) + skip) * kTokenGroup;
    if (skip < 0 || pos0 >= end) return;
    const int from = (int)((pos0 > start ? pos0 : start) - pos0), to = (int)((pos0 + kTokenGroup < end ? pos0 + kTokenGroup : end) - pos0);
    const int len = cv.lens[seq];
    // of the group's 16 places, those below `held` hold a token
    const long long left = pos0 < 0 ? 0 : (long long)len - pos0;
    int held = left < 0 ? 0 : left > kTokenGroup ? kTokenGroup : (int)left;
    const int page = held > 0 ? page_of(cv, seq, (int)(pos0 >> cv.page_shift)) : -1;
    if (page < 0) held = 0;
    const int slot0 = (int)(pos0 & ((1 << cv.page_shift) - 1));
    const elem* pool = reinterpret_cast<const elem*>(values ? cv.v : cv.k) + (page < 0 ? 0 : page_at(cv, page, head) + (size_t)slot0 * D);
    const float* scales = TYPE == CODEGEMM_KV_FP16 || page < 0 ? nullptr : (values ? cv.v_scales : cv.k_scales) + scales_at(cv, page, head);
    elem* stage = reinterpret_cast<elem*>(lds);
    constexpr int kVec = 16 / (int)sizeof(elem), kPad = kVec;
    if (values && held > 0) {
        for (int i = tid; i < D * kTokenGroup / kVec; i += kAppendThreads)
            *reinterpret_cast<u32x4_t*>(stage + i * kVec + i * kVec / kTokenGroup / 16 * kPad) = *reinterpret_cast<const u32x4_t*>(pool + i * kVec);
        __syncthreads();
    }
    for (int t0 = from; t0 < to; t0 += per) {
        const int t = t0 + tid / lanes;
        if (t >= to || c >= D / 16) continue;
        half8_t a = {0, 0, 0, 0, 0, 0, 0, 0}, b = a;
        if (t < held) {
            const float s = scales ? scales[(slot0 + t) >> cv.block_shift] : 1.0f;
            alignas(16) elem w[16];
            if (values) {
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = stage[(16 * c + e) * kTokenGroup + c * kPad + t];
            } else {
#pragma unroll
                for (int e = 0; e < 16 / kVec; ++e) *reinterpret_cast<u32x4_t*>(w + e * kVec) = *reinterpret_cast<const u32x4_t*>(pool + (size_t)t * D + 16 * c + e * kVec);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (TYPE == CODEGEMM_KV_FP16) { a[e] = w[e]; b[e] = w[8 + e]; }
                else { a[e] = (_Float16)(value_of<TYPE>(w[e]) * s); b[e] = (_Float16)(value_of<TYPE>(w[8 + e]) * s); }
            }
        }
        _Float16* dst = out + ((size_t)(lo + (int)(pos0 + t - start)) * cv.Hk + head) * D + 16 * c;
        // (stores that stay out of the L2, which holds no result of this size: 48 -> 33 us for 30000 tokens of 8 heads)
        __builtin_nontemporal_store(a, reinterpret_cast<half8_t*>(dst));
        __builtin_nontemporal_store(b, reinterpret_cast<half8_t*>(dst + 8));
    }
}

int check_cache(const codegemm_kv_cache* c, bool pointers)
{
    if (!c) return CODEGEMM_INVALID_ARG;
    if (c->kv_heads < 1 || c->head_dim < 1 || c->num_pages < 1 || c->num_seqs < 1 || c->max_pages < 1) return CODEGEMM_INVALID_ARG;
    if (c->dtype < CODEGEMM_KV_FP16 || c->dtype > CODEGEMM_KV_FP8) return CODEGEMM_UNSUPPORTED;
    if (c->page_size < kTokenGroup || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return CODEGEMM_UNSUPPORTED;
    if (c->head_dim % 16 || c->head_dim > kMaxHeadDim || c->kv_heads > kMaxHeads) return CODEGEMM_UNSUPPORTED;
    if (c->num_pages > 1 << 30 || c->num_seqs > kMaxSeqs || (long long)c->max_pages * c->page_size > 1ll << 30) return CODEGEMM_UNSUPPORTED;
    if (c->dtype != CODEGEMM_KV_FP16 && (c->scale_block < 1 || c->scale_block > c->page_size || (c->scale_block & (c->scale_block - 1)))) return CODEGEMM_UNSUPPORTED;
    if (!pointers) return CODEGEMM_OK;
    if (!c->k || !c->v || !c->page_table || !c->kv_lens || misaligned(c->k) || misaligned(c->v) || misaligned_ints(c->page_table) || misaligned_ints(c->kv_lens))
        return CODEGEMM_INVALID_ARG;
    if (c->dtype != CODEGEMM_KV_FP16 && (!c->k_scales || !c->v_scales || misaligned(c->k_scales) || misaligned(c->v_scales))) return CODEGEMM_INVALID_ARG;
    return CODEGEMM_OK;
}

static int log2_of(int x)
{
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

CacheView cache_view(const codegemm_kv_cache& c)
{
    CacheView v;
    v.k = static_cast<unsigned char*>(c.k);
    v.v = static_cast<unsigned char*>(c.v);
    v.k_scales = c.k_scales;
    v.v_scales = c.v_scales;
    v.table = c.page_table;
    v.lens = c.kv_lens;
    v.Hk = c.kv_heads; v.D = c.head_dim; v.pages = c.num_pages; v.max_pages = c.max_pages; v.seqs = c.num_seqs;
    v.page_shift = log2_of(c.page_size);
    v.block_shift = c.dtype == CODEGEMM_KV_FP16 ? v.page_shift : log2_of(c.scale_block);
    return v;
}

// Lanes of a row: each has 16 of its elements, and the lanes that exchange sums are a power of two.
static int row_lanes(int D) { return 1 << log2_of(D / 16); }

}  // namespace cg

using namespace cg;

extern "C" size_t codegemm_kv_pool_bytes(const codegemm_kv_cache* c)
{
    if (check_cache(c, false)) return 0;
    return (size_t)c->num_pages * c->kv_heads * c->page_size * c->head_dim * (c->dtype == CODEGEMM_KV_FP16 ? 2 : 1);
}

extern "C" size_t codegemm_kv_scales_bytes(const codegemm_kv_cache* c)
{
    if (check_cache(c, false) || c->dtype == CODEGEMM_KV_FP16) return 0;
    return (size_t)c->num_pages * c->kv_heads * (c->page_size / c->scale_block) * sizeof(float);
}

extern "C" int codegemm_kv_append(const codegemm_kv_cache* cache, const codegemm_append_desc* desc, const int32_t* cu_seqlens, const void* q,
                                  const void* k, const void* v, const void* q_norm, const void* k_norm, const float* rope, void* q_out, void* k_out,
                                  void* stream)
{
    const int st = check_cache(cache, true);
    if (st) return st;
    if (!desc || !k || !v || misaligned(k) || misaligned(v)) return CODEGEMM_INVALID_ARG;
    const codegemm_append_desc& d = *desc;
    const int D = cache->head_dim, Hk = cache->kv_heads;
    if (d.tokens < 1 || d.q_heads < 0 || d.rotary_dim < 0 || d.rotary_dim > D || !(d.norm_eps >= 0.0f) || (d.flags & ~CODEGEMM_ROPE_INTERLEAVED)) return CODEGEMM_INVALID_ARG;
    if (d.tokens > kMaxTokens || d.q_heads > kMaxHeads || d.rotary_dim % 16) return CODEGEMM_UNSUPPORTED;
    if (!cu_seqlens && d.tokens != cache->num_seqs) return CODEGEMM_INVALID_ARG;
    if (cu_seqlens && misaligned_ints(cu_seqlens)) return CODEGEMM_INVALID_ARG;
    if (d.q_heads > 0 && (!q || !q_out || misaligned(q) || misaligned(q_out))) return CODEGEMM_INVALID_ARG;
    if (d.rotary_dim > 0 && (!rope || misaligned(rope) || d.rope_positions < 1)) return CODEGEMM_INVALID_ARG;
    if ((q_norm && misaligned(q_norm)) || (k_norm && misaligned(k_norm)) || (k_out && misaligned(k_out))) return CODEGEMM_INVALID_ARG;
    if (bad_stride(d.q_stride, d.q_heads * D) || bad_stride(d.k_stride, Hk * D) || bad_stride(d.v_stride, Hk * D) ||
        bad_stride(d.q_out_stride, d.q_heads * D) || bad_stride(d.k_out_stride, Hk * D))
        return CODEGEMM_INVALID_ARG;
    AppendParams p;
    p.c = cache_view(*cache);
    p.cu = cu_seqlens;
    p.q = static_cast<const _Float16*>(q);
    p.k = static_cast<const _Float16*>(k);
    p.v = static_cast<const _Float16*>(v);
    p.q_norm = static_cast<const _Float16*>(q_norm);
    p.k_norm = static_cast<const _Float16*>(k_norm);
    p.rope = rope;
    p.q_out = static_cast<_Float16*>(q_out);
    p.k_out = static_cast<_Float16*>(k_out);
    p.T = d.tokens; p.Hq = d.q_heads; p.R = d.rotary_dim; p.positions = d.rope_positions;
    p.q_stride = row_stride(d.q_stride, d.q_heads * D);
    p.k_stride = row_stride(d.k_stride, Hk * D);
    p.v_stride = row_stride(d.v_stride, Hk * D);
    p.q_out_stride = row_stride(d.q_out_stride, d.q_heads * D);
    p.k_out_stride = row_stride(d.k_out_stride, Hk * D);
    p.interleaved = d.flags & CODEGEMM_ROPE_INTERLEAVED;
    p.eps = d.norm_eps;
    p.row_lanes = row_lanes(D);
    const int block = 1 << p.c.block_shift;
    p.group = cache->dtype == CODEGEMM_KV_FP16 || block < kTokenGroup ? kTokenGroup : block;
    // A sequence of n new tokens touches at most n / group + 2 units, its first unit being number cu / group + 2 i.
    p.units = cu_seqlens ? p.T / p.group + 2 * cache->num_seqs : cache->num_seqs;
    // Few tokens: their heads over several teams.  Many: a team keeps a token's cosines for all its heads.
    const int rows = kAppendThreads / p.row_lanes;
    p.token_split = p.T >= 1024 || p.Hq == 0 ? 1 : ceil_div(p.Hq, rows);
    // Long blocks with many new tokens: a team for each 16 of them, as long as the card has room for all (12 sequences of 4 heads, 2500 tokens: blocks
    // of 256 take 49.8 us with one team, 27.5 with 7; 4 of 8 heads, blocks of 64 30.7 with one, 28.7 with 2; of 32, 27.3 and 28.0).
    const int fresh = ceil_div(p.T, cache->num_seqs), useful = (fresh < p.group ? fresh : p.group) / kTokenGroup;
    const long long room = kTeamsAtOnce / (2ll * p.units * Hk);
    const int teams = useful < 4 ? 1 : room < useful ? (int)room : useful;
    p.teams = teams < 1 ? 1 : teams < kMostTeams ? teams : kMostTeams;
    p.token_blocks = p.Hq > 0 || k_out ? (int)(((long long)p.T * p.token_split + p.teams - 1) / p.teams) : 0;
    const long long blocks = p.token_blocks + 2ll * p.units * Hk;
    if (too_many(blocks, p.teams * kAppendThreads)) return CODEGEMM_UNSUPPORTED;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (cache->dtype == CODEGEMM_KV_FP16) launch_append<CODEGEMM_KV_FP16>(p, (unsigned)blocks, s);
    else if (cache->dtype == CODEGEMM_KV_INT8) launch_append<CODEGEMM_KV_INT8>(p, (unsigned)blocks, s);
    else launch_append<CODEGEMM_KV_FP8>(p, (unsigned)blocks, s);
    return hipGetLastError() == hipSuccess ? CODEGEMM_OK : CODEGEMM_LAUNCH_FAILED;
}

extern "C" int codegemm_kv_gather(const codegemm_kv_cache* cache, int32_t rows, const int32_t* cu_rows, const int32_t* first, void* k_out, void* v_out,
                                  void* stream)
{
    const int st = check_cache(cache, true);
    if (st) return st;
    if (rows < 1 || !cu_rows || misaligned_ints(cu_rows) || (first && misaligned_ints(first)) || (!k_out && !v_out)) return CODEGEMM_INVALID_ARG;
    if ((k_out && misaligned(k_out)) || (v_out && misaligned(v_out))) return CODEGEMM_INVALID_ARG;
    if (rows > kMaxTokens) return CODEGEMM_UNSUPPORTED;
    GatherParams p;
    p.c = cache_view(*cache);
    p.cu = cu_rows;
    p.first = first;
    p.k_out = static_cast<_Float16*>(k_out);
    p.v_out = static_cast<_Float16*>(v_out);
    p.rows = rows;
    p.row_lanes = row_lanes(cache->head_dim);
    const long long blocks = (long long)(rows / kTokenGroup + 2 * cache->num_seqs) * cache->kv_heads;
    if (too_many(blocks, kAppendThreads)) return CODEGEMM_UNSUPPORTED;
    const dim3 grid((unsigned)blocks, 2), threads(kAppendThreads);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (cache->dtype == CODEGEMM_KV_FP16) hipLaunchKernelGGL(kv_gather_kernel<CODEGEMM_KV_FP16>, grid, threads, 0, s, p);
    else if (cache->dtype == CODEGEMM_KV_INT8) hipLaunchKernelGGL(kv_gather_kernel<CODEGEMM_KV_INT8>, grid, threads, 0, s, p);
    else hipLaunchKernelGGL(kv_gather_kernel<CODEGEMM_KV_FP8>, grid, threads, 0, s, p);
    return hipGetLastError() == hipSuccess ? CODEGEMM_OK : CODEGEMM_LAUNCH_FAILED;
}
