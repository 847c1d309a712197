// Attention of one query token per sequence over the paged cache.
//
// A workgroup takes a range of one sequence's keys for up to 16 query heads that share a key head.  Each of its wavefronts works on
// its own on steps of 32 A tokens: scores as S^T = K Q^T on the matrix cores (rows: tokens, columns: query heads), the softmax's
// running maximum and sum per column, and O^T += V^T P^T, whose right operand is what the score tiles leave in the lanes, because
// a step's tokens are dealt out to the lanes' groups g in runs of 8 A: row 4 g + r of score tile n is token 8 A g + 4 n + r, so
// lane group g holds 8 A consecutive tokens of P^T, and, in the value pool's layout (16 tokens innermost), the 8 A tokens of V^T that
// go with them are one or two loads.  Keys, values and weights never pass through LDS, and no wavefront waits for another before the end.
// 8-bit codes become fp16 exactly on the way into the matrix cores; a key's scale multiplies its score, a value's scale its weight.
#include <cmath>

#include "attn_common.h"

namespace cg {

constexpr int kDecodeWaves = 4;
constexpr int kDecodeRows = 16;             // query heads of a workgroup
constexpr int kMaxSplits = 64;
constexpr float kLeastLog = -40.0f;         // of a scale's logarithm in the running maximum

struct DecodeParams {
    CacheView c;
    const _Float16* q;
    _Float16* out;
    float* part;            // [item][split][16][D + 2] of sequences in several ranges: sums, then maximum and weight
    uint32_t* counters;
    int cstride;
    int r;                  // query heads of a key head
    int tiles;              // workgroups of 16 of them
    int q_stride, out_stride;
    int window;
    int min_steps;          // of a range, before there is a second one
    float scale;            // times log2(e)
};

typedef float float2_t __attribute__((ext_vector_type(2)));

// 8 codes to fp16, exactly.
template <int TYPE>
__device__ __forceinline__ half8_t codes_to_half(uint32_t lo, uint32_t hi)
{
    if constexpr (TYPE == CODEGEMM_KV_INT8) {
        // code + 128 in the low byte of 0x6400 is 1024 + code + 128
        const half2_t off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
        lo ^= 0x80808080u;
        hi ^= 0x80808080u;
        const half2_t a = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u)) + off;
        const half2_t b = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u)) + off;
        const half2_t c = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u)) + off;
        const half2_t d = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)) + off;
        return half8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
        const half2_t a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, true);
        const half2_t c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, true);
        return half8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
}

// What one lane holds of a step.  K rows: 16 elements of each of 2 A tokens per 64 dimensions; V: 8 A tokens of one dimension in 16.
template <int TYPE, int DP, int A, int SC>
struct Step {
    static constexpr bool kHalf = TYPE == CODEGEMM_KV_FP16;
    static constexpr int kTiles = 2 * A, kChunks = DP / 64, kBlocks = DP / 16;
    uint32_t k[kTiles][kChunks][kHalf ? 8 : 4];
    uint32_t v[kBlocks][kHalf ? 4 * A : 2 * A];
    float ks[SC == 2 ? 4 * kTiles : 1], vs[SC == 2 ? 4 * kTiles : 1];
    bool ok;                     // the lane group's tokens have a page
};

// TYPE: of the cache.  DP: head_dim rounded up to 64, 128 or 256; EXACT: it is head_dim.  SC: 0 no scales, 1 one for the lane group's
// run of tokens, 2 several.  A: 32 A tokens a step.
template <int TYPE, int DP, int SC, bool EXACT>
__global__ void __launch_bounds__(kDecodeWaves * kWave) attn_decode_kernel(const DecodeParams p)
{
    constexpr int A = TYPE == CODEGEMM_KV_FP16 || DP == 256 || SC == 2 ? 1 : 2;
    constexpr int kRun = 8 * A, kStep = 32 * A, kTiles = 2 * A;
    typedef Step<TYPE, DP, A, SC> stage_t;
    constexpr int kPitch = DP + 4;                                   // floats of a row's sums in LDS
    __shared__ __align__(16) float merge[(kDecodeWaves / 2) * kDecodeRows * kPitch];
    __shared__ float merge_ml[(kDecodeWaves / 2) * kDecodeRows * 2];
    __shared__ uint32_t flag;

    const CacheView& cv = p.c;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int col = lane & 15, g = lane >> 4;
    const int split = blockIdx.x, seq = blockIdx.z, head = blockIdx.y / p.tiles, row0 = (blockIdx.y % p.tiles) * kDecodeRows;
    const int rows = p.r - row0 < kDecodeRows ? p.r - row0 : kDecodeRows;
    const int D = EXACT ? DP : cv.D;

    const int len0 = cv.lens[seq], held = cv.max_pages << cv.page_shift;
    const int len = len0 < 0 ? 0 : len0 < held ? len0 : held;
    const int lo = p.window > 0 && len0 > p.window ? len0 - p.window : 0;
    const int first = lo & ~(kStep - 1);                             // steps start at multiples of their length
    const int steps = len > lo ? (len - first + kStep - 1) / kStep : 0;
    const int by_grid = (steps + (int)gridDim.x - 1) / (int)gridDim.x;
    const int per = by_grid > p.min_steps ? by_grid : p.min_steps;
    const int splits = steps > per ? (steps + per - 1) / per : 1;
    if (split >= splits) return;
    const int s_end = (split + 1) * per < steps ? (split + 1) * per : steps;

    // Q^T: column `col`, dimensions 64 j + 16 g + 8 a .. + 7 for products 2 j + a; zeros beyond the head's rows and dimensions.
    half8_t qf[DP / 32];
#pragma unroll
    for (int j = 0; j < DP / 64; ++j)
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            half8_t w = {0, 0, 0, 0, 0, 0, 0, 0};
            const int d = 64 * j + 16 * g + 8 * a;
            if (col < rows && d < D) w = *reinterpret_cast<const half8_t*>(p.q + (size_t)seq * p.q_stride + (size_t)(head * p.r + row0 + col) * D + d);
            qf[2 * j + a] = w;
        }

    float4_t o[DP / 16];
#pragma unroll
    for (int b = 0; b < DP / 16; ++b) o[b] = float4_t{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;

    // Tokens of runs that start at or past the end take the last run's place: what is loaded there is masked.
    auto run_at = [&](int step, int x) {
        const int t = first + step * kStep + kRun * x;
        return t < len ? t : (len - 1) & ~(kRun - 1);
    };
    auto load = [&](stage_t& st, int step) {
        const int tk = run_at(step, col >> 2), tv = run_at(step, g);
        int pk = page_of(cv, seq, tk >> cv.page_shift), pv = page_of(cv, seq, tv >> cv.page_shift);
        st.ok = pv >= 0;
        pk = pk < 0 ? 0 : pk;
        pv = pv < 0 ? 0 : pv;
        const int in_page = (1 << cv.page_shift) - 1, sk = tk & in_page, sv = tv & in_page;
        constexpr int kSize = stage_t::kHalf ? 2 : 1;
        const unsigned char* kp = cv.k + (page_at(cv, pk, head) + (size_t)(sk + (col & 3)) * D) * kSize;
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int j = 0; j < DP / 64; ++j) {
                const int d = 64 * j + 16 * g;
                const bool in = EXACT || d < D;
                const u32x4_t* src = reinterpret_cast<const u32x4_t*>(kp + (size_t)(4 * n * D + (in ? d : 0)) * kSize);
#pragma unroll
                for (int h = 0; h < kSize; ++h) {
                    const u32x4_t w = src[h];
#pragma unroll
                    for (int e = 0; e < 4; ++e) st.k[n][j][4 * h + e] = in ? w[e] : 0u;
                }
            }
        // [16 tokens of a dimension] in the group of 16 that the run is in
        const unsigned char* vp = cv.v + (page_at(cv, pv, head) + (size_t)(sv & ~(kTokenGroup - 1)) * D + (size_t)col * kTokenGroup + (sv & (kTokenGroup - 1))) * kSize;
#pragma unroll
        for (int b = 0; b < DP / 16; ++b) {
            if (!EXACT && 16 * b >= D) {
#pragma unroll
                for (int e = 0; e < kRun * kSize / 4; ++e) st.v[b][e] = 0;
                continue;
            }
            const unsigned char* src = vp + (size_t)b * 16 * kTokenGroup * kSize;
            if constexpr (kRun * kSize == 8) {
                const u32x2_t w = *reinterpret_cast<const u32x2_t*>(src);
                st.v[b][0] = w[0];
                st.v[b][1] = w[1];
            } else {
#pragma unroll
                for (int h = 0; h < kRun * kSize / 16; ++h) {
                    const u32x4_t w = reinterpret_cast<const u32x4_t*>(src)[h];
#pragma unroll
                    for (int e = 0; e < 4; ++e) st.v[b][4 * h + e] = w[e];
                }
            }
        }
        if constexpr (SC != 0) {
            const float* ksp = cv.k_scales + scales_at(cv, pv, head);
            const float* vsp = cv.v_scales + scales_at(cv, pv, head);
            if constexpr (SC == 1) {
                st.ks[0] = ksp[sv >> cv.block_shift];
                st.vs[0] = vsp[sv >> cv.block_shift];
            } else {
#pragma unroll
                for (int n = 0; n < kTiles; ++n) {
                    const int at = (sv + 4 * n) >> cv.block_shift;
                    float4_t a, b;
                    if (cv.block_shift == 0) {
                        a = *reinterpret_cast<const float4_t*>(ksp + at);
                        b = *reinterpret_cast<const float4_t*>(vsp + at);
                    } else if (cv.block_shift == 1) {
                        const float2_t c = *reinterpret_cast<const float2_t*>(ksp + at), d = *reinterpret_cast<const float2_t*>(vsp + at);
                        a = float4_t{c[0], c[0], c[1], c[1]};
                        b = float4_t{d[0], d[0], d[1], d[1]};
                    } else {
                        const float c = ksp[at], d = vsp[at];
                        a = float4_t{c, c, c, c};
                        b = float4_t{d, d, d, d};
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) { st.ks[4 * n + r] = a[r]; st.vs[4 * n + r] = b[r]; }
                }
            }
        }
    };

    auto compute = [&](stage_t& st, int step) {
        float4_t s[kTiles];
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
            s[n] = float4_t{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < DP / 64; ++j)
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    half8_t kf;
                    if constexpr (stage_t::kHalf) kf = __builtin_bit_cast(half8_t, u32x4_t{st.k[n][j][4 * a], st.k[n][j][4 * a + 1], st.k[n][j][4 * a + 2], st.k[n][j][4 * a + 3]});
                    else kf = codes_to_half<TYPE>(st.k[n][j][2 * a], st.k[n][j][2 * a + 1]);
                    s[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[2 * j + a], s[n], 0, 0, 0);
                }
        }
        const int t0 = first + step * kStep, t = t0 + kRun * g;
        const bool whole = t0 >= lo && t0 + kStep <= len && __all(st.ok);
        float vs[SC == 2 ? 4 * kTiles : 1], lg[SC == 2 ? 4 * kTiles : 1];
#pragma unroll
        for (int i = 0; i < (SC == 2 ? 4 * kTiles : 1); ++i) vs[i] = SC ? st.vs[i] : 1.0f;
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[n][r] *= (SC == 0 ? 1.0f : st.ks[SC == 2 ? 4 * n + r : 0]) * p.scale;
        const int vlo = lo > t ? lo - t : 0, vhi = !st.ok || t >= len ? 0 : len - t;        // of the run's tokens, those that count
        if (!whole) {
#pragma unroll
            for (int n = 0; n < kTiles; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bool seen = 4 * n + r >= vlo && 4 * n + r < vhi;
                    s[n][r] = seen ? s[n][r] : -INFINITY;
                    if (SC == 2) vs[4 * n + r] = seen ? vs[4 * n + r] : 0.0f;
                }
            if (SC == 1) vs[0] = vhi > vlo ? vs[0] : 0.0f;
            // values that do not count are zeros: what lies there may be a NaN
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                const bool seen = i >= vlo && i < vhi;
#pragma unroll
                for (int b = 0; b < DP / 16; ++b) {
                    if constexpr (stage_t::kHalf) st.v[b][i / 2] = seen ? st.v[b][i / 2] : st.v[b][i / 2] & (i & 1 ? 0x0000ffffu : 0xffff0000u);
                    else st.v[b][i / 4] = seen ? st.v[b][i / 4] : st.v[b][i / 4] & ~(0xffu << (8 * (i & 3)));
                }
            }
        }
        // The maximum is taken over score + log2 of the value's scale, so that weight times scale, rounded to fp16, is at most 1.
        float most = -INFINITY;
        if constexpr (SC != 0) {
#pragma unroll
            for (int i = 0; i < (SC == 2 ? 4 * kTiles : 1); ++i) lg[i] = fmaxf(__builtin_amdgcn_logf(vs[i]), kLeastLog);
        }
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) most = fmaxf(most, SC == 2 ? s[n][r] + lg[4 * n + r] : s[n][r]);
        if (SC == 1) most += lg[0];
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const float m_new = fmaxf(m, most), base = m_new == -INFINITY ? 0.0f : m_new;
        const float keep = __builtin_amdgcn_exp2f(m - base);
        m = m_new;
        float sum = 0.0f;
        half8_t pf[A];
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float w = __builtin_amdgcn_exp2f(s[n][r] - base);
                sum += w;
                pf[n / 2][4 * (n & 1) + r] = (_Float16)(SC == 0 ? w : w * vs[SC == 2 ? 4 * n + r : 0]);
            }
        l = l * keep + sum;
#pragma unroll
        for (int b = 0; b < DP / 16; ++b) {
#pragma unroll
            for (int r = 0; r < 4; ++r) o[b][r] *= keep;
#pragma unroll
            for (int a = 0; a < A; ++a) {
                half8_t vf;
                if constexpr (stage_t::kHalf) vf = __builtin_bit_cast(half8_t, u32x4_t{st.v[b][4 * a], st.v[b][4 * a + 1], st.v[b][4 * a + 2], st.v[b][4 * a + 3]});
                else vf = codes_to_half<TYPE>(st.v[b][2 * a], st.v[b][2 * a + 1]);
                o[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[a], o[b], 0, 0, 0);
            }
        }
    };

    {
        stage_t st0, st1;
        int s = split * per + wave;
        if (s < s_end) load(st0, s);
        while (s < s_end) {
            if (s + kDecodeWaves < s_end) load(st1, s + kDecodeWaves);
            __builtin_amdgcn_sched_barrier(0);
            compute(st0, s);
            s += kDecodeWaves;
            if (s >= s_end) break;
            if (s + kDecodeWaves < s_end) load(st0, s + kDecodeWaves);
            __builtin_amdgcn_sched_barrier(0);
            compute(st1, s);
            s += kDecodeWaves;
        }
    }

    // The lane groups' sums, then the wavefronts': the upper half hands its own to the lower half, in rounds.
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
#pragma unroll
    for (int half = kDecodeWaves / 2; half > 0; half >>= 1) {
        if (wave >= half && wave < 2 * half) {
            float* to = merge + ((wave - half) * kDecodeRows + col) * kPitch;
#pragma unroll
            for (int b = 0; b < DP / 16; ++b) *reinterpret_cast<float4_t*>(to + 16 * b + 4 * g) = o[b];
            if (g == 0) {
                merge_ml[((wave - half) * kDecodeRows + col) * 2] = m;
                merge_ml[((wave - half) * kDecodeRows + col) * 2 + 1] = l;
            }
        }
        __syncthreads();
        if (wave < half) {
            const float* from = merge + (wave * kDecodeRows + col) * kPitch;
            const float m2 = merge_ml[(wave * kDecodeRows + col) * 2], l2 = merge_ml[(wave * kDecodeRows + col) * 2 + 1];
            const float m_new = fmaxf(m, m2), base = m_new == -INFINITY ? 0.0f : m_new;
            const float a = __builtin_amdgcn_exp2f(m - base), c = __builtin_amdgcn_exp2f(m2 - base);
            m = m_new;
            l = l * a + l2 * c;
#pragma unroll
            for (int b = 0; b < DP / 16; ++b) {
                const float4_t w = *reinterpret_cast<const float4_t*>(from + 16 * b + 4 * g);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[b][r] = o[b][r] * a + w[r] * c;
            }
        }
        __syncthreads();
    }

    _Float16* out = p.out + (size_t)seq * p.out_stride + (size_t)(head * p.r + row0) * D;
    if (splits == 1) {
        if (wave == 0 && col < rows) {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
            for (int b = 0; b < DP / 16; ++b)
                if (EXACT || 16 * b < D)
                    *reinterpret_cast<half4_t*>(out + (size_t)col * D + 16 * b + 4 * g) =
                        half4_t{(_Float16)(o[b][0] * inv), (_Float16)(o[b][1] * inv), (_Float16)(o[b][2] * inv), (_Float16)(o[b][3] * inv)};
        }
        return;
    }

    // Several ranges: all data that crosses workgroups is moved by device-scope accesses, acknowledged before the ticket is taken; the
    // last workgroup of the sequence's heads adds the ranges in order and leaves the counter at zero.
    const size_t item = (size_t)seq * gridDim.y + blockIdx.y;
    float* part = p.part + item * gridDim.x * (kDecodeRows * (size_t)(D + 2));
    if (wave == 0 && col < rows) {
        float* to = part + ((size_t)split * kDecodeRows + col) * (D + 2);
        auto put = [&](float* at, float a, float b) {
            const unsigned long long w = (unsigned long long)__builtin_bit_cast(uint32_t, b) << 32 | __builtin_bit_cast(uint32_t, a);
            __hip_atomic_store(reinterpret_cast<unsigned long long*>(at), w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        };
#pragma unroll
        for (int b = 0; b < DP / 16; ++b)
            if (EXACT || 16 * b < D) {
                put(to + 16 * b + 4 * g, o[b][0], o[b][1]);
                put(to + 16 * b + 4 * g + 2, o[b][2], o[b][3]);
            }
        if (g == 0) put(to + D, m, l);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
        uint32_t* ctr = p.counters + item * p.cstride;
        const bool last = __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(splits - 1);
        if (last) __hip_atomic_store(ctr, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        flag = last ? 1u : 0u;
    }
    __syncthreads();
    if (flag == 0u) return;
    auto get = [&](const float* at) {
        return __hip_atomic_load(reinterpret_cast<const unsigned long long*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    auto low = [](unsigned long long w) { return __builtin_bit_cast(float, (uint32_t)w); };
    auto high = [](unsigned long long w) { return __builtin_bit_cast(float, (uint32_t)(w >> 32)); };
    static_assert(kMaxSplits * 2 <= (kDecodeWaves / 2) * (64 + 4), "the ranges' weights fit where the wavefronts' sums were");
    float* ml = merge;                                                // [split][16][2]
    for (int i = tid; i < splits * kDecodeRows; i += kDecodeWaves * kWave) {
        unsigned long long w = 0;
        if (i % kDecodeRows < rows) w = get(part + (size_t)i * (D + 2) + D);
        ml[2 * i] = low(w);
        ml[2 * i + 1] = high(w);
    }
    __syncthreads();
    if (tid < rows) {
        float most = -INFINITY, sum = 0.0f;
        for (int i = 0; i < splits; ++i) most = fmaxf(most, ml[2 * (i * kDecodeRows + tid)]);
        const float base = most == -INFINITY ? 0.0f : most;
        for (int i = 0; i < splits; ++i) {
            const float w = __builtin_amdgcn_exp2f(ml[2 * (i * kDecodeRows + tid)] - base);
            sum += w * ml[2 * (i * kDecodeRows + tid) + 1];
            ml[2 * (i * kDecodeRows + tid)] = w;
        }
        merge_ml[tid] = sum == 0.0f ? 0.0f : 1.0f / sum;
    }
    __syncthreads();
    for (int i = tid; i < rows * (D / 2); i += kDecodeWaves * kWave) {
        const int row = i / (D / 2), d = i % (D / 2) * 2;
        const float* from = part + (size_t)row * (D + 2) + d;
        float a = 0.0f, b = 0.0f;
#pragma unroll 8
        for (int k = 0; k < splits; ++k) {
            const unsigned long long w = get(from + (size_t)k * kDecodeRows * (D + 2));
            const float by = ml[2 * (k * kDecodeRows + row)];
            a += by * low(w);
            b += by * high(w);
        }
        const float inv = merge_ml[row];
        *reinterpret_cast<half2_t*>(out + (size_t)row * D + d) = half2_t{(_Float16)(a * inv), (_Float16)(b * inv)};
    }
}

int check_attn(const codegemm_attn_desc* d)
{
    if (!d) return CODEGEMM_INVALID_ARG;
    if (d->q_heads < 1 || d->kv_heads < 1 || d->head_dim < 1 || d->num_seqs < 1 || d->total_q < 1 || d->total_kv < 0 || d->max_kv < 1 || d->window < 0)
        return CODEGEMM_INVALID_ARG;
    if (d->q_heads % d->kv_heads || (d->flags & ~CODEGEMM_ATTN_CAUSAL) || !std::isfinite(d->scale)) return CODEGEMM_INVALID_ARG;
    if (d->head_dim % 16 || d->head_dim > kMaxHeadDim || d->q_heads > kMaxHeads) return CODEGEMM_UNSUPPORTED;
    if (d->num_seqs > kMaxSeqs || d->total_q > kMaxTokens || d->total_kv > kMaxTokens) return CODEGEMM_UNSUPPORTED;
    const int q = d->q_heads * d->head_dim, kv = d->kv_heads * d->head_dim;
    if (bad_stride(d->q_stride, q) || bad_stride(d->k_stride, kv) || bad_stride(d->v_stride, kv) || bad_stride(d->out_stride, q)) return CODEGEMM_INVALID_ARG;
    return CODEGEMM_OK;
}

namespace {

struct DecodePlan {
    int r, tiles, splits, step, min_steps, cstride;
    size_t bytes;        // of workspace
};

int decode_plan(const codegemm_kv_cache* cache, const codegemm_attn_desc* d, DecodePlan* p)
{
    int st = check_cache(cache, false);
    if (!st) st = check_attn(d);
    if (st) return st;
    if (d->kv_heads != cache->kv_heads || d->head_dim != cache->head_dim || d->num_seqs != cache->num_seqs || d->total_q != d->num_seqs) return CODEGEMM_INVALID_ARG;
    p->r = d->q_heads / d->kv_heads;
    p->tiles = ceil_div(p->r, kDecodeRows);
    const bool half = cache->dtype == CODEGEMM_KV_FP16;
    p->step = half || d->head_dim > 128 || cache->scale_block < kTokenGroup ? 32 : 64;
    // Keys in ranges until the workgroups fill the chip twice, but no range under two steps for each wavefront.
    const int items = d->num_seqs * d->kv_heads * p->tiles;
    const int keys = d->window > 0 && d->window < d->max_kv ? d->window : d->max_kv;
    const int steps = ceil_div(keys, p->step) + 1;
    p->min_steps = 2 * kDecodeWaves;
    int splits = items >= 512 ? 1 : ceil_div(512, items);
    if (splits > ceil_div(steps, p->min_steps)) splits = ceil_div(steps, p->min_steps);
    if (splits > kMaxSplits) splits = kMaxSplits;
    if (items > kCounterAreaWords) splits = 1;
    p->splits = splits;
    p->cstride = items * kCounterStride <= kCounterAreaWords ? kCounterStride : items > 0 && items <= kCounterAreaWords ? kCounterAreaWords / items : 0;
    p->bytes = (size_t)kCounterAreaWords * sizeof(uint32_t) + kPairAreaBytes;
    if (splits > 1) p->bytes += (size_t)items * splits * kDecodeRows * (d->head_dim + 2) * sizeof(float);
    return CODEGEMM_OK;
}

template <int TYPE, int DP, int SC>
void launch_decode(const DecodeParams& p, dim3 grid, hipStream_t s)
{
    const dim3 threads(kDecodeWaves * kWave);
    if (p.c.D == DP) hipLaunchKernelGGL((attn_decode_kernel<TYPE, DP, SC, true>), grid, threads, 0, s, p);
    else hipLaunchKernelGGL((attn_decode_kernel<TYPE, DP, SC, false>), grid, threads, 0, s, p);
}

template <int TYPE, int SC>
void launch_decode_of(const DecodeParams& p, dim3 grid, hipStream_t s)
{
    if (p.c.D <= 64) launch_decode<TYPE, 64, SC>(p, grid, s);
    else if (p.c.D <= 128) launch_decode<TYPE, 128, SC>(p, grid, s);
    else launch_decode<TYPE, 256, SC>(p, grid, s);
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" size_t codegemm_attn_decode_workspace_bytes(const codegemm_kv_cache* cache, const codegemm_attn_desc* desc)
{
    DecodePlan plan;
    return decode_plan(cache, desc, &plan) ? 0 : plan.bytes;
}

extern "C" int codegemm_attn_decode(const codegemm_kv_cache* cache, const codegemm_attn_desc* desc, const void* q, void* out, void* workspace,
                                    size_t workspace_bytes, void* stream)
{
    DecodePlan plan;
    int st = decode_plan(cache, desc, &plan);
    if (!st) st = check_cache(cache, true);
    if (st) return st;
    if (!q || !out || !workspace || misaligned(q) || misaligned(out) || misaligned(workspace)) return CODEGEMM_INVALID_ARG;
    if (workspace_bytes < plan.bytes) return CODEGEMM_WORKSPACE_TOO_SMALL;
    DecodeParams p;
    p.c = cache_view(*cache);
    p.q = static_cast<const _Float16*>(q);
    p.out = static_cast<_Float16*>(out);
    p.counters = static_cast<uint32_t*>(workspace);
    p.part = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + (size_t)kCounterAreaWords * sizeof(uint32_t) + kPairAreaBytes);
    p.cstride = plan.cstride;
    p.r = plan.r;
    p.tiles = plan.tiles;
    p.q_stride = row_stride(desc->q_stride, desc->q_heads * desc->head_dim);
    p.out_stride = row_stride(desc->out_stride, desc->q_heads * desc->head_dim);
    p.window = desc->window;
    p.min_steps = plan.min_steps;
    p.scale = (float)(desc->scale * 1.4426950408889634);
    const dim3 grid((unsigned)plan.splits, (unsigned)(desc->kv_heads * plan.tiles), (unsigned)desc->num_seqs);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool single = cache->scale_block >= kTokenGroup;
    if (cache->dtype == CODEGEMM_KV_FP16) launch_decode_of<CODEGEMM_KV_FP16, 0>(p, grid, s);
    else if (cache->dtype == CODEGEMM_KV_INT8) single ? launch_decode_of<CODEGEMM_KV_INT8, 1>(p, grid, s) : launch_decode_of<CODEGEMM_KV_INT8, 2>(p, grid, s);
    else single ? launch_decode_of<CODEGEMM_KV_FP8, 1>(p, grid, s) : launch_decode_of<CODEGEMM_KV_FP8, 2>(p, grid, s);
    return hipGetLastError() == hipSuccess ? CODEGEMM_OK : CODEGEMM_LAUNCH_FAILED;
}
