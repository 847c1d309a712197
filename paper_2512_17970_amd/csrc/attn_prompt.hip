// Attention of packed prompts: causal, grouped heads, sequences of different lengths.
//
// A workgroup takes 32 NW consecutive queries of one sequence and head, each wavefront 32 of them, and walks over the keys in tiles of
// BN.  S^T = K Q^T (rows: keys, columns: queries) in 32x32x16 products, so a lane holds all its scores for one query, and what the
// running maximum and sum of the softmax need from other lanes is one exchange with the other half of the wavefront.  P^T goes from the
// score tiles into the right operand of O^T += V^T P^T as it lies; V^T comes out of LDS transposed (ds_read_tr16).  Keys and values
// come into LDS by the memory pipeline (buffer_load .. lds), one tile ahead.
//
// Tiles in which some query of the workgroup does not see some key come first.  A value that a query does not see has weight 0 there,
// which leaves its sum alone unless the value is a NaN or an infinity; so the sums are looked at once after these tiles, and where they are
// not all finite, the tiles are run again key by key, each product added only where the query sees the key.
#include "attn_common.h"

namespace cg {

struct PromptParams {
    const _Float16 *q, *k, *v;
    _Float16* out;
    const int32_t *cu_q, *cu_kv;
    int seqs, total_q, total_kv;
    int Hq, Hk, D;
    int q_stride, k_stride, v_stride, out_stride;
    int window, causal;
    int negate;             // a negative scale: of -q
    float scale;            // its size, times log2(e)
    int units;              // query tiles, at most
};

typedef __attribute__((address_space(3))) half8_t lds_h8;
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t lds_s4;
typedef __attribute__((address_space(3))) unsigned char lds_byte;

// Resource words of the 32-bit addressed buffer [base, base + bytes).
__device__ __forceinline__ u32x4_t tile_words(const void* base, uint32_t bytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    u32x4_t words = {(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a), (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu)),
                     (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
    asm volatile("s_nop 4" : "+s"(words));
    return words;
}

// 16 bytes per lane from voff of the buffer to LDS byte address lds + 16 lane; zeros where voff is past the buffer's end.
__device__ __forceinline__ void tile_to_lds(uint32_t lds, int voff, u32x4_t words)
{
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "{m0}"(lds), "v"(voff), "s"(words) : "memory");
}

template <int DP, int NW>
struct PromptTile {
    static constexpr int kRows = 32 * NW;                 // queries of a workgroup
    static constexpr int kKeys = DP == 256 ? 32 : 64;     // BN
    static constexpr int kUnits = DP / 8;                 // 16-byte units of a row
    static constexpr int kBytes = kKeys * DP * 2;         // of a tile of keys, or of values
    static constexpr int kLoads = kBytes / 1024 / NW;     // a wavefront's requests for one of them
    static constexpr int kLds = 4 * kBytes + 16;          // two tiles of each, and a flag
    // Unit u of row `row` lies in place u ^ turn(row): the 8 (16) lanes of a read that the LDS serves together take the same
    // unit of 8 rows (4 halves of 2 units of 4 rows) and find it in different banks.
    __host__ __device__ static constexpr int turn_k(int row) { return row & (kUnits - 1); }
    __host__ __device__ static constexpr int turn_v(int row) { return kUnits == 8 ? row & 6 : 2 * (row & 7); }
};

template <int DP, int NW, bool EXACT>
__global__ void __launch_bounds__(NW * kWave, DP == 256 ? 1 : 2) attn_prompt_kernel(const PromptParams p)
{
    typedef PromptTile<DP, NW> T;
    constexpr int BM = T::kRows, BN = T::kKeys, KB = BN / 32, DB = DP / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((lds_byte*)smem);
    volatile uint32_t* flag = reinterpret_cast<volatile uint32_t*>(smem + 4 * T::kBytes);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int qc = lane & 31, h = lane >> 5;
    const int D = EXACT ? DP : p.D;

    // Workgroups that follow each other land on the 8 XCDs in turn: where the heads divide evenly, an XCD keeps to its own, so
    // that a key head's tiles are read through one L2.  A sequence's last tile, the longest, comes first.
    int head, unit;
    {
        const int id = blockIdx.x;
        if (p.Hq % 8 == 0) {
            const int per = p.Hq / 8, at = id / 8;
            head = id % 8 * per + at % per;
            unit = at / per;
        } else {
            head = id % p.Hq;
            unit = id / p.Hq;
        }
    }
    const int seq = last_at_most(p.seqs, unit, [&](int i) { return p.cu_q[i] / BM + i; });
    auto clamp = [](int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; };
    const int q0 = clamp(p.cu_q[seq], 0, p.total_q), n = clamp(p.cu_q[seq + 1], q0, p.total_q) - q0;
    const int32_t* cu_kv = p.cu_kv ? p.cu_kv : p.cu_q;
    const int k0 = clamp(cu_kv[seq], 0, p.total_kv), n_kv = clamp(cu_kv[seq + 1], k0, p.total_kv) - k0;
    const int tiles = (n + BM - 1) / BM, at = unit - (p.cu_q[seq] / BM + seq);
    if (at < 0 || at >= tiles) return;
    const int row0 = (tiles - 1 - at) * BM;                              // first query of the workgroup
    const int back = n_kv - n;                                           // position of query 0
    const int last = (row0 + BM < n ? row0 + BM : n) - 1;

    // keys that any query of the workgroup sees
    int k_lo = 0, k_hi = n_kv;
    if (p.causal && back + last + 1 < k_hi) k_hi = back + last + 1;
    if (p.window > 0 && back + row0 - p.window + 1 > 0) k_lo = back + row0 - p.window + 1;
    const int t_lo = k_lo / BN, t_hi = k_hi > k_lo ? (k_hi + BN - 1) / BN : t_lo;
    // tiles that all its queries see whole: t_a .. t_b - 1
    int t_a = t_lo, t_b = n_kv / BN;
    if (p.causal && (back + row0 + 1 < 0 ? 0 : (back + row0 + 1) / BN) < t_b) t_b = back + row0 + 1 < 0 ? 0 : (back + row0 + 1) / BN;
    if (p.window > 0 && back + last - p.window >= 0) t_a = (back + last - p.window) / BN + 1;
    if (t_a < t_lo) t_a = t_lo;
    if (t_b > t_hi) t_b = t_hi;
    if (t_b < t_a) t_b = t_a;
    if (t_a > t_hi) t_a = t_b = t_hi;
    const int masked = (t_a - t_lo) + (t_hi - t_b), all = t_hi - t_lo;
    // i-th tile of the walk: above the whole ones from the last down, below them, the whole ones
    auto tile_of = [&](int i) {
        if (i < t_hi - t_b) return t_hi - 1 - i;
        if (i < masked) return t_lo + (i - (t_hi - t_b));
        return t_b - 1 - (i - masked);
    };

    const int kv_head = head / (p.Hq / p.Hk);
    const unsigned char* kbase = reinterpret_cast<const unsigned char*>(p.k + (size_t)k0 * p.k_stride + (size_t)kv_head * D);
    const unsigned char* vbase = reinterpret_cast<const unsigned char*>(p.v + (size_t)k0 * p.v_stride + (size_t)kv_head * D);

    // a wavefront's part of a tile: rows of kUnits places, each request 1 KB of them
    int koff[T::kLoads], voff[T::kLoads];
#pragma unroll
    for (int i = 0; i < T::kLoads; ++i) {
        const int place = (wave * T::kLoads + i) * kWave + lane, row = place / T::kUnits, u = place % T::kUnits;
        const int uk = u ^ T::turn_k(row), uv = u ^ T::turn_v(row);
        koff[i] = EXACT || 8 * uk < D ? row * p.k_stride * 2 + uk * 16 : 0x7ffffff0;
        voff[i] = EXACT || 8 * uv < D ? row * p.v_stride * 2 + uv * 16 : 0x7ffffff0;
    }
    auto request = [&](int tile, int buf) {
        const int t0 = tile * BN, left = n_kv - t0 < BN ? n_kv - t0 : BN;
        const u32x4_t kw = tile_words(kbase + (size_t)t0 * p.k_stride * 2, (uint32_t)((left - 1) * p.k_stride * 2 + D * 2));
        const u32x4_t vw = tile_words(vbase + (size_t)t0 * p.v_stride * 2, (uint32_t)((left - 1) * p.v_stride * 2 + D * 2));
        const uint32_t at_k = lds0 + (uint32_t)(buf * 2 * T::kBytes + wave * T::kLoads * 1024);
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) tile_to_lds(at_k + i * 1024, koff[i], kw);
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) tile_to_lds(at_k + T::kBytes + i * 1024, voff[i], vw);
    };

    // Q^T: column qc, dimensions 16 s + 8 h .. + 7
    half8_t qf[DP / 16];
    const int row = row0 + 32 * wave + qc;
    {
        const _Float16* src = p.q + (size_t)(q0 + (row < n ? row : 0)) * p.q_stride + (size_t)head * D;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            half8_t w = {0, 0, 0, 0, 0, 0, 0, 0};
            const int d = 16 * s + 8 * h;
            if (row < n && (EXACT || d < D)) w = *reinterpret_cast<const half8_t*>(src + d);
            qf[s] = p.negate ? -w : w;
        }
    }
    const int pos = back + row;                                          // the lane's query
    const int wave_first = back + row0 + 32 * wave, wave_last = wave_first + 31;

    float16_t o[DB];
    float m, l;
    auto clear = [&]() {
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[b][e] = 0.0f;
        m = -INFINITY;
        l = 0.0f;
    };
    clear();

    // where the lane's operands lie in a tile
    const uint32_t k_at = lds0 + (uint32_t)(qc * DP * 2);                // + (2 s + h) ^ turn, 32 rows a block
    const int vrow = 4 * h + ((lane & 15) >> 2);                         // + 16 ks, + 8
    const uint32_t v_at = lds0 + (uint32_t)(T::kBytes + vrow * DP * 2 + 8 * (lane & 1));
    const int vunit = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);         // + 4 b
    auto v_operand = [&](int buf, int ks, int b) {
        const uint32_t a = v_at + (uint32_t)(buf * 2 * T::kBytes + ks * 16 * DP * 2) + (uint32_t)(((4 * b + vunit) ^ T::turn_v(vrow)) * 16);
        const uint32_t c = v_at + (uint32_t)(buf * 2 * T::kBytes + (ks * 16 + 8) * DP * 2) + (uint32_t)(((4 * b + vunit) ^ T::turn_v(vrow + 8)) * 16);
        const short4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(uintptr_t)a);
        const short4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(uintptr_t)c);
        return __builtin_bit_cast(half8_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto sees = [&](int key) { return key < n_kv && (!p.causal || key <= pos) && (p.window == 0 || key > pos - p.window); };

    auto compute = [&](int tile, int buf, bool is_masked, bool by_key) {
        const int t0 = tile * BN;
        if (is_masked && ((p.causal && t0 > wave_last) || (p.window > 0 && t0 + BN - 1 <= wave_first - p.window))) return;   // none of the wavefront's
        float16_t s[KB];
#pragma unroll
        for (int b = 0; b < KB; ++b) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[b][e] = 0.0f;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                const half8_t kf = *(const lds_h8*)(uintptr_t)(k_at + (uint32_t)(buf * 2 * T::kBytes + b * 32 * DP * 2) + (uint32_t)(((2 * i + h) ^ T::turn_k(32 * b + qc)) * 16));
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[i], s[b], 0, 0, 0);
            }
        }
        if (is_masked) {
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!sees(t0 + 32 * b + 8 * (e / 4) + 4 * h + e % 4)) s[b][e] = -INFINITY;
        }
        float most = -INFINITY;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) most = fmaxf(most, s[b][e]);
        {
            const uint32_t w = __builtin_bit_cast(uint32_t, most);
            const auto x = __builtin_amdgcn_permlane32_swap(w, w, false, false);
            most = fmaxf(__builtin_bit_cast(float, (uint32_t)x[0]), __builtin_bit_cast(float, (uint32_t)x[1]));
        }
        const float m_new = fmaxf(m, most), base = m_new == -INFINITY ? 0.0f : m_new;
        const float keep = __builtin_amdgcn_exp2f((m - base) * p.scale);
        m = m_new;
        const float shift = -base * p.scale;
        float sum = 0.0f;
        half8_t pf[BN / 16];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][e], p.scale, shift));
                sum += w;
                pf[2 * b + e / 8][e % 8] = (_Float16)w;
            }
        l = l * keep + sum;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[b][e] *= keep;
        if (!by_key) {
#pragma unroll
            for (int ks = 0; ks < BN / 16; ++ks)
#pragma unroll
                for (int b = 0; b < DB; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v_operand(buf, ks, b), pf[ks], o[b], 0, 0, 0);
        } else {
#pragma unroll
            for (int ks = 0; ks < BN / 16; ++ks)
                for (int j = 0; j < 16; ++j) {                           // one key of the 16, in both operands
                    const bool seen = sees(t0 + 16 * ks + j);
                    half8_t one = pf[ks];
#pragma unroll
                    for (int e = 0; e < 8; ++e) one[e] = 8 * (e / 4) + 4 * h + e % 4 == j && seen ? one[e] : (_Float16)0.0f;
#pragma unroll
                    for (int b = 0; b < DB; ++b) {
                        half8_t v = v_operand(buf, ks, b);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = 8 * (e / 4) + 4 * h + e % 4 == j ? v[e] : (_Float16)0.0f;
                        float16_t x;
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = 0.0f;
                        x = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, one, x, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[b][e] += seen ? x[e] : 0.0f;
                    }
                }
        }
    };

    // The tile of step i is in LDS when all wavefronts have waited for their own requests and met; then the next one's requests
    // go to the buffer that all have finished reading.
    auto arrive = [&]() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    bool by_key = false;
    if (all > 0) {
        for (;;) {
            request(tile_of(0), 0);
            int i = 0;
            for (; i < masked; ++i) {
                arrive();
                if (i + 1 < all) request(tile_of(i + 1), (i + 1) & 1);
                compute(tile_of(i), i & 1, true, by_key);
            }
            if (!by_key && masked > 0) {
                float probe = 0.0f;
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) probe = __builtin_fmaf(o[b][e], 0.0f, probe);
                if (tid == 0) *flag = 0;
                __syncthreads();
                if (__any(probe != 0.0f) && lane == 0) *flag = 1;        // a NaN: 0 times a NaN or an infinity
                arrive();
                if (*flag != 0) {
                    __syncthreads();
                    clear();
                    by_key = true;
                    continue;
                }
                __syncthreads();
            }
            for (; i < all; ++i) {
                arrive();
                if (i + 1 < all) request(tile_of(i + 1), (i + 1) & 1);
                compute(tile_of(i), i & 1, false, false);
            }
            break;
        }
    }

    {
        const uint32_t w = __builtin_bit_cast(uint32_t, l);
        const auto x = __builtin_amdgcn_permlane32_swap(w, w, false, false);
        l = __builtin_bit_cast(float, (uint32_t)x[0]) + __builtin_bit_cast(float, (uint32_t)x[1]);
    }
    if (row >= n) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    _Float16* out = p.out + (size_t)(q0 + row) * p.out_stride + (size_t)head * D;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int d = 32 * b + 2 * e + 4 * h;
            if (EXACT || d < D)
                *reinterpret_cast<half4_t*>(out + d) = half4_t{(_Float16)(o[b][e] * inv), (_Float16)(o[b][e + 1] * inv), (_Float16)(o[b][e + 2] * inv), (_Float16)(o[b][e + 3] * inv)};
        }
}

int set_max_lds(const void* fn, size_t bytes);

namespace {

template <int DP, int NW, bool EXACT>
int launch_prompt_one(PromptParams p, const codegemm_attn_desc& d, hipStream_t s)
{
    typedef PromptTile<DP, NW> T;
    auto fn = attn_prompt_kernel<DP, NW, EXACT>;
    const int st = set_max_lds(reinterpret_cast<const void*>(fn), T::kLds);
    if (st) return st;
    // n queries are at most n / kRows + 1 tiles, the first of a sequence being number cu_q / kRows + i
    p.units = d.total_q / T::kRows + d.num_seqs;
    const long long blocks = (long long)p.units * d.q_heads;
    if (blocks > 0x7fffffffll) return CODEGEMM_UNSUPPORTED;
    hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(NW * kWave), T::kLds, s, p);
    return hipGetLastError() == hipSuccess ? CODEGEMM_OK : CODEGEMM_LAUNCH_FAILED;
}

template <int DP, int NW>
int launch_prompt(const PromptParams& p, const codegemm_attn_desc& d, hipStream_t s)
{
    return d.head_dim == DP ? launch_prompt_one<DP, NW, true>(p, d, s) : launch_prompt_one<DP, NW, false>(p, d, s);
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" size_t codegemm_attn_prompt_workspace_bytes(const codegemm_attn_desc* desc)
{
    if (check_attn(desc)) return 0;
    return (size_t)kCounterAreaWords * sizeof(uint32_t) + kPairAreaBytes;
}

extern "C" int codegemm_attn_prompt(const codegemm_attn_desc* desc, const void* q, const void* k, const void* v, const int32_t* cu_q,
                                    const int32_t* cu_kv, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    const int st = check_attn(desc);
    if (st) return st;
    const codegemm_attn_desc& d = *desc;
    if (!q || !out || !cu_q || !workspace || misaligned(q) || misaligned(out) || misaligned(workspace) || misaligned_ints(cu_q)) return CODEGEMM_INVALID_ARG;
    if (d.total_kv > 0 && (!k || !v || misaligned(k) || misaligned(v))) return CODEGEMM_INVALID_ARG;
    if (cu_kv ? misaligned_ints(cu_kv) : d.total_kv != d.total_q) return CODEGEMM_INVALID_ARG;
    if (workspace_bytes < codegemm_attn_prompt_workspace_bytes(desc)) return CODEGEMM_WORKSPACE_TOO_SMALL;
    PromptParams p;
    p.q = static_cast<const _Float16*>(q);
    p.k = static_cast<const _Float16*>(k);
    p.v = static_cast<const _Float16*>(v);
    p.out = static_cast<_Float16*>(out);
    p.cu_q = cu_q;
    p.cu_kv = cu_kv;
    p.seqs = d.num_seqs; p.total_q = d.total_q; p.total_kv = d.total_kv;
    p.Hq = d.q_heads; p.Hk = d.kv_heads; p.D = d.head_dim;
    p.q_stride = row_stride(d.q_stride, d.q_heads * d.head_dim);
    p.k_stride = row_stride(d.k_stride, d.kv_heads * d.head_dim);
    p.v_stride = row_stride(d.v_stride, d.kv_heads * d.head_dim);
    p.out_stride = row_stride(d.out_stride, d.q_heads * d.head_dim);
    p.window = d.window < kMaxTokens ? d.window : 0;               // one that reaches past every key is none
    p.causal = d.flags & CODEGEMM_ATTN_CAUSAL;
    p.negate = d.scale < 0.0f;
    const float size = d.scale < 0.0f ? -d.scale : d.scale;
    p.scale = (float)((size > 1e-30f ? size : 1e-30f) * 1.4426950408889634);      // not 0: 0 times an infinite maximum is no number
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (d.head_dim <= 64) return launch_prompt<64, 4>(p, d, s);
    if (d.head_dim <= 128) return launch_prompt<128, 4>(p, d, s);
    return launch_prompt<256, 4>(p, d, s);
}
