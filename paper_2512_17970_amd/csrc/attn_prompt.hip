// Attention of packed prompts: causal, grouped heads, sequences of different lengths.
//
// A workgroup takes 32 NW rows, each wavefront 32 of them: the query heads of one key head for some consecutive queries of a sequence, head after
// head for each query (with a tile of queries to each head, 256 prompts of 128 tokens, 32 and 8 heads, took 190 us, so 170: fewer tiles that are part
// full, fewer keys that only some rows see).  It walks over the keys in tiles of
// BN.  S^T = K Q^T (rows: keys, columns: queries) in 32x32x16 products, so a lane holds all its scores for one query, and what the
// softmax's running maximum and sum need from other lanes is one exchange with the other half of the wavefront.  P^T goes from the
// score tiles into the right operand of O^T += V^T P^T as it lies; V^T comes out of LDS transposed (ds_read_tr16).  Keys and values
// come into LDS by the memory pipeline (buffer_load .. lds), one tile ahead.  A wavefront goes on in blocks of 32 keys, three at a time: the
// scores of one and the product of another's weights with its values on the matrix cores, the weights of the one between by vector
// instructions; none waits for the others.  (Matrix and vector instructions of one wavefront overlap; those of two disturb each other.)
// What weights are scaled by follows the scores only where one would pass 2^kReach, so that the sums are seldom rescaled.
//
// Tiles in which some query of the workgroup does not see some key come first.  A value that a query does not see has weight 0 there,
// which leaves its sum alone unless the value is a NaN or an infinity; so the sums are looked at once after these tiles, and where they are
// not all finite, the tiles are run again key by key, each product added only where the query sees the key.
//
// Why 32 rows a wavefront and four of those: S^T and O^T of 32 rows and 128 dimensions take 96 registers, Q^T and the weights 48, which
// leaves room for two wavefronts on a SIMD; two workgroups on a compute unit fill each other's waits (one of 8 wavefronts: 1134 for 1117 us, of 2:
// 1634), and 128 rows share a tile of keys and values in LDS.
// Bound by: power, where sequences are long.  8192 causal queries, 64 and 8 heads of 128: 1095 to 1180 us from card to card, 0.93 to 1.00 PFLOP/s (a
// library product of 8192^3 reaches 1.12; launches apart from each other, under a tracer, take up to 1270), the matrix cores busy in 52 % of the cycles at
// 1.7 GHz; all zeros take 943 us.  Of ragged prompts of 500 to 1100 tokens, 32 and 8 heads: 69 to 76 us, 0.61 to 0.68 PFLOP/s; a tile of rows costs
// some 7 us besides its keys.
// Heads of 64: 640 to 680 us for 8192 queries of 64 heads, 0.81 to 0.86 PFLOP/s, 49 us for 4 x 2048 of 32, 0.52 (as many vector instructions a score as
// for 128, for half the products).  Of 256: 3.10 ms and 0.71 PFLOP/s, 118 us for 4 x 2048 of 16, 0.43: one wavefront a SIMD, which has 512 registers
// and spills 7.  Of 80, worked on as 128: 71 us for 4 x 2048 of 32, 0.45.
#include "attn_common.h"

namespace cg {

struct PromptParams {
    const _Float16 *q, *k, *v;
    _Float16* out;
    const int32_t *cu_q, *cu_kv;
    int seqs, total_q, total_kv;
    int Hk, r, D;           // r: query heads of a key head
    float by_r;             // 1 / r
    int q_stride, k_stride, v_stride, out_stride;
    int window, causal;
    int negate;             // a negative scale: of -q
    float scale;            // its size, times log2(e)
    float unit;             // 1 / scale
    int splits;             // workgroups of a tile of queries and head, at most
    float* part;            // [item][split][NW][DP / 8][64 lanes][4] sums, [NW][64] maximum and weight
    uint32_t* counters;     // of an item
};

// Where there are fewer than kPromptItems tiles of queries and heads, as many workgroups as run at once share the keys of each, and the last of them
// to end adds the parts up, in order.  A tile of keys takes about twice what adding a part does, so that sqrt(2 tiles) parts are best, of kLeastTiles
// at least: 16 queries behind 8000 keys, 64 and 8 heads: 162 us in one, 38 in 32 parts, 31 in 16; a prompt of 953, 7 heads: 19.3 in parts
// of 8 tiles, 17.5 of 3.
constexpr int kPromptItems = 256, kLeastTiles = 3;
constexpr int prompt_groups(int dp) { return dp == 256 ? 256 : 512; }        // that run at once
__host__ __device__ inline int parts_worth(int tiles)
{
    const int most = (tiles + kLeastTiles - 1) / kLeastTiles, best = (int)__builtin_sqrtf(2.0f * (float)tiles) + 1;
    return most < 1 ? 1 : most < best ? most : best;
}

// A query's largest weight so far is between 2^(kLift - 1) and 2^kReach: fp16 holds weights down to 2^-24 of it with all their places, and down to 2^-34 at
// all.  Behind one key that has most of the weight and values near zero, thousands of others with little weight each make the result.  (With 1 to 2^8 for the
// largest, 50000 keys 12.5 nats below such a key lost 0.7 % of their weight, at 17 it was off by 44 %, and zero at 18.  The further kReach is from kLift,
// the seldomer weights are rescaled: 8192 queries of 64 heads take 1143 us, 1131 with 8 powers of two between them, 3 % more than that with 2.)
constexpr float kLift = 11.0f, kReach = 15.9f;
// From this size on, times scale, scores have too few places for that: weights are those of the differences from the largest score.
constexpr float kFine = 65536.0f;
constexpr float kNone = -3.402823466e38f;               // the logarithm of nothing

constexpr int kLdsReads = 0x100, kProducts = 0x8;       // groups of instructions, for the scheduler

typedef __attribute__((address_space(3))) half8_t lds_h8;
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t lds_s4;
typedef __attribute__((address_space(3))) unsigned char lds_byte;

// Resource words of the 32-bit addressed buffer [base, base + bytes).
__device__ __forceinline__ u32x4_t tile_words(const void* base, uint32_t bytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    u32x4_t words = {(uint32_t)a, (uint32_t)(a >> 32) & 0xffffu, bytes, 0x00020000u};
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
    static constexpr int kKeys = 64;                      // BN
    static constexpr int kUnits = DP / 8;                 // 16-byte units of a row
    static constexpr int kBytes = kKeys * DP * 2;         // of a tile of keys, or of values
    static constexpr int kLoads = kBytes / 1024 / NW;     // a wavefront's requests for one of them
    static constexpr int kLds = 4 * kBytes + 16;          // two tiles of each, a flag
    // Unit u of row `row` lies in place u ^ turn(row): the 16 lanes that the LDS serves together take the same unit of 16 rows of keys, the 32 take
    // 4 units of 4 rows of values, and find them in different banks (256 bytes of them).
    __host__ __device__ static constexpr int turn_k(int row) { return kUnits == 8 ? (row >> 1) & 7 : row & 15; }
    __host__ __device__ static constexpr int turn_v(int row) { return kUnits == 8 ? 4 * ((row >> 1) & 1) : 4 * (row & 3); }
    static constexpr int kRowsPerLoad = 64 / kUnits;      // rows of a request
    // requests after which the turns repeat: rows 16 apart for keys, 4 for values
    static constexpr int kTurnsK = 16 / kRowsPerLoad < kLoads ? 16 / kRowsPerLoad : kLoads;
    static constexpr int kTurnsV = kRowsPerLoad >= 4 ? 1 : 4 / kRowsPerLoad;
};

template <int DP, int NW, bool EXACT>
__global__ void __launch_bounds__(NW * kWave, DP == 256 ? 1 : 2) attn_prompt_kernel(const PromptParams p)
{
    typedef PromptTile<DP, NW> T;
    constexpr int BM = T::kRows, BN = T::kKeys, DB = DP / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((lds_byte*)smem);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int qc = lane & 31, h = lane >> 5;
    const int D = EXACT ? DP : p.D;

    // Workgroups that follow each other land on the 8 XCDs in turn: where the key heads divide evenly, an XCD keeps to its own, so that a key
    // head's tiles are read through one L2.
    int head, unit, split = 0;                                           // key head
    {
        const int id = blockIdx.x;
        if (p.Hk % 8 == 0) {
            const int per = p.Hk / 8;
            unit = id / 8;
            head = id % 8 * per + unit % per;
            unit /= per;
        } else {
            head = id % p.Hk;
            unit = id / p.Hk;
        }
        if (p.splits > 1) {
            split = unit % p.splits;
            unit /= p.splits;
        }
    }
    auto clamp = [](int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; };
    // A sequence's last tile, which sees most keys, comes first: it is under way when the workgroups run out.  (The last tiles of all sequences before
    // their others were slower: 256 for 248 us with 4 sequences of 2048, more keys at once in an L2.)
    // (Up to 64 sequences: one load of all their ends; more: a search, and scalar loads of the one that is found.)
    auto first_of = [&](int q, int seq) { return (int)((long long)q * p.r / BM) + seq; };        // a sequence's first tile is at most this one
    int q0, q1, k0, k1, at;
    if (p.seqs <= kWave) {
        const int32_t* ends = p.cu_kv ? p.cu_kv : p.cu_q;
        int from = 0, to = 0, kv_from = 0, kv_to = 0;
        if (lane < p.seqs) {
            from = p.cu_q[lane];
            to = p.cu_q[lane + 1];
            kv_from = ends[lane];
            kv_to = ends[lane + 1];
        }
        const int first = first_of(from, lane);
        const int below = __popcll(__ballot(lane < p.seqs && first <= unit)), seq = below > 0 ? below - 1 : 0;
        at = unit - __builtin_amdgcn_readlane(first, seq);
        q0 = __builtin_amdgcn_readlane(from, seq);
        q1 = __builtin_amdgcn_readlane(to, seq);
        k0 = __builtin_amdgcn_readlane(kv_from, seq);
        k1 = __builtin_amdgcn_readlane(kv_to, seq);
    } else {
        typedef __attribute__((address_space(4))) const int32_t const_int;
        const_int *cu_q = (const_int*)(uintptr_t)p.cu_q, *cu_kv = p.cu_kv ? (const_int*)(uintptr_t)p.cu_kv : cu_q;
        const int seq = last_at_most(p.seqs, unit, [&](int i) { return first_of(p.cu_q[i], i); });
        q0 = cu_q[seq];
        q1 = cu_q[seq + 1];
        k0 = cu_kv[seq];
        k1 = cu_kv[seq + 1];
        at = unit - first_of(q0, seq);
    }
    q0 = clamp(q0, 0, p.total_q);
    k0 = clamp(k0, 0, p.total_kv);
    const int n = clamp(q1, q0, p.total_q) - q0, n_kv = clamp(k1, k0, p.total_kv) - k0;
    const int rows = n * p.r, tiles = (rows + BM - 1) / BM;              // (the host sees to it that this is less than 2^31)
    if (at < 0 || at >= tiles) return;
    const int row0 = (tiles - 1 - at) * BM, rows_here = rows - row0 < BM ? rows - row0 : BM;
    const int first = row0 / p.r, ahead = row0 - first * p.r;            // its first query, and the rows of that one that are not the workgroup's
    // The query of a row of the workgroup, counted from the first: a quotient of numbers under 2^11, which the product with the reciprocal is exact for.
    auto query_of = [&](int r) __attribute__((always_inline)) { return (int)(((float)(ahead + r) + 0.5f) * p.by_r); };
    const int back = n_kv - n;                                           // position of query 0
    const int last = first + __builtin_amdgcn_readfirstlane(query_of(rows_here - 1));

    // keys that any query of the workgroup sees
    int k_lo = 0, k_hi = n_kv;
    if (p.causal && back + last + 1 < k_hi) k_hi = back + last + 1;
    if (p.window > 0 && back + first - p.window + 1 > 0) k_lo = back + first - p.window + 1;
    const int t_lo = k_lo / BN, t_hi = k_hi > k_lo ? (k_hi + BN - 1) / BN : t_lo;
    // tiles that all its queries see whole: t_a .. t_b - 1
    int t_a = t_lo, t_b = n_kv / BN;
    if (p.causal && (back + first + 1 < 0 ? 0 : (back + first + 1) / BN) < t_b) t_b = back + first + 1 < 0 ? 0 : (back + first + 1) / BN;
    if (p.window > 0 && back + last - p.window >= 0) t_a = (back + last - p.window) / BN + 1;
    if (t_a < t_lo) t_a = t_lo;
    if (t_b > t_hi) t_b = t_hi;
    if (t_b < t_a) t_b = t_a;
    if (t_a > t_hi) t_a = t_b = t_hi;
    const int masked = (t_a - t_lo) + (t_hi - t_b), walk = t_hi - t_lo;
    // i-th tile of the walk: above the whole ones from the last down, below them, the whole ones
    auto tile_of = [&](int i) __attribute__((always_inline)) {
        if (i < t_hi - t_b) return t_hi - 1 - i;
        if (i < masked) return t_lo + (i - (t_hi - t_b));
        return t_b - 1 - (i - masked);
    };

    // the workgroup's part of the walk
    int parts = 1, begin = 0, all = walk;
    if (p.splits > 1) {
        const int worth = parts_worth(walk);
        parts = worth < p.splits ? worth : p.splits;
        if (split >= parts) return;
        begin = walk * split / parts;
        all = walk * (split + 1) / parts;
    }

    const unsigned char* kbase = reinterpret_cast<const unsigned char*>(p.k + (size_t)k0 * p.k_stride + (size_t)head * D);
    const unsigned char* vbase = reinterpret_cast<const unsigned char*>(p.v + (size_t)k0 * p.v_stride + (size_t)head * D);

    // a wavefront's part of a tile: rows of kUnits places, each request 1 KB of them
    int koff[T::kTurnsK], voff[T::kTurnsV];
    const int load_row = wave * T::kLoads * T::kRowsPerLoad + lane / T::kUnits, load_unit = lane % T::kUnits;
#pragma unroll
    for (int i = 0; i < T::kTurnsK; ++i) {
        const int row = load_row + i * T::kRowsPerLoad, u = load_unit ^ T::turn_k(row);
        koff[i] = EXACT || 8 * u < D ? row * p.k_stride * 2 + u * 16 : 0x7f000000;
    }
#pragma unroll
    for (int i = 0; i < T::kTurnsV; ++i) {
        const int row = load_row + i * T::kRowsPerLoad, u = load_unit ^ T::turn_v(row);
        voff[i] = EXACT || 8 * u < D ? row * p.v_stride * 2 + u * 16 : 0x7f000000;
    }
    // keys in buffers 0 and 1, values in 2 and 3
    // left: keys from the tile's first on
    auto request = [&](const unsigned char* tile, int stride, const int* off, int turns, int left, int buf) __attribute__((always_inline)) {
        const u32x4_t words = tile_words(tile, (uint32_t)(((left < BN ? left : BN) - 1) * stride * 2 + D * 2));
        const uint32_t to = lds0 + (uint32_t)(buf * T::kBytes + wave * T::kLoads * 1024);
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) tile_to_lds(to + i * 1024, off[i % turns] + i / turns * turns * T::kRowsPerLoad * 2 * stride, words);
    };
    const int64_t k_step = (int64_t)BN * p.k_stride * 2, v_step = (int64_t)BN * p.v_stride * 2;
    auto request_k = [&](int tile, int buf) __attribute__((always_inline)) { request(kbase + tile * k_step, p.k_stride, koff, T::kTurnsK, n_kv - tile * BN, buf); };
    auto request_v = [&](int tile, int buf) __attribute__((always_inline)) { request(vbase + tile * v_step, p.v_stride, voff, T::kTurnsV, n_kv - tile * BN, 2 + buf); };

    // The first tile, and Q: a wavefront's own rows to the places of its parts of the second one, 16 to a buffer, in the order of keys.  (Loaded row by
    // row into registers, an instruction would touch 32 lines for 1 KB.)
    const int row = 32 * wave + qc;                                      // the lane's, of the workgroup's
    const uint32_t own = lds0 + (uint32_t)(wave * T::kLoads * 1024);
    if (begin < all) {
        request_k(tile_of(begin), begin & 1);
        request_v(tile_of(begin), begin & 1);
        const u32x4_t words = tile_words(p.q + (size_t)(q0 + first) * p.q_stride + (size_t)head * p.r * D, 0x70000000u);
#pragma unroll
        for (int i = 0; i < 2 * T::kLoads; ++i) {
            const int in = i * T::kRowsPerLoad + lane / T::kUnits, r = 32 * wave + in, u = lane % T::kUnits ^ T::turn_k(in), q = query_of(r);
            tile_to_lds(own + (uint32_t)((i < T::kLoads ? 1 - (begin & 1) : 3 - (begin & 1)) * T::kBytes + i % T::kLoads * 1024),
                        r < rows_here && (EXACT || 8 * u < D) ? (q * p.q_stride + (ahead + r - q * p.r) * D + 8 * u) * 2 : 0x7f000000, words);
        }
    }
    half8_t qf[DP / 16];                                                 // Q^T: column qc, dimensions 16 s + 8 h .. + 7
    const int pos = back + first + query_of(row);                                          // the lane's query

    // A weight is 2^((score - origin) scale + shift), the origin being 0 but for scores of kFine and more; l: the sum of the weights as they are rounded.
    float16_t o[DB];
    float l, origin, shift, limit;  // limit: the score from which on these follow
    uint64_t moved = 0;             // the lanes whose origin is not 0
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[b][e] = 0.0f;
        limit = -INFINITY;
        l = origin = shift = 0.0f;
        moved = 0;
    };
    clear();

    // Where the lane's operands lie in the tile of keys that is read next, and in that of values: kept, and turned to the other buffer once a tile
    // (1170 -> 1150 us; an address each would be a vector instruction).  The unit's number, and the buffer's, are exclusive-ored in: rows of 16 bytes
    // times a power of two start at a multiple of that, in LDS too, as a kernel without static LDS has its own from address 0 on.
    uint32_t k_at[DP / 16], v_at[DB];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) k_at[i] = lds0 + (uint32_t)(qc * DP * 2 + ((2 * i + h) ^ T::turn_k(qc)) * 16);       // + 32 rows a block
    const int vrow = 4 * h + ((lane & 15) >> 2);                         // + 16 ks, + 8
#pragma unroll
    for (int b = 0; b < DB; ++b)
        v_at[b] = lds0 + (uint32_t)(2 * T::kBytes + vrow * DP * 2 + ((4 * b + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ T::turn_v(vrow)) * 16 + 8 * (lane & 1));
    auto other_keys = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            k_at[i] ^= (uint32_t)T::kBytes;
            asm volatile("" : "+v"(k_at[i]));                            // no address of the first buffer and a difference
        }
    };
    auto other_values = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < DB; ++b) {
            v_at[b] ^= (uint32_t)T::kBytes;
            asm volatile("" : "+v"(v_at[b]));
        }
    };
    // of products 16 ks ..
    auto v_operand = [&](int ks, int b) __attribute__((always_inline)) {
        const uint32_t at = v_at[b] + (uint32_t)(ks * 16 * DP * 2);
        const short4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(uintptr_t)at);
        const short4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(uintptr_t)(at + 8 * DP * 2));
        return __builtin_bit_cast(half8_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // the keys that the lane's query sees: from .. to
    const int see_from = p.window > 0 ? pos - p.window + 1 : 0, see_to = p.causal && pos < n_kv ? pos : n_kv - 1;
    auto sees = [&](int key) __attribute__((always_inline)) { return (key >= see_from) & (key <= see_to); };

    // Scores of 32 keys.
    auto scores = [&](float16_t& to, int block) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) to[e] = 0.0f;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i)
            to = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const lds_h8*)(uintptr_t)(k_at[i] + (uint32_t)(block * 32 * DP * 2)), qf[i], to, 0, 0, 0);
    };
    auto hide = [&](float16_t& of, int key0) __attribute__((always_inline)) {
        // a bit for each key that is seen, spread over the score by a field insert: no compare, whose result a scalar register would hold
        const int from = see_from - key0 - 4 * h, to = see_to - key0 - 4 * h;
        const uint32_t seen = (to < 0 ? 0u : to >= 31 ? ~0u : (2u << to) - 1u) & (from <= 0 ? ~0u : from > 31 ? 0u : ~0u << from);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)seen, 8 * (e / 4) + e % 4, 1);
            const float x = of[e];                                        // (bit-cast in place, a vector's element would be its first)
            of[e] = __builtin_bit_cast(float, (keep & __builtin_bit_cast(uint32_t, x)) | (~keep & 0xff800000u));
        }
    };
    // The largest score of the lane's query.
    auto largest = [&](const float16_t& of) __attribute__((always_inline)) {
        float most = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) most = fmaxf(most, of[e]);
        const uint32_t w = __builtin_bit_cast(uint32_t, most);
        const auto x = __builtin_amdgcn_permlane32_swap(w, w, false, false);
        return fmaxf(__builtin_bit_cast(float, (uint32_t)x[0]), __builtin_bit_cast(float, (uint32_t)x[1]));
    };
    // The shift follows the scores where it has to, by whole numbers, and with it the sums and the weights that are still to go into them, which a power of two
    // leaves all their places.  Where one query's does, those of others come along.
    auto follow = [&](float most, half8_t (&pending)[2], auto&... scores) __attribute__((always_inline)) {
        if ((__ballot(most > limit) | moved) == 0) return;
        const float size = most * p.scale, weight = __builtin_fmaf(most - origin, p.scale, shift);      // its logarithm as it is
        const bool fine = fabsf(size) < kFine, far = (most > limit) | (fine & (weight > kLift));
        const float to = fine ? kLift - ceilf(size) : kLift, less = (fine ? __builtin_fmaf(most, p.scale, to) : kLift) - weight;
        const float last = limit;
        limit = far ? (fine ? (kReach - to) * p.unit : most) : limit;
        shift = far ? to : shift;
        origin = far ? (fine ? 0.0f : most) : origin;
        const float keep = __builtin_amdgcn_exp2f(far ? (last == -INFINITY ? -INFINITY : less) : 0.0f);
        moved = __ballot(origin != 0.0f);
        l *= keep;
#pragma unroll
        for (int i = 0; i < 2; ++i) pending[i] *= (_Float16)keep;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[b][e] *= keep;
        if (moved == 0) return;
        auto from_origin = [&](float16_t& of) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 16; ++e) of[e] -= origin;
        };
        (from_origin(scores), ...);
    };
    // Weights, and their sum as they are rounded.
    auto weights = [&](half8_t (&pf)[2], const float16_t& of) __attribute__((always_inline)) {
        const half2_t ones = {(_Float16)1.0f, (_Float16)1.0f};
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const half2_t w = {(_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(of[e], p.scale, shift)), (_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(of[e + 1], p.scale, shift))};
            pf[e / 8][e % 8] = w[0];
            pf[e / 8][e % 8 + 1] = w[1];
            sum = __builtin_amdgcn_fdot2(w, ones, sum, false);
        }
        return sum;
    };

    // A tile is in LDS when all wavefronts have waited for their own requests and met; then the next ones' requests go to buffers that all
    // have finished reading.
    auto arrive = [&]() __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    float16_t s0, s1;
    half8_t p0[2], p1[2];
    // Before step i: the scores of its 64 keys and the weights of the first 32 of them are there, the maximum has followed the scores; its values
    // are there or on their way, and so are the next keys.  (prime() finds its keys.)
    auto prime = [&](int i) __attribute__((always_inline)) {
        if (i + 1 < all) request_k(tile_of(i + 1), (i + 1) & 1);
        scores(s0, 0);
        scores(s1, 1);
        if (i < masked) {
            hide(s0, tile_of(i) * BN);
            hide(s1, tile_of(i) * BN + 32);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) p0[e] = half8_t{0, 0, 0, 0, 0, 0, 0, 0};
        follow(fmaxf(largest(s0), largest(s1)), p0, s0, s1);
        l += weights(p0, s0);
    };
    // Three blocks of 32 keys: scores of the next (kind 0: there is none, what is computed is not looked at; 1: all are seen; 2: masked), weights
    // of the present one, the last one's product with its values.
    auto half_step = [&](float16_t& next, int kind, int next_key0, const float16_t& of, half8_t (&pf)[2], bool counts, const half8_t (&last)[2], int block) __attribute__((always_inline)) {
        scores(next, block);
        const float sum = weights(pf, of);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int b = 0; b < DB; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v_operand(2 * block + ks, b), last[ks], o[b], 0, 0, 0);
        l = counts ? l + sum : l;
        float most = largest(next);
        // 3 DP / 16 LDS reads for 2 DP / 16 products: the first four before all of them, two more with each of the next, so that none waits for
        // its own.  (1141 -> 1117 us for 8192 queries of 64 heads.)
        __builtin_amdgcn_sched_group_barrier(kLdsReads, 4, 0);
#pragma unroll
        for (int e = 0; e < (3 * DP / 16 - 4) / 2; ++e) {
            __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 2, 0);
        }
        if (kind != 1) {
            if (kind == 0) return;
            hide(next, next_key0);
            most = largest(next);
        }
        follow(most, pf, next);
    };
    // The tile of step i, but for its scores and first weights; those of the next.
    auto step = [&](int i) __attribute__((always_inline)) {
        arrive();                                                        // keys of i + 1, values of i
        const int after = tile_of(i + 1);
        if (i + 2 < all) request_k(tile_of(i + 2), i & 1);
        const int kind = i + 1 >= all ? 0 : i + 1 < masked ? 2 : 1;
        half_step(s0, kind, after * BN, s1, p1, true, p0, 0);
        if (i + 1 < all) request_v(after, (i + 1) & 1);
        half_step(s1, kind, after * BN + 32, s0, p0, kind != 0, p1, 1);
        other_keys();                                                    // of i + 2
        other_values();
    };
    // The masked tiles once more, key by key, after step `at`.
    auto by_key = [&](int at) __attribute__((always_inline)) {
        clear();
        if (at & 1) other_keys();                                        // both to the first buffer
        else other_values();
        for (int i = begin; i < masked && i < all; ++i)
            for (int block = 0; block < 2; ++block) {
                const int tile = tile_of(i), key0 = tile * BN + 32 * block;
                if (block == 0) {
                    arrive();
                    request_k(tile, 0);
                    request_v(tile, 0);
                    arrive();
                }
                scores(s0, block);
                hide(s0, key0);
                half8_t pf[2] = {};
                follow(largest(s0), pf, s0);
                l += weights(pf, s0);
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
                    for (int j = 0; j < 16; ++j) {                       // one key of the 16, in both operands
                        const bool seen = sees(key0 + 16 * ks + j);
                        half8_t one = pf[ks];
#pragma unroll
                        for (int e = 0; e < 8; ++e) one[e] = ((8 * (e / 4) + 4 * h + e % 4 == j) & seen) ? one[e] : (_Float16)0.0f;
#pragma unroll
                        for (int b = 0; b < DB; ++b) {
                            half8_t v = v_operand(2 * block + ks, b);
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
        arrive();
        if (!(at & 1)) {                                                 // to those of step at + 1
            other_keys();
            other_values();
        }
    };
    // Whether a wavefront's sums are not all finite (0 times a NaN or an infinity is a NaN); once for a workgroup.
    volatile uint32_t* spoilt_flag = reinterpret_cast<volatile uint32_t*>(smem + 4 * T::kBytes);
    auto spoilt = [&]() __attribute__((always_inline)) {
        float probe = 0.0f;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) probe = __builtin_fmaf(o[b][e], 0.0f, probe);
        if (__any(probe != 0.0f) && lane == 0) *spoilt_flag = 1;
        __syncthreads();
        return __builtin_amdgcn_readfirstlane((int)*spoilt_flag) != 0;
    };
    if (begin < all) {
        if (tid == 0) *spoilt_flag = 0;
        arrive();
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            qf[i] = *(const lds_h8*)(uintptr_t)(own + (uint32_t)((qc < 16 ? 1 - (begin & 1) : 3 - (begin & 1)) * T::kBytes + qc % 16 * DP * 2 + ((2 * i + h) ^ T::turn_k(qc)) * 16));
            if (p.negate) qf[i] = -qf[i];
        }
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) asm volatile("" : "+v"(qf[i]));           // read before its places are asked to take keys
        if (begin & 1) {
            other_keys();
            other_values();
        }
        prime(begin);
        other_keys();
        for (int i = begin; i < all; ++i) {
            step(i);
            if (i < masked && (i + 1 == masked || i + 1 == all) && spoilt()) {
                by_key(i);
                if (i + 1 < all) {
                    request_k(tile_of(i + 1), (i + 1) & 1);
                    request_v(tile_of(i + 1), (i + 1) & 1);
                    arrive();
                    prime(i + 1);
                    other_keys();
                }
            }
        }
    }

    {
        const uint32_t w = __builtin_bit_cast(uint32_t, l);
        const auto x = __builtin_amdgcn_permlane32_swap(w, w, false, false);
        l = __builtin_bit_cast(float, (uint32_t)x[0]) + __builtin_bit_cast(float, (uint32_t)x[1]);
    }
    if (parts > 1) {
        // Stores acknowledged before the ticket is taken; the last workgroup of the item adds the parts in order and leaves the counter at zero.
        constexpr int kPart = (BM * DP + NW * kWave * 2) * 4;
        const __amdgpu_buffer_rsrc_t sums = parts_of(p.part + ((size_t)unit * p.Hk + head) * p.splits * (kPart / 4));
        auto place = [&](int b, int e) __attribute__((always_inline)) { return ((wave * (DP / 8) + b * 4 + e / 4) * kWave + lane) * 16; };
        const int own_part = split * kPart, ml = BM * DP * 4 + (wave * kWave + lane) * 8;
        if (row < rows_here) {
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int e = 0; e < 16; e += 4) put16(sums, own_part + place(b, e), float4_t{o[b][e], o[b][e + 1], o[b][e + 2], o[b][e + 3]});
            put8(sums, own_part + ml, limit == -INFINITY ? kNone : origin * p.scale - shift, l);      // the logarithm of what l and the sums are multiples of
        }
        arrive();
        volatile uint32_t* flag = reinterpret_cast<volatile uint32_t*>(smem);
        if (tid == 0) {
            uint32_t* ctr = p.counters + ((size_t)unit * p.Hk + head) * (kCounterAreaWords / kPromptItems);
            const bool done = __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(parts - 1);
            if (done) __hip_atomic_store(ctr, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            *flag = done ? 1u : 0u;
        }
        __syncthreads();
        if (*flag == 0u) return;
        clear();
        float m = kNone;
        if (row < rows_here)
            for (int k = 0; k < parts; ++k) {
                float4_t w[DB * 4];
                const Pair other = get8(sums, k * kPart + ml);
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int e = 0; e < 16; e += 4) w[b * 4 + e / 4] = get16(sums, k * kPart + place(b, e));
                const float m_new = fmaxf(m, other.a), keep = __builtin_amdgcn_exp2f(m - m_new), add = __builtin_amdgcn_exp2f(other.a - m_new);
                m = m_new;
                l = l * keep + add * other.b;
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[b][e] = o[b][e] * keep + add * w[b * 4 + e / 4][e % 4];
            }
    }
    // Out through LDS, row after row: a wavefront stores whole rows, not 16 bytes of each of 32.  With Q's way in: 256 prompts of 128 tokens, 32 heads,
    // from 246 to 199 us; 8 of 1024, from 126 to 119.
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    arrive();
    unsigned char* mine = smem + wave * 32 * DP * 2;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<half4_t*>(mine + qc * DP * 2 + ((4 * b + e / 4) ^ T::turn_k(qc)) * 16 + 8 * h) =
                half4_t{(_Float16)(o[b][e] * inv), (_Float16)(o[b][e + 1] * inv), (_Float16)(o[b][e + 2] * inv), (_Float16)(o[b][e + 3] * inv)};
    _Float16* out = p.out + (size_t)(q0 + first) * p.out_stride + (size_t)head * p.r * D;
#pragma unroll
    for (int i = 0; i < 32 / T::kRowsPerLoad; ++i) {
        const int in = i * T::kRowsPerLoad + lane / T::kUnits, r = 32 * wave + in, u = lane % T::kUnits, q = query_of(r);
        if (r < rows_here && (EXACT || 8 * u < D))
            __builtin_nontemporal_store(*reinterpret_cast<const half8_t*>(mine + in * DP * 2 + (u ^ T::turn_k(in)) * 16),
                                        reinterpret_cast<half8_t*>(out + (size_t)q * p.out_stride + (ahead + r - q * p.r) * D + 8 * u));
    }
}

int set_max_lds(const void* fn, size_t bytes);

namespace {

struct PromptPlan {
    int dp, units, splits;
    size_t bytes;           // of workspace
};

constexpr int kPromptWaves = 4;

int prompt_plan(const codegemm_attn_desc* desc, PromptPlan* p)
{
    const int st = check_attn(desc);
    if (st) return st;
    const codegemm_attn_desc& d = *desc;
    constexpr int rows = 32 * kPromptWaves;
    p->dp = d.head_dim <= 64 ? 64 : d.head_dim <= 128 ? 128 : 256;
    // n rows are at most n / rows + 1 tiles
    const long long units = (long long)d.total_q * (d.q_heads / d.kv_heads) / rows + d.num_seqs, items = units * d.kv_heads;
    if (too_many(items, kPromptWaves * kWave)) return CODEGEMM_UNSUPPORTED;
    p->units = (int)units;
    // Few tiles of queries: their keys over several workgroups, as long as each has some tiles of them (as far as the host knows).
    p->splits = 1;
    if (items < kPromptItems) {
        const int held = d.max_kv < d.total_kv ? d.max_kv : d.total_kv > 0 ? d.total_kv : 1;
        const int keys = d.window > 0 && d.window < held - rows ? d.window + rows : held;
        const int worth = parts_worth(ceil_div(keys, 64)), room = prompt_groups(p->dp) / (int)items;
        p->splits = worth < room ? worth : room;
    }
    p->bytes = (size_t)kCounterAreaWords * sizeof(uint32_t) + kPairAreaBytes;
    if (p->splits > 1) p->bytes += (size_t)items * p->splits * (rows * p->dp + kPromptWaves * kWave * 2) * sizeof(float);
    return CODEGEMM_OK;
}

template <int DP, bool EXACT>
int launch_prompt_one(const PromptParams& p, int units, hipStream_t s)
{
    typedef PromptTile<DP, kPromptWaves> T;
    auto fn = attn_prompt_kernel<DP, kPromptWaves, EXACT>;
    const int st = set_max_lds(reinterpret_cast<const void*>(fn), T::kLds);
    if (st) return st;
    hipLaunchKernelGGL(fn, dim3((unsigned)(units * p.Hk * p.splits)), dim3(kPromptWaves * kWave), T::kLds, s, p);
    return hipGetLastError() == hipSuccess ? CODEGEMM_OK : CODEGEMM_LAUNCH_FAILED;
}

template <int DP>
int launch_prompt(const PromptParams& p, int units, hipStream_t s)
{
    return p.D == DP ? launch_prompt_one<DP, true>(p, units, s) : launch_prompt_one<DP, false>(p, units, s);
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" size_t codegemm_attn_prompt_workspace_bytes(const codegemm_attn_desc* desc)
{
    PromptPlan plan;
    return prompt_plan(desc, &plan) ? 0 : plan.bytes;
}

extern "C" int codegemm_attn_prompt(const codegemm_attn_desc* desc, const void* q, const void* k, const void* v, const int32_t* cu_q,
                                    const int32_t* cu_kv, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    PromptPlan plan;
    const int st = prompt_plan(desc, &plan);
    if (st) return st;
    const codegemm_attn_desc& d = *desc;
    if (!q || !out || !cu_q || !workspace || misaligned(q) || misaligned(out) || misaligned(workspace) || misaligned_ints(cu_q)) return CODEGEMM_INVALID_ARG;
    if (d.total_kv > 0 && (!k || !v || misaligned(k) || misaligned(v))) return CODEGEMM_INVALID_ARG;
    if (cu_kv ? misaligned_ints(cu_kv) : d.total_kv != d.total_q) return CODEGEMM_INVALID_ARG;
    if (workspace_bytes < plan.bytes) return CODEGEMM_WORKSPACE_TOO_SMALL;
    PromptParams p;
    p.q = static_cast<const _Float16*>(q);
    p.k = static_cast<const _Float16*>(k);
    p.v = static_cast<const _Float16*>(v);
    p.out = static_cast<_Float16*>(out);
    p.cu_q = cu_q;
    p.cu_kv = cu_kv;
    p.seqs = d.num_seqs; p.total_q = d.total_q; p.total_kv = d.total_kv;
    p.Hk = d.kv_heads; p.r = d.q_heads / d.kv_heads; p.D = d.head_dim;
    p.by_r = 1.0f / (float)p.r;
    p.q_stride = row_stride(d.q_stride, d.q_heads * d.head_dim);
    p.k_stride = row_stride(d.k_stride, d.kv_heads * d.head_dim);
    p.v_stride = row_stride(d.v_stride, d.kv_heads * d.head_dim);
    p.out_stride = row_stride(d.out_stride, d.q_heads * d.head_dim);
    p.window = d.window < kMaxTokens ? d.window : 0;               // one that reaches past every key is none
    p.causal = d.flags & CODEGEMM_ATTN_CAUSAL;
    p.negate = d.scale < 0.0f;
    const float size = d.scale < 0.0f ? -d.scale : d.scale;
    p.scale = log2_scale(size > 1e-30f ? size : 1e-30f);           // not 0: 0 times an infinite score is no number
    p.unit = 1.0f / p.scale;
    p.splits = plan.splits;
    p.counters = static_cast<uint32_t*>(workspace);
    p.part = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + (size_t)kCounterAreaWords * sizeof(uint32_t) + kPairAreaBytes);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (plan.dp == 64) return launch_prompt<64>(p, plan.units, s);
    if (plan.dp == 128) return launch_prompt<128>(p, plan.units, s);
    return launch_prompt<256>(p, plan.units, s);
}
