// Softmax weights summed per cached token: what a token gets from the last queries of its sequence, in all query heads of its key head.
//
// A weight needs its row's maximum and sum first, so the keys are gone through twice: kernels of STATS leave both for every row (a query in a query head) and
// part of the keys, a small one joins the parts, and the last adds up exp2(score - maximum) / sum per token.  Single tokens have the first from the
// attention itself.
//
// A wavefront has 16 TILES tokens of a sequence and key head in registers, as left operands of 16x16x32 products; the rows come by as right operands, 16 at
// a time, from LDS, where the workgroup's four wavefronts share them.  The score tiles have four tokens and one row a lane: what rows need is
// joined over four lanes, what tokens need over 16 at the very end, in a fixed order.
#include <type_traits>

#include "attn_common.h"

namespace cg {

constexpr int kScoreWaves = 4;
constexpr int kScoreThreads = kScoreWaves * kWave;
constexpr int kRowsAtOnce = 128;            // in LDS
constexpr int kScoreGroups = 2048;          // workgroups that are worth sharing the keys, at least
constexpr size_t kMostParts = 32u << 20;    // bytes of rows' parts

// Tokens of a wavefront at once: what leaves room for four (two) wavefronts on a SIMD.
constexpr int score_tiles(int dp) { return dp == 256 ? 2 : 4; }

struct ScoreParams {
    CacheView c;
    const _Float16* q;
    const int32_t *cu, *first;
    const float* earlier;
    float* scores;
    Pair* part;             // [slot][row]: maximum and sum over a slot's keys
    Pair* stats;            // [row]: what weights' logarithms lie below, 1 / sum
    int rows;               // total_q * query heads
    int total_q, r, q_stride, window;
    int slots;              // workgroups that share the keys
    float scale;            // times log2(e)
};

// Queries of a sequence: rows row0 .. row0 + n - 1 of q, the j-th at position at + j.
struct Queries {
    int row0, n, at, len;
};
__device__ __forceinline__ Queries queries_of(const ScoreParams& p, int seq)
{
    int lo = p.cu ? p.cu[seq] : seq, hi = p.cu ? p.cu[seq + 1] : seq + 1;
    lo = lo < 0 ? 0 : lo > p.total_q ? p.total_q : lo;
    hi = hi < lo ? lo : hi > p.total_q ? p.total_q : hi;
    const int held = p.c.max_pages << p.c.page_shift, given = p.c.lens[seq], len = given < 0 ? 0 : given;
    return Queries{lo, hi - lo, len - (hi - lo), len < held ? len : held};
}
__device__ __forceinline__ int first_seen(const ScoreParams& p, int position)
{
    return p.window > 0 && position >= p.window ? position - p.window + 1 : 0;
}

typedef __attribute__((address_space(4))) const int32_t const_int;

// A wavefront's tokens t0 .. t0 + 16 TILES - 1 as they lie in the cache: lane (col, g) has of every tile's token `col` the dimensions that operand_dim deals out.
template <int TYPE, int DP, bool EXACT>
struct Codes {
    static constexpr int TILES = score_tiles(DP), PARTS = DP / 32;
    static constexpr bool HALF = TYPE == CODEGEMM_KV_FP16, FOUR = TYPE == CODEGEMM_KV_INT4, SCALED = !HALF && !FOUR;
    static constexpr int WORDS = HALF ? 4 * PARTS : FOUR ? PARTS : 2 * PARTS;
    uint32_t w[TILES][WORDS], so[TILES][FOUR ? (DP + 127) / 128 : 1];
    float4_t by[TILES];     // 8 bits: the scales of tokens 4 g ..
    int ok;                 // bit n: tile n has a page

    __device__ __forceinline__ void load(const ScoreParams& p, int seq, int head, int t0, int len, int col, int g)
    {
        const CacheView& c = p.c;
        const int D = EXACT ? DP : c.D;
        const_int* table = (const_int*)(uintptr_t)c.table + (size_t)seq * c.max_pages;
        ok = 0;
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            const int t = t0 + 16 * n < len ? t0 + 16 * n : len - 1, found = table[t >> c.page_shift];
            const bool in = (unsigned)found < (unsigned)c.pages && t0 + 16 * n < len;
            ok |= in ? 1 << n : 0;
            const int page = in ? found : 0, slot = (t0 + 16 * n) & ((1 << c.page_shift) - 1);
            const size_t at = page_at(c, page, head) + (size_t)slot * D;                // (uniform)
            if constexpr (FOUR) {
                const unsigned char* row = c.k + at / 2 + col * (D / 2);
                const uint32_t* runs = reinterpret_cast<const uint32_t*>(c.k_scales) + runs_at(c, page, head, slot) + col * c.runs;
#pragma unroll
                for (int j = 0; j < (DP + 127) / 128; ++j) {
                    const int given = operand_dim<TYPE, DP>(4 * j, g), d = EXACT || given < D ? given : 0;
                    so[n][j] = runs[d >> c.run_shift];
                    if constexpr (DP < 128) {
                        const u32x2_t x = *reinterpret_cast<const u32x2_t*>(row + d / 2);
                        w[n][0] = x[0]; w[n][1] = x[1];
                    } else {
                        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(row + d / 2);
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[n][4 * j + i] = x[i];
                    }
                }
            } else {
                constexpr int SIZE = HALF ? 2 : 1;
                const unsigned char* row = c.k + at * SIZE + col * D * SIZE;
#pragma unroll
                for (int j = 0; j < DP / 64; ++j) {
                    const int given = 64 * j + 16 * g, d = EXACT || given < D ? given : 0;
#pragma unroll
                    for (int h = 0; h < SIZE; ++h) {
                        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(row + d * SIZE + 16 * h);
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[n][(j * SIZE + h) * 4 + i] = x[i];
                    }
                }
                if constexpr (SCALED) {
                    const float* s = c.k_scales + scales_at(c, page, head);
#pragma unroll
                    for (int r = 0; r < 4; ++r) by[n][r] = s[(slot + 4 * g + r) >> c.block_shift];
                }
            }
        }
    }
};

// .. as left operands of the products.
template <int TYPE, int DP, bool EXACT>
struct Keys {
    typedef Codes<TYPE, DP, EXACT> C;
    static constexpr int TILES = C::TILES, PARTS = C::PARTS;
    half8_t k[TILES][PARTS];
    float4_t by[TILES];     // of the scores: scale, times those of 8-bit codes
    int ok;

    __device__ __forceinline__ void take(const C& c, const ScoreParams& p, int g)
    {
        const int D = EXACT ? DP : p.c.D;
        const uint32_t mask = C::FOUR ? code_mask() : 0u;
        ok = c.ok;
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
#pragma unroll
            for (int i = 0; i < PARTS; ++i) {
                if constexpr (C::FOUR) k[n][i] = four_bits(c.w[n][i], both_low(c.so[n][i / 4]), both_high(c.so[n][i / 4]), mask);
                else if constexpr (C::HALF) k[n][i] = __builtin_bit_cast(half8_t, u32x4_t{c.w[n][4 * i], c.w[n][4 * i + 1], c.w[n][4 * i + 2], c.w[n][4 * i + 3]});
                else k[n][i] = codes_to_half<TYPE>(c.w[n][2 * i], c.w[n][2 * i + 1]);
                if (!EXACT && operand_dim<TYPE, DP>(i, g) >= D) k[n][i] = half8_t{0, 0, 0, 0, 0, 0, 0, 0};
            }
            if constexpr (C::SCALED) by[n] = c.by[n] * p.scale;
            else by[n] = float4_t{p.scale, p.scale, p.scale, p.scale};
        }
    }
};

// Rows from .. from + count - 1 of the queries in query heads `head` r .. + r - 1 into LDS, as right operands [tile][part][lane][8]; rows of queries that are none are zeros.
template <int TYPE, int DP>
__device__ __forceinline__ void load_rows(const ScoreParams& p, const Queries& qs, int head, int from, int count, int D, _Float16* to)
{
    constexpr int PARTS = DP / 32;
    const int pieces = (count + 15) / 16 * PARTS * kWave;
    for (int i = threadIdx.x; i < pieces; i += kScoreThreads) {
        const int lane = i % kWave, part = i / kWave % PARTS, row = from + i / (kWave * PARTS) * 16 + (lane & 15), d = operand_dim<TYPE, DP>(part, lane >> 4);
        half8_t x = {0, 0, 0, 0, 0, 0, 0, 0};
        if (row < from + count && d < D) x = *reinterpret_cast<const half8_t*>(p.q + (size_t)(qs.row0 + row / p.r) * p.q_stride + (size_t)(head * p.r + row % p.r) * D + d);
        *reinterpret_cast<half8_t*>(to + (size_t)i * 8) = x;
    }
}

// 16 rows against the wavefront's keys; a lane's scores are those of row `col` for tokens 4 g + r of every tile, before they are scaled.  (Scaled scores are rounded
// before a maximum is taken off, everywhere alike: fused, the largest score's own weight would be off by what large scores are rounded by.)
template <int TYPE, int DP, bool EXACT>
__device__ __forceinline__ void score_tile(const Keys<TYPE, DP, EXACT>& keys, const _Float16* rows, int lane, float4_t (&s)[score_tiles(DP)])
{
    constexpr int TILES = score_tiles(DP), PARTS = DP / 32;
#pragma unroll
    for (int n = 0; n < TILES; ++n) s[n] = float4_t{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        const half8_t q = *reinterpret_cast<const half8_t*>(rows + (size_t)(i * kWave + lane) * 8);
#pragma unroll
        for (int n = 0; n < TILES; ++n) s[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(keys.k[n][i], q, s[n], 0, 0, 0);
    }
}

// Which tokens of its row a lane sees: t - t0 in lo .. hi, in tiles that have a page.
struct Seen {
    int lo, hi, ok;
    __device__ __forceinline__ bool operator()(int n, int r, int g) const { const int t = 16 * n + 4 * g + r; return (ok >> n & 1) && t >= lo && t <= hi; }
};
template <class T>
__device__ __forceinline__ Seen seen_of(const ScoreParams& p, const Queries& qs, int at, int t0, const T& keys)
{
    return Seen{first_seen(p, at) - t0, (at < qs.len ? at : qs.len - 1) - t0, keys.ok};
}
// Whether rows row .. row + 15 all see all of a wavefront's tokens.
template <class T>
__device__ __forceinline__ bool see_all(const ScoreParams& p, const Queries& qs, const int* at, int t0, const T& keys)
{
    const int first = __builtin_amdgcn_readfirstlane(at[0]), last = __builtin_amdgcn_readfirstlane(at[15]);
    return keys.ok == (1 << T::TILES) - 1 && t0 + 16 * T::TILES - 1 <= first && t0 >= first_seen(p, last);
}

// What a workgroup keeps in LDS of up to kRowsAtOnce rows: the right operands, positions, and per wavefront (STATS) or once what is known of their weights.
template <int DP>
struct RowSpace {
    _Float16* rows;         // [tile][part][lane][8]
    Pair* sums;
    int* at;
    __device__ __forceinline__ explicit RowSpace(unsigned char* smem)
        : rows(reinterpret_cast<_Float16*>(smem)), sums(reinterpret_cast<Pair*>(smem + (size_t)kRowsAtOnce * DP * 2)), at(reinterpret_cast<int*>(sums + kScoreWaves * kRowsAtOnce))
    {
    }
    static constexpr size_t bytes = (size_t)kRowsAtOnce * DP * 2 + kScoreWaves * kRowsAtOnce * sizeof(Pair) + kRowsAtOnce * sizeof(int);
};
__device__ __forceinline__ void load_positions(const ScoreParams& p, const Queries& qs, int from, int count, int* at)
{
    for (int i = threadIdx.x; i < (count + 15) / 16 * 16; i += kScoreThreads) at[i] = qs.at + (from + i) / p.r;
}

// Workgroup (sequence and key head, slot, z): rows z * 128 .. and on, over every slots-th block of keys.
template <int TYPE, int DP, bool EXACT>
__global__ void __launch_bounds__(kScoreThreads, DP == 256 ? 2 : 3) score_stats_kernel(const ScoreParams p)
{
    constexpr int TILES = score_tiles(DP), PARTS = DP / 32, BLOCK = 16 * TILES * kScoreWaves;
    extern __shared__ __align__(16) unsigned char smem[];
    const RowSpace<DP> space(smem);
    const int D = EXACT ? DP : p.c.D, tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave), col = lane & 15, g = lane >> 4;
    const int seq = blockIdx.x / p.c.Hk, head = blockIdx.x % p.c.Hk;
    const Queries qs = queries_of(p, seq);
    const int count_all = qs.n * p.r, lowest = first_seen(p, qs.at) / BLOCK * BLOCK;   // of the first query's keys
    for (int from = blockIdx.z * kRowsAtOnce; from < count_all; from += gridDim.z * kRowsAtOnce) {
        const int count = count_all - from < kRowsAtOnce ? count_all - from : kRowsAtOnce;
        __syncthreads();
        load_rows<TYPE, DP>(p, qs, head, from, count, D, space.rows);
        load_positions(p, qs, from, count, space.at);
        for (int i = tid; i < kScoreWaves * kRowsAtOnce; i += kScoreThreads) space.sums[i] = Pair{-INFINITY, 0.0f};
        __syncthreads();
        for (int b = lowest + blockIdx.y * BLOCK; b < qs.len; b += p.slots * BLOCK) {
            const int t0 = b + wave * 16 * TILES;
            if (t0 >= qs.len) continue;
            Codes<TYPE, DP, EXACT> codes;
            Keys<TYPE, DP, EXACT> keys;
            codes.load(p, seq, head, t0, qs.len, col, g);
            keys.take(codes, p, g);
            for (int tile = 0; 16 * tile < count; ++tile) {
                float4_t s[TILES];
                score_tile<TYPE, DP, EXACT>(keys, space.rows + (size_t)tile * PARTS * kWave * 8, lane, s);
                Pair* mine = space.sums + wave * kRowsAtOnce + 16 * tile + col;
                const Pair old = *mine;
                auto add = [&](auto is_whole, const Seen& seen) {
                    constexpr bool whole = decltype(is_whole)::value;
                    float most = -INFINITY;
#pragma unroll
                    for (int n = 0; n < TILES; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            s[n][r] *= keys.by[n][r];
                            if (!whole) s[n][r] = seen(n, r, g) ? s[n][r] : -INFINITY;
                            most = fmaxf(most, s[n][r]);
                        }
                    most = over_groups(most, [](float a, float c) { return fmaxf(a, c); });
                    const float m = fmaxf(old.a, most), base = m == -INFINITY ? 0.0f : m;
                    float sum = 0.0f;
#pragma unroll
                    for (int n = 0; n < TILES; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f(s[n][r] - base);
                    sum = over_groups(sum, [](float a, float c) { return a + c; });
                    if (g == 0) *mine = Pair{m, __builtin_fmaf(old.b, __builtin_amdgcn_exp2f(old.a - base), sum)};
                };
                if (see_all(p, qs, space.at + 16 * tile, t0, keys)) add(std::true_type(), Seen{});
                else add(std::false_type(), seen_of(p, qs, space.at[16 * tile + col], t0, keys));
            }
        }
        __syncthreads();
        for (int i = tid; i < count; i += kScoreThreads) {
            const Pair* state = space.sums + i;
            float m = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kScoreWaves; ++w) m = fmaxf(m, state[w * kRowsAtOnce].a);
            const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int w = 0; w < kScoreWaves; ++w) sum += state[w * kRowsAtOnce].b * __builtin_amdgcn_exp2f(state[w * kRowsAtOnce].a - base);
            const int row = from + i;
            p.part[(size_t)blockIdx.y * p.rows + (size_t)(qs.row0 + row / p.r) * (p.c.Hk * p.r) + head * p.r + row % p.r] = Pair{m, sum};
        }
    }
}

// A row's parts, in order.
__global__ void __launch_bounds__(kScoreThreads) score_join_kernel(const ScoreParams p)
{
    const int row = blockIdx.x * kScoreThreads + threadIdx.x;
    if (row >= p.rows) return;
    float m = -INFINITY, sum = 0.0f;
    for (int i = 0; i < p.slots; ++i) {
        const Pair x = p.part[(size_t)i * p.rows + row];
        const float now = fmaxf(m, x.a), base = now == -INFINITY ? 0.0f : now;
        sum = sum * __builtin_amdgcn_exp2f(m - base) + x.b * __builtin_amdgcn_exp2f(x.a - base);
        m = now;
    }
    p.stats[row] = sum == 0.0f ? Pair{0.0f, 0.0f} : Pair{m, 1.0f / sum};
}

// Workgroup (sequence and key head, slot): every slots-th block of keys, all rows.  The next block's codes are on their way while one is worked on.
template <int TYPE, int DP, bool EXACT>
__global__ void __launch_bounds__(kScoreThreads, DP == 256 || (DP == 128 && TYPE != CODEGEMM_KV_INT4) ? 2 : 3) score_sum_kernel(const ScoreParams p)
{
    constexpr int TILES = score_tiles(DP), PARTS = DP / 32, BLOCK = 16 * TILES * kScoreWaves, VALUES = 4 * TILES;
    extern __shared__ __align__(16) unsigned char smem[];
    const RowSpace<DP> space(smem);
    const int D = EXACT ? DP : p.c.D, tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave), col = lane & 15, g = lane >> 4;
    const int seq = blockIdx.x / p.c.Hk, head = blockIdx.x % p.c.Hk;
    const Queries qs = queries_of(p, seq);
    const int count_all = qs.n * p.r, lowest = first_seen(p, qs.at), fresh = p.first ? p.first[seq] : qs.at;
    auto active = [&](int t0) { return t0 < qs.len && t0 + 16 * TILES > lowest; };
    int b = blockIdx.y * BLOCK;
    if (b >= qs.len) return;
    auto load = [&](int from) {
        const int count = count_all - from < kRowsAtOnce ? count_all - from : kRowsAtOnce;
        __syncthreads();
        load_rows<TYPE, DP>(p, qs, head, from, count, D, space.rows);
        load_positions(p, qs, from, count, space.at);
        for (int i = tid; i < (count + 15) / 16 * 16; i += kScoreThreads) {
            const int row = from + i;
            space.sums[i] = i < count ? p.stats[(size_t)(qs.row0 + row / p.r) * (p.c.Hk * p.r) + head * p.r + row % p.r] : Pair{0.0f, 0.0f};
        }
        __syncthreads();
        return count;
    };
    Codes<TYPE, DP, EXACT> codes;
    if (active(b + wave * 16 * TILES)) codes.load(p, seq, head, b + wave * 16 * TILES, qs.len, col, g);
    const bool once = count_all <= kRowsAtOnce;                                        // the rows stay
    if (once) load(0);
    for (; b < qs.len; b += p.slots * BLOCK) {
        const int t0 = b + wave * 16 * TILES, t_next = t0 + p.slots * BLOCK;
        const bool mine = active(t0);
        Keys<TYPE, DP, EXACT> keys;
        if (mine) keys.take(codes, p, g);
        if (t_next > t0 && active(t_next)) codes.load(p, seq, head, t_next, qs.len, col, g);
        float sum[VALUES];
#pragma unroll
        for (int i = 0; i < VALUES; ++i) sum[i] = 0.0f;
        if (b + BLOCK > lowest) {                                                      // uniform
            for (int from = 0; from < count_all; from += kRowsAtOnce) {
                const int count = once ? count_all : load(from);
                if (!mine) continue;
                for (int tile = 0; 16 * tile < count; ++tile) {
                    float4_t s[TILES];
                    score_tile<TYPE, DP, EXACT>(keys, space.rows + (size_t)tile * PARTS * kWave * 8, lane, s);
                    const Pair st = space.sums[16 * tile + col];
                    auto add = [&](auto is_whole, const Seen& seen) {
                        constexpr bool whole = decltype(is_whole)::value;
#pragma unroll
                        for (int n = 0; n < TILES; ++n)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const float w = __builtin_amdgcn_exp2f(s[n][r] * keys.by[n][r] - st.a), more = __builtin_fmaf(w, st.b, sum[4 * n + r]);
                                sum[4 * n + r] = whole || (seen(n, r, g) && st.b != 0.0f) ? more : sum[4 * n + r];
                            }
                    };
                    // (rows that are none have no weight in the first form either: a score of 0, and 1 / sum 0)
                    if (see_all(p, qs, space.at + 16 * tile, t0, keys)) add(std::true_type(), Seen{});
                    else add(std::false_type(), seen_of(p, qs, space.at[16 * tile + col], t0, keys));
                }
            }
        }
        // Over the 16 rows: lanes that differ in a bit of `col` share out the tokens by it, as long as there are several.
        int left = VALUES;
#pragma unroll
        for (int bit = 8; bit > 0; bit >>= 1) {
            if (VALUES > bit) {
                left = bit;
#pragma unroll
                for (int i = 0; i < VALUES; ++i) {
                    if (i >= left) break;
                    const float keep = col & bit ? sum[i + bit] : sum[i], give = col & bit ? sum[i] : sum[i + bit];
                    sum[i] = keep + __shfl_xor(give, bit);
                }
            } else {
#pragma unroll
                for (int i = 0; i < VALUES; ++i) sum[i] += __shfl_xor(sum[i], bit);
            }
        }
        // token: tile col / 4, row 4 g + col % 4
        const int t = t0 + 16 * (col >> 2) + 4 * g + (col & 3);
        if (t0 < qs.len && t < qs.len && col < VALUES) {
            const int page = page_of(p.c, seq, t >> p.c.page_shift);
            if (page >= 0) {
                const size_t at = (((size_t)page * p.c.Hk + head) << p.c.page_shift) + (t & ((1 << p.c.page_shift) - 1));
                p.scores[at] = (p.earlier && t < fresh ? p.earlier[at] : 0.0f) + sum[0];
            }
        }
    }
}

namespace {

struct ScorePlan {
    int slots, z, rows;
    size_t part, bytes;     // where parts begin (behind rows' stats), of workspace
};

constexpr size_t kFixedArea = (size_t)kCounterAreaWords * sizeof(uint32_t) + kPairAreaBytes;       // that other calls keep their counters in

int score_plan(const codegemm_kv_cache* cache, const codegemm_attn_desc* d, bool single, ScorePlan* p)
{
    int st = check_cache(cache, false);
    if (!st) st = check_attn(d);
    if (st) return st;
    if (d->kv_heads != cache->kv_heads || d->head_dim != cache->head_dim || d->num_seqs != cache->num_seqs) return CODEGEMM_INVALID_ARG;
    const long long rows = (long long)d->total_q * d->q_heads, items = (long long)d->num_seqs * d->kv_heads;
    if (rows >= 1ll << 31) return CODEGEMM_UNSUPPORTED;
    if (too_many(items, kScoreThreads)) return CODEGEMM_UNSUPPORTED;
    const int held = cache->max_pages * cache->page_size, longest = d->max_kv < held ? d->max_kv : held;
    const int block = 16 * score_tiles(d->head_dim > 128 ? 256 : 128) * kScoreWaves;
    const long long mean = (rows / d->kv_heads + d->num_seqs - 1) / d->num_seqs;           // rows of a sequence and key head
    p->z = (int)((mean + kRowsAtOnce - 1) / kRowsAtOnce);
    p->z = p->z < 1 ? 1 : p->z > 256 ? 256 : p->z;
    const long long blocks = ceil_div(longest, block), share = (kScoreGroups + items - 1) / items;
    long long slots = blocks < share ? blocks : share;
    if (!single && (size_t)slots * rows * sizeof(Pair) > kMostParts) slots = kMostParts / (rows * sizeof(Pair));
    p->slots = slots < 1 ? 1 : (int)slots;
    p->rows = (int)rows;
    p->part = kFixedArea + ((size_t)rows * sizeof(Pair) + 255) / 256 * 256;
    p->bytes = p->part + (single ? 0 : (size_t)p->slots * rows * sizeof(Pair));
    return CODEGEMM_OK;
}

int check_scores(const void* q, const int32_t* cu, const int32_t* first, const float* earlier, const float* scores, const void* workspace)
{
    if (!q || !scores || !workspace || misaligned(q) || misaligned(scores) || misaligned(workspace) || (earlier && misaligned(earlier))) return CODEGEMM_INVALID_ARG;
    return (cu && misaligned_ints(cu)) || (first && misaligned_ints(first)) ? CODEGEMM_INVALID_ARG : CODEGEMM_OK;
}

ScoreParams score_params(const codegemm_kv_cache* cache, const codegemm_attn_desc* d, const ScorePlan& plan, const void* q, const int32_t* cu, const int32_t* first,
                         const float* earlier, float* scores, void* workspace)
{
    ScoreParams p;
    p.c = cache_view(*cache);
    p.q = static_cast<const _Float16*>(q);
    p.cu = cu;
    p.first = first;
    p.earlier = earlier;
    p.scores = scores;
    p.stats = reinterpret_cast<Pair*>(static_cast<unsigned char*>(workspace) + kFixedArea);
    p.part = reinterpret_cast<Pair*>(static_cast<unsigned char*>(workspace) + plan.part);
    p.rows = plan.rows;
    p.total_q = d->total_q;
    p.r = d->q_heads / d->kv_heads;
    p.q_stride = row_stride(d->q_stride, d->q_heads * d->head_dim);
    p.window = d->window;
    p.slots = plan.slots;
    p.scale = log2_scale(d->scale);
    return p;
}

template <int TYPE, int DP, bool EXACT>
int launch_scores_one(const ScoreParams& p, const ScorePlan& plan, bool stats, hipStream_t s)
{
    const dim3 threads(kScoreThreads), items((unsigned)(p.c.seqs * p.c.Hk), (unsigned)plan.slots);
    constexpr size_t lds = RowSpace<DP>::bytes;
    if (stats) {
        auto fn = score_stats_kernel<TYPE, DP, EXACT>;
        const int st = set_max_lds(reinterpret_cast<const void*>(fn), lds);
        if (st) return st;
        hipLaunchKernelGGL(fn, dim3(items.x, items.y, (unsigned)plan.z), threads, lds, s, p);
        hipLaunchKernelGGL(score_join_kernel, dim3((unsigned)ceil_div(p.rows, kScoreThreads)), threads, 0, s, p);
    }
    auto fn = score_sum_kernel<TYPE, DP, EXACT>;
    const int st = set_max_lds(reinterpret_cast<const void*>(fn), lds);
    if (st) return st;
    hipLaunchKernelGGL(fn, items, threads, lds, s, p);
    return hipGetLastError() == hipSuccess ? CODEGEMM_OK : CODEGEMM_LAUNCH_FAILED;
}

template <int TYPE>
int launch_scores_of(const ScoreParams& p, const ScorePlan& plan, bool stats, hipStream_t s)
{
    if (p.c.D <= 64) return p.c.D == 64 ? launch_scores_one<TYPE, 64, true>(p, plan, stats, s) : launch_scores_one<TYPE, 64, false>(p, plan, stats, s);
    if (p.c.D <= 128) return p.c.D == 128 ? launch_scores_one<TYPE, 128, true>(p, plan, stats, s) : launch_scores_one<TYPE, 128, false>(p, plan, stats, s);
    return p.c.D == 256 ? launch_scores_one<TYPE, 256, true>(p, plan, stats, s) : launch_scores_one<TYPE, 256, false>(p, plan, stats, s);
}

int launch_scores(const ScoreParams& p, int dtype, const ScorePlan& plan, bool stats, hipStream_t s)
{
    if (dtype == CODEGEMM_KV_FP16) return launch_scores_of<CODEGEMM_KV_FP16>(p, plan, stats, s);
    if (dtype == CODEGEMM_KV_INT8) return launch_scores_of<CODEGEMM_KV_INT8>(p, plan, stats, s);
    if (dtype == CODEGEMM_KV_INT4) return launch_scores_of<CODEGEMM_KV_INT4>(p, plan, stats, s);
    return launch_scores_of<CODEGEMM_KV_FP8>(p, plan, stats, s);
}

// Of a call for single tokens: the attention's own workspace, and behind it that of the scores.
int decode_scores_plan(const codegemm_kv_cache* cache, const codegemm_attn_desc* d, ScorePlan* plan, size_t* first, size_t* bytes)
{
    const int st = score_plan(cache, d, true, plan);
    if (st) return st;
    const size_t need = codegemm_attn_decode_workspace_bytes(cache, d);
    if (!need) return d->total_q != d->num_seqs ? CODEGEMM_INVALID_ARG : CODEGEMM_UNSUPPORTED;
    *first = (need + 255) / 256 * 256;
    *bytes = *first + (plan->bytes - kFixedArea);
    return CODEGEMM_OK;
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" size_t codegemm_attn_scores_workspace_bytes(const codegemm_kv_cache* cache, const codegemm_attn_desc* desc)
{
    ScorePlan plan;
    return score_plan(cache, desc, false, &plan) ? 0 : plan.bytes;
}

extern "C" int codegemm_attn_scores(const codegemm_kv_cache* cache, const codegemm_attn_desc* desc, const void* q, const int32_t* cu_q, const int32_t* first,
                                    const float* earlier, float* scores, void* workspace, size_t workspace_bytes, void* stream)
{
    ScorePlan plan;
    int st = score_plan(cache, desc, false, &plan);
    if (!st) st = check_cache(cache, true);
    if (!st) st = check_scores(q, cu_q, first, earlier, scores, workspace);
    if (st) return st;
    if (!cu_q && desc->total_q != desc->num_seqs) return CODEGEMM_INVALID_ARG;
    if (workspace_bytes < plan.bytes) return CODEGEMM_WORKSPACE_TOO_SMALL;
    return launch_scores(score_params(cache, desc, plan, q, cu_q, first, earlier, scores, workspace), cache->dtype, plan, true, static_cast<hipStream_t>(stream));
}

extern "C" size_t codegemm_attn_decode_scores_workspace_bytes(const codegemm_kv_cache* cache, const codegemm_attn_desc* desc)
{
    ScorePlan plan;
    size_t first, bytes;
    return decode_scores_plan(cache, desc, &plan, &first, &bytes) ? 0 : bytes;
}

extern "C" int codegemm_attn_decode_scores(const codegemm_kv_cache* cache, const codegemm_attn_desc* desc, const void* q, void* out, const int32_t* first,
                                           const float* earlier, float* scores, void* workspace, size_t workspace_bytes, void* stream)
{
    ScorePlan plan;
    size_t behind, bytes;
    int st = decode_scores_plan(cache, desc, &plan, &behind, &bytes);
    if (!st) st = check_cache(cache, true);
    if (!st) st = check_scores(q, nullptr, first, earlier, scores, workspace);
    if (st) return st;
    if (workspace_bytes < bytes) return CODEGEMM_WORKSPACE_TOO_SMALL;
    ScoreParams p = score_params(cache, desc, plan, q, nullptr, first, earlier, scores, workspace);
    p.stats = reinterpret_cast<Pair*>(static_cast<unsigned char*>(workspace) + behind);
    st = attn_decode(cache, desc, q, out, p.stats, workspace, behind, stream);
    return st ? st : launch_scores(p, cache->dtype, plan, false, static_cast<hipStream_t>(stream));
}
