// Softmax weights summed per cached token: what a token gets from the last queries of its sequence, in all query heads of its key head.
//
// A weight needs its row's sum first, so the keys are gone through twice: kernels of STATS leave a maximum and a sum for every row (a query in a query head) and
// part of the keys, a small one joins the parts, and the last adds up exp2(score - maximum) / sum per token.  Single tokens have the first from the
// attention itself.
//
// A wavefront has 16 TILES tokens of a sequence and key head in registers, as left operands of 16x16x32 products; the rows come by as right operands, 16 at
// a time, from LDS, where the workgroup's four wavefronts share them.  The score tiles have four tokens and one row a lane: what rows need is
// joined over four lanes, what tokens need over 16 at the very end, in a fixed order.  Keys are read and their codes turned into operands once for all rows (up to
// 256), and nothing is written but 4 bytes a token.
//
// Rows by the hundred are bound by waits, on the two wavefronts a SIMD that 64 tokens' operands in registers allow: for every four products of 16x16x32 (a head of 128) a lane has
// four scores, an exponential and two or three instructions more each, beside what turns codes into operands, and of a pass's cycles matrix cores are busy for a sixth and vector
// instructions for two fifths; wavefronts wait for half of theirs.  The last 32 queries of four prompts of 8192, 64 and 8 heads of 128, 8 bits: 32 us for the rows' sums (maxima followed
// throughout: 42), 5 for the join, 34 for the weights; in all 63 us, 211 TFLOP/s; scores far from zero, whose maxima are followed, 99.  The next product's instructions set between
// those of the last one's weights, by hand, gained nothing.  Every block of keys is multiplied with every row, whether these see it or not, and with a window the weights' kernels load
// keys that no row sees: all queries of a prompt of 2048 take 900 us, the 32 queries above with a window of 500 48.  Few rows are bound by the keys' bytes and the wait for them: 32 sequences of 206 000
// tokens in all, 8 rows, 4 bits, 36 us beside the attention's 59, 4.0 TB/s with what tokens had before and have now.
#include <type_traits>

#include "attn_common.h"

namespace cg {

constexpr int kScoreWaves = 4;
constexpr int kScoreThreads = kScoreWaves * kWave;
constexpr int rows_at_once(int dp, bool stats) { return stats || dp == 256 ? 128 : 256; }       // in LDS, at most
constexpr int kStatsGroups = 512, kSumGroups = 512, kFewGroups = 2048;        // workgroups that are worth sharing the keys, at least
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
    int many;               // rows that LDS has room for
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
    size_t token[TILES];    // of a tile's first token, in [page][head][slot]; the same for all lanes
    int ok;                 // bit n: tile n has a page

    // (Wherever t0 lies: what is asked for is in the cache, and `ok` says what of it counts.)
    __device__ __forceinline__ void load(const ScoreParams& p, int seq, int head, int from, int len, int col, int g)
    {
        const CacheView& c = p.c;
        const int t0 = from < len ? from : (len - 1) / (16 * TILES) * (16 * TILES);
        const int D = EXACT ? DP : c.D;
        const_int* table = (const_int*)(uintptr_t)c.table + (size_t)seq * c.max_pages;
        if ((16 * TILES - 1) >> c.page_shift == 0) {                                    // (t0 is a multiple of 16 TILES: one page)
            const int found = table[t0 >> c.page_shift];
            const bool in = (unsigned)found < (unsigned)c.pages;
            const int tiles = (len - t0 + 15) / 16;
            ok = in ? tiles < TILES ? (1 << tiles) - 1 : (1 << TILES) - 1 : 0;          // (places behind the last token are in the page too)
            const int page = in ? found : 0, slot = t0 & ((1 << c.page_shift) - 1);
            const size_t at = (((size_t)page * c.Hk + head) << c.page_shift) + slot;
#pragma unroll
            for (int n = 0; n < TILES; ++n) {
                token[n] = at + 16 * n;
                take_tile(c, D, n, at, 16 * n, scales_at(c, page, head), slot, col, g);
            }
            return;
        }
        ok = 0;
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            const int t = t0 + 16 * n < len ? t0 + 16 * n : len - 1, found = table[t >> c.page_shift];
            const bool in = (unsigned)found < (unsigned)c.pages && t0 + 16 * n < len;
            ok |= in ? 1 << n : 0;
            const int page = in ? found : 0, slot = (t0 + 16 * n) & ((1 << c.page_shift) - 1);
            token[n] = (((size_t)page * c.Hk + head) << c.page_shift) + slot;
            take_tile(c, D, n, token[n], 0, scales_at(c, page, head), slot - 16 * n, col, g);
        }
    }

    // Tile n: its first token is the `ahead`-th behind token `at` of the pool, at slot slot0 + 16 n of its page, whose scales begin at scale0.  (at, scale0 and
    // slot0 are the same for all lanes, what is added to them fits into 32 bits.)
    __device__ __forceinline__ void take_tile(const CacheView& c, int D, int n, size_t at, int ahead, size_t scale0, int slot0, int col, int g)
    {
        if constexpr (FOUR) {
            const unsigned char* rows = c.k + at * (size_t)(D / 2);
            const unsigned char* runs = reinterpret_cast<const unsigned char*>(c.k_scales) + at * (size_t)(4 * c.runs);
#pragma unroll
            for (int j = 0; j < (DP + 127) / 128; ++j) {
                const int given = operand_dim<TYPE, DP>(4 * j, g), d = EXACT || given < D ? given : 0;
                so[n][j] = *reinterpret_cast<const uint32_t*>(runs + (uint32_t)(((ahead + col) * c.runs + (d >> c.run_shift)) * 4));
                const unsigned char* from = rows + (uint32_t)(((ahead + col) * D + d) / 2);
                if constexpr (DP < 128) {
                    const u32x2_t x = *reinterpret_cast<const u32x2_t*>(from);
                    w[n][0] = x[0]; w[n][1] = x[1];
                } else {
                    const u32x4_t x = *reinterpret_cast<const u32x4_t*>(from);
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[n][4 * j + i] = x[i];
                }
            }
        } else {
            constexpr int SIZE = HALF ? 2 : 1;
            const unsigned char* rows = c.k + at * (size_t)(D * SIZE);
#pragma unroll
            for (int j = 0; j < DP / 64; ++j) {
                const int given = 64 * j + 16 * g, d = EXACT || given < D ? given : 0;
#pragma unroll
                for (int h = 0; h < SIZE; ++h) {
                    const u32x4_t x = *reinterpret_cast<const u32x4_t*>(rows + (uint32_t)(((ahead + col) * D + d) * SIZE + 16 * h));
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[n][(j * SIZE + h) * 4 + i] = x[i];
                }
            }
            if constexpr (SCALED) {
                const float* s = c.k_scales + scale0;
                const int slot = slot0 + 16 * n + 4 * g;
                if (c.block_shift >= 2) {
                    const float x = s[slot >> c.block_shift];
                    by[n] = float4_t{x, x, x, x};
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) by[n][r] = s[(slot + r) >> c.block_shift];
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

// A row's sum of exp2(score) within these limits needs no maximum.
constexpr float kLeastSum = 1.0e-18f, kMostSum = 1.0e30f;

// Rows are worked on 32 at a time: two tiles, so that one's instructions fill the other's waits.
constexpr int kPair = 2, kPairRows = 16 * kPair;

// A row of a sequence and key head: query row / r of the sequence, query head `head` r + row % r.  Stepping on by 16 rows takes no division.
struct Row {
    int query, head;
    __device__ __forceinline__ Row(int row, int r) : query(row / r), head(row - row / r * r) {}
    __device__ __forceinline__ void next(int rows_q, int rows_h, int r)
    {
        query += rows_q;
        head += rows_h;
        const bool past = head >= r;
        query += past ? 1 : 0;
        head -= past ? r : 0;
    }
};

// Rows from .. from + count - 1 into LDS, as right operands [tile][part][lane][8]; behind them the last one again, up to a pair of tiles.
template <int DP>
__device__ __forceinline__ void load_rows(const ScoreParams& p, const Queries& qs, int head, int from, int count, int D, int type_is_four, _Float16* to)
{
    constexpr int PARTS = DP / 32, TILES = kScoreWaves / (PARTS < kScoreWaves ? PARTS : kScoreWaves);      // that the workgroup takes at once
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane & 15, g = lane >> 4;
    const int tile0 = wave / PARTS, step = 16 * TILES;
    Row row(from + 16 * tile0 + col, p.r);
    const Row last(from + count - 1, p.r);
    const int end = ceil_div(count, kPairRows) * kPairRows, rows_q = step / p.r, rows_h = step % p.r;
    constexpr int EACH = (PARTS + kScoreWaves - 1) / kScoreWaves, AT_ONCE = 8 / EACH;                       // all of them under way before the first is put down
    for (int i0 = 16 * tile0 + col; i0 < end; i0 += AT_ONCE * step) {
        half8_t x[AT_ONCE][EACH];
#pragma unroll
        for (int t = 0; t < AT_ONCE; ++t) {
            const bool in = i0 + t * step < count;
            const _Float16* q = p.q + (size_t)(qs.row0 + (in ? row.query : last.query)) * p.q_stride + (size_t)(head * p.r + (in ? row.head : last.head)) * D;
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                const int part = wave % PARTS + k * kScoreWaves, d = type_is_four ? operand_dim<CODEGEMM_KV_INT4, DP>(part, g) : operand_dim<CODEGEMM_KV_FP16, DP>(part, g);
                x[t][k] = *reinterpret_cast<const half8_t*>(q + (d < D ? d : 0));
                if (d >= D) x[t][k] = half8_t{0, 0, 0, 0, 0, 0, 0, 0};
            }
            row.next(rows_q, rows_h, p.r);
        }
#pragma unroll
        for (int t = 0; t < AT_ONCE; ++t)
#pragma unroll
            for (int k = 0; k < EACH; ++k)
                if (i0 + t * step < end) *reinterpret_cast<half8_t*>(to + ((size_t)((i0 + t * step) / 16 * PARTS + wave % PARTS + k * kScoreWaves) * kWave + lane) * 8) = x[t][k];
    }
}

// 32 rows against the wavefront's keys; a lane's scores are those of rows `col` and 16 + `col` for tokens 4 g + r of every tile of keys, before they are scaled.  (Scaled scores are
// rounded to 32 bits before a maximum is taken off, in every kernel that makes a row's sum, the attention among them, and in every one that makes its weights: were it fused in some, a
// row would give out 2^(half of the last place of its scores) times 1, 2 % from scores of 2^20 on.)
template <int TYPE, int DP, bool EXACT>
__device__ __forceinline__ void score_pair(const Keys<TYPE, DP, EXACT>& keys, const _Float16* rows, int lane, float4_t (&s)[kPair][score_tiles(DP)])
{
    constexpr int TILES = score_tiles(DP), PARTS = DP / 32;
#pragma unroll
    for (int k = 0; k < kPair; ++k)
#pragma unroll
        for (int n = 0; n < TILES; ++n) s[k][n] = float4_t{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < PARTS; ++i)
#pragma unroll
        for (int k = 0; k < kPair; ++k) {
            const half8_t q = *reinterpret_cast<const half8_t*>(rows + (size_t)((k * PARTS + i) * kWave + lane) * 8);
#pragma unroll
            for (int n = 0; n < TILES; ++n) s[k][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(keys.k[n][i], q, s[k][n], 0, 0, 0);
        }
}

// .. and 16 rows.
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

// Which of the tokens t0 + 16 n + 4 g + r a lane's row sees: those that lie `span` at most behind the first one, in tiles that have a page; rows that are not to have
// weight see none.  One compare each, nothing through the scalar unit: few blocks need it, but the workgroups that all others wait for have them (two compares and a bit
// joined there: 69.5 us for the 63 above; a loop of one body for all tiles 90, tiles that are seen as a whole told apart 72).
constexpr int kNowhere = 0x40000000;        // a span is less
template <int TILES>
struct Seen {
    int from[TILES];
    unsigned span;
    __device__ __forceinline__ bool operator()(int n, int r) const { return (unsigned)(from[n] + r) <= span; }
};
template <int TILES>
__device__ __forceinline__ Seen<TILES> seen_of(const ScoreParams& p, const Queries& qs, int at, int t0, int ok, int g, bool weighs = true)
{
    const int lo = first_seen(p, at) - t0, hi = (at < qs.len ? at : qs.len - 1) - t0;
    const bool any = hi >= lo && weighs;
    Seen<TILES> s;
    s.span = any ? (unsigned)(hi - lo) : 0u;
#pragma unroll
    for (int n = 0; n < TILES; ++n) s.from[n] = (ok >> n & 1) && any ? 16 * n + 4 * g - lo : kNowhere;
    return s;
}
// Whether 32 rows all see all of a wavefront's tokens.
template <class T>
__device__ __forceinline__ bool see_all(const ScoreParams& p, const Queries& qs, const int* at, int t0, const T& keys)
{
    const int first = __builtin_amdgcn_readfirstlane(at[0]), last = __builtin_amdgcn_readfirstlane(at[kPairRows - 1]);
    return keys.ok == (1 << T::TILES) - 1 && t0 + 16 * T::TILES - 1 <= first && t0 >= first_seen(p, last);
}

// What a workgroup keeps in LDS of up to `many` rows: the right operands, positions, and once, or (stats) for every wavefront, what is known of their weights.
template <int DP>
struct RowSpace {
    _Float16* rows;         // [tile][part][lane][8]
    Pair* sums;
    int* at;
    float* lanes;           // (stats) [wavefront][tile][lane]: what a lane has added up itself
    __device__ __forceinline__ RowSpace(unsigned char* smem, int many, int copies)
        : rows(reinterpret_cast<_Float16*>(smem)), sums(reinterpret_cast<Pair*>(smem + (size_t)many * DP * 2)), at(reinterpret_cast<int*>(sums + many * copies)), lanes(reinterpret_cast<float*>(at + many))
    {
    }
    static size_t bytes(int many, int copies) { return (size_t)many * (DP * 2 + copies * sizeof(Pair) + sizeof(int)); }
    static size_t lane_bytes(int many) { return (size_t)many * kScoreWaves * (kWave / 16) * sizeof(float); }
};
__device__ __forceinline__ void load_positions(const ScoreParams& p, const Queries& qs, int from, int count, int* at)
{
    for (int i = threadIdx.x; i < ceil_div(count, kPairRows) * kPairRows; i += kScoreThreads) at[i] = qs.at + (from + (i < count ? i : count - 1)) / p.r;
}

// Workgroup (sequence and key head, slot, z): rows z * 128 .. and on, over every slots-th block of keys.
template <int TYPE, int DP, bool EXACT>
__global__ void __launch_bounds__(kScoreThreads, 2) score_stats_kernel(const ScoreParams p)
{
    constexpr int TILES = score_tiles(DP), BLOCK = 16 * TILES * kScoreWaves;
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr bool AHEAD = TYPE == CODEGEMM_KV_INT4;                                   // wider codes would not fit into the registers beside the operands
    const int many = p.many;
    const RowSpace<DP> space(smem, many, kScoreWaves);
    const int D = EXACT ? DP : p.c.D, tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave), col = lane & 15, g = lane >> 4;
    const int seq = blockIdx.x / p.c.Hk, head = blockIdx.x % p.c.Hk;
    const Queries qs = queries_of(p, seq);
    const int count_all = qs.n * p.r, seen0 = first_seen(p, qs.at), lowest = (seen0 < qs.len ? seen0 : qs.len) / BLOCK * BLOCK;       // of the first query's keys
    for (int from = blockIdx.z * many; from < count_all; from += gridDim.z * many) {
        const int count = count_all - from < many ? count_all - from : many;
        const int begin = lowest + blockIdx.y * BLOCK;
        Codes<TYPE, DP, EXACT> codes;
        if (begin < qs.len) codes.load(p, seq, head, begin + wave * 16 * TILES, qs.len, col, g);
        __syncthreads();
        load_rows<DP>(p, qs, head, from, count, D, TYPE == CODEGEMM_KV_INT4, space.rows);
        load_positions(p, qs, from, count, space.at);
        for (int i = tid; i < kScoreWaves * many; i += kScoreThreads) space.sums[i] = Pair{0.0f, 0.0f};
        for (int i = tid; i < kScoreWaves * many * (kWave / 16); i += kScoreThreads) space.lanes[i] = 0.0f;
        __syncthreads();
        // work(keys, t0, row) for the wavefront's blocks and pairs of tiles
        auto all_blocks = [&](auto work) {
            for (int b = begin; b < qs.len; b += p.slots * BLOCK) {
                const int t0 = b + wave * 16 * TILES;
                Keys<TYPE, DP, EXACT> keys;
                if (!AHEAD && b != begin) codes.load(p, seq, head, t0, qs.len, col, g);
                keys.take(codes, p, g);
                if (AHEAD) {
                    __builtin_amdgcn_sched_barrier(0);                                 // (the next codes come into the same registers)
                    if (qs.len - b > p.slots * BLOCK) codes.load(p, seq, head, t0 + p.slots * BLOCK, qs.len, col, g);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (t0 >= qs.len) continue;
                for (int row = 0; row < count; row += kPairRows) work(keys, t0, row);
            }
        };
        // At first weights are exp2(score) as they are, which needs no maximum, and a lane adds up its own.  Sums that come out between kLeastSum and kMostSum are as
        // good as any: what is lost below 2^-126 is nothing beside them.
        all_blocks([&](const Keys<TYPE, DP, EXACT>& keys, int t0, int row) {
            float4_t s[kPair][TILES];
            score_pair<TYPE, DP, EXACT>(keys, space.rows + (size_t)row * DP, lane, s);
            float* lanes = space.lanes + (wave * many + row) * (kWave / 16) + lane;
            float sum[kPair] = {lanes[0], lanes[kWave]};
            if (see_all(p, qs, space.at + row, t0, keys)) {
#pragma unroll
                for (int n = 0; n < TILES; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int k = 0; k < kPair; ++k) sum[k] += __builtin_amdgcn_exp2f(s[k][n][r] * keys.by[n][r]);
            } else {
#pragma unroll
                for (int k = 0; k < kPair; ++k) {
                    const Seen<TILES> seen = seen_of<TILES>(p, qs, space.at[row + 16 * k + col], t0, keys.ok, g);
#pragma unroll
                    for (int n = 0; n < TILES; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) sum[k] += seen(n, r) ? __builtin_amdgcn_exp2f(s[k][n][r] * keys.by[n][r]) : 0.0f;
                }
            }
            lanes[0] = sum[0];
            lanes[kWave] = sum[1];
        });
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");                              // (its own sums, by other lanes)
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        bool fine = true;
        if (begin + wave * 16 * TILES < qs.len)
            for (int row = lane; row < count; row += kWave) {
                const float* lanes = space.lanes + (wave * many + row / 16 * 16) * (kWave / 16) + row % 16;
                const float sum = (lanes[0] + lanes[16]) + (lanes[32] + lanes[48]);
                fine = fine && ((sum > kLeastSum && sum < kMostSum) || (sum == 0.0f && space.at[row] < begin + wave * 16 * TILES));     // (it stands before all of them)
            }
        // Where they do not, once more with every maximum followed.  (Also where a row sees none of the wavefront's keys for another reason: its window begins behind them, or they
        // have no page.  The sum is zero again then.)
        if (!__all(fine)) {
            if (!AHEAD || begin + p.slots * BLOCK < qs.len) codes.load(p, seq, head, begin + wave * 16 * TILES, qs.len, col, g);
            for (int row = lane; row < count; row += kWave) space.sums[wave * many + row] = Pair{-INFINITY, 0.0f};
            for (int i = lane; i < many * (kWave / 16); i += kWave) space.lanes[wave * many * (kWave / 16) + i] = 0.0f;
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            all_blocks([&](const Keys<TYPE, DP, EXACT>& keys, int t0, int row) {
#pragma unroll 1
                for (int k = 0; k < kPair; ++k) {
                    if (row + 16 * k >= count) break;
                    float4_t s[TILES];
                    score_tile<TYPE, DP, EXACT>(keys, space.rows + (size_t)(row + 16 * k) * DP, lane, s);
                    Pair* mine = space.sums + wave * many + row + 16 * k + col;
                    const bool is_row = row + 16 * k + col < count;
                    const Pair old = is_row ? *mine : Pair{-INFINITY, 0.0f};
                    const Seen<TILES> seen = seen_of<TILES>(p, qs, space.at[row + 16 * k + col], t0, keys.ok, g);
                    float most = -INFINITY;
#pragma unroll
                    for (int n = 0; n < TILES; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) most = fmaxf(most, seen(n, r) ? s[n][r] * keys.by[n][r] : -INFINITY);
                    most = over_groups(most, [](float a, float c) { return fmaxf(a, c); });
                    const float m = fmaxf(old.a, most), base = m == -INFINITY ? 0.0f : m;
                    float sum = 0.0f;
#pragma unroll
                    for (int n = 0; n < TILES; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float w = __builtin_amdgcn_exp2f(s[n][r] * keys.by[n][r] - base);
                            sum += seen(n, r) ? w : 0.0f;
                        }
                    sum = over_groups(sum, [](float a, float c) { return a + c; });
                    if (g == 0 && is_row) *mine = Pair{m, __builtin_fmaf(old.b, __builtin_amdgcn_exp2f(old.a - base), sum)};
                }
            });
        }
        __syncthreads();
        for (int i = tid; i < count; i += kScoreThreads) {
            // of a wavefront; one that has nothing says nothing about the maximum
            Pair state[kScoreWaves];
            float m = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kScoreWaves; ++w) {
                const float* lanes = space.lanes + (w * many + i / 16 * 16) * (kWave / 16) + i % 16;
                const Pair x = space.sums[w * many + i];
                state[w].b = x.b + ((lanes[0] + lanes[16]) + (lanes[32] + lanes[48]));
                state[w].a = state[w].b == 0.0f ? -INFINITY : x.a;
                m = fmaxf(m, state[w].a);
            }
            const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int w = 0; w < kScoreWaves; ++w) sum += state[w].b * __builtin_amdgcn_exp2f(state[w].a - base);
            const int row = from + i;
            p.part[(size_t)blockIdx.y * p.rows + (size_t)(qs.row0 + row / p.r) * (p.c.Hk * p.r) + head * p.r + row % p.r] = Pair{m, sum};
        }
    }
}

// x of the lane whose `col` has another bit 8, 4, 2 or 1.
template <int BIT>
__device__ __forceinline__ float other_column(float x)
{
    const int w = __builtin_bit_cast(int, x);
    if constexpr (BIT == 8) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, w, 0x128, 0xf, 0xf, false));        // row_ror 8
    else if constexpr (BIT == 4) return __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(w, 0x101f));                        // xor 4
    else if constexpr (BIT == 2) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, w, 0x4e, 0xf, 0xf, false));    // quad_perm 2 3 0 1
    else return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, w, 0xb1, 0xf, 0xf, false));                             // quad_perm 1 0 3 2
}
// Sums of N (8 or 16) values over the 16 columns: value i in the lanes of column i (and i + 8).
template <int N, int BIT = 8>
__device__ __forceinline__ void over_columns(float (&x)[N], int col)
{
    if constexpr (BIT >= N) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += other_column<BIT>(x[i]);
    } else {
        const bool up = col & BIT;
#pragma unroll
        for (int i = 0; i < BIT; ++i) {
            const float keep = up ? x[i + BIT] : x[i], give = up ? x[i] : x[i + BIT];
            x[i] = keep + other_column<BIT>(give);
        }
    }
    if constexpr (BIT > 1) over_columns<N, BIT / 2>(x, col);
}

// A row's parts, in order.
__global__ void __launch_bounds__(kScoreThreads) score_join_kernel(const ScoreParams p)
{
    const int row = blockIdx.x * kScoreThreads + threadIdx.x;
    if (row >= p.rows) return;
    float m = -INFINITY, sum = 0.0f;
    constexpr int AT_ONCE = 8;
    for (int i0 = 0; i0 < p.slots; i0 += AT_ONCE) {
        Pair x[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) x[i] = p.part[(size_t)(i0 + i < p.slots ? i0 + i : i0) * p.rows + row];
        float now = m;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) now = fmaxf(now, x[i].a);
        const float base = now == -INFINITY ? 0.0f : now;
        sum *= __builtin_amdgcn_exp2f(m - base);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) sum += i0 + i < p.slots ? x[i].b * __builtin_amdgcn_exp2f(x[i].a - base) : 0.0f;
        m = now;
    }
    p.stats[row] = sum == 0.0f ? Pair{0.0f, 0.0f} : Pair{m, 1.0f / sum};
}

// Workgroup (sequence and key head, slot): every slots-th block of keys, all rows.  The next block's codes are on their way while one is worked on.
template <int TYPE, int DP, bool EXACT>
__global__ void __launch_bounds__(kScoreThreads, 2) score_sum_kernel(const ScoreParams p)
{
    constexpr int TILES = score_tiles(DP), BLOCK = 16 * TILES * kScoreWaves, VALUES = 4 * TILES;
    extern __shared__ __align__(16) unsigned char smem[];
    const int many = p.many;
    const RowSpace<DP> space(smem, many, 1);
    const int D = EXACT ? DP : p.c.D, tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave), col = lane & 15, g = lane >> 4;
    const int seq = blockIdx.x / p.c.Hk, head = blockIdx.x % p.c.Hk;
    const Queries qs = queries_of(p, seq);
    const int count_all = qs.n * p.r, lowest = first_seen(p, qs.at), fresh = p.first ? p.first[seq] : qs.at;
    auto active = [&](int t0) { return t0 < qs.len && t0 + 16 * TILES > lowest; };
    int b = blockIdx.y * BLOCK;
    if (b >= qs.len) return;
    auto load = [&](int from) {
        const int count = count_all - from < many ? count_all - from : many;
        __syncthreads();
        load_rows<DP>(p, qs, head, from, count, D, TYPE == CODEGEMM_KV_INT4, space.rows);
        load_positions(p, qs, from, count, space.at);
        for (int i = tid; i < ceil_div(count, kPairRows) * kPairRows; i += kScoreThreads) {
            const int row = from + (i < count ? i : count - 1);
            Pair st = p.stats[(size_t)(qs.row0 + row / p.r) * (p.c.Hk * p.r) + head * p.r + row % p.r];
            if (i >= count) st.b = 0.0f;
            space.sums[i] = st;
        }
        __syncthreads();
        return count;
    };
    // what a lane's token had before (where nothing says so: what lies in its place, which is not looked at) comes with its block's codes
    const float* earlier = p.earlier ? p.earlier : p.scores;
    const int tile_of = (col >> 2) & (TILES - 1), in_tile = 4 * g + (col & 3);
    Codes<TYPE, DP, EXACT> codes;
    size_t place_next;
    float had_next;
    auto ask = [&](int from) {
        codes.load(p, seq, head, from, qs.len, col, g);
        place_next = codes.token[0];
#pragma unroll
        for (int n = 1; n < TILES; ++n) place_next = tile_of == n ? codes.token[n] : place_next;
        place_next += in_tile;
        had_next = earlier[place_next];
    };
    ask(b + wave * 16 * TILES);
    const bool once = count_all <= many;                                               // the rows stay
    if (once) load(0);
    // A block's result is stored after the next block's codes have come: the wait for these is one for all that is under way.
    size_t place_last = 0;
    float last = 0.0f;
    bool to_store = false;
    for (; b < qs.len; b += p.slots * BLOCK) {
        const int t0 = b + wave * 16 * TILES, t = t0 + 16 * tile_of + in_tile;
        const bool mine = active(t0);
        Keys<TYPE, DP, EXACT> keys;
        keys.take(codes, p, g);
        const size_t place = place_next;
        const float had = had_next;
        __builtin_amdgcn_sched_barrier(0);                                             // (the next codes come into the same registers)
        if (to_store) p.scores[place_last] = last;
        if (qs.len - b > p.slots * BLOCK) ask(t0 + p.slots * BLOCK);
        __builtin_amdgcn_sched_barrier(0);
        float sum[VALUES];
#pragma unroll
        for (int i = 0; i < VALUES; ++i) sum[i] = 0.0f;
        if (b + BLOCK > lowest) {                                                      // uniform
            for (int from = 0; from < count_all; from += many) {
                const int count = once ? count_all : load(from);
                if (!mine) continue;
                for (int row = 0; row < count; row += kPairRows) {
                    float4_t s[kPair][TILES];
                    score_pair<TYPE, DP, EXACT>(keys, space.rows + (size_t)row * DP, lane, s);
                    const Pair st[kPair] = {space.sums[row + col], space.sums[row + 16 + col]};
                    auto add = [&](auto is_plain) {
                        constexpr bool plain = decltype(is_plain)::value;
#pragma unroll
                        for (int k = 0; k < kPair; ++k) {
                            const Seen<TILES> seen = plain ? Seen<TILES>{} : seen_of<TILES>(p, qs, space.at[row + 16 * k + col], t0, keys.ok, g, st[k].b != 0.0f);
#pragma unroll
                            for (int n = 0; n < TILES; ++n)
#pragma unroll
                                for (int r = 0; r < 4; ++r) {
                                    const float score = s[k][n][r] * keys.by[n][r];
                                    const float w = __builtin_amdgcn_exp2f(plain ? score : score - st[k].a);
                                    const float more = __builtin_fmaf(w, st[k].b, sum[4 * n + r]);
                                    sum[4 * n + r] = plain || seen(n, r) ? more : sum[4 * n + r];
                                }
                        }
                    };
                    // Nearly always: rows whose sums needed no maximum, which is 0 then, and keys that all of them see.  (Rows that are none have no weight here either: scores of
                    // one that is, and 1 / sum 0.)
                    if (__all(st[0].a == 0.0f && st[1].a == 0.0f) && see_all(p, qs, space.at + row, t0, keys)) add(std::true_type());
                    else add(std::false_type());
                }
            }
        }
        // Over the 16 rows: lanes that differ in a bit of `col` share out the tokens by it, as long as there are several.
        over_columns<VALUES>(sum, col);
        to_store = t < qs.len && col < VALUES && (keys.ok >> tile_of & 1);
        place_last = place;
        last = (p.earlier && t < fresh ? had : 0.0f) + sum[0];
    }
    if (to_store) p.scores[place_last] = last;
}

// Up to 16 rows, as single tokens have where a key head serves no more query heads: they stay in registers, and a wavefront goes through its blocks of keys by
// itself, the next one's codes under way.  Wavefront (sequence and key head, 4 slots and its own).
template <int TYPE, int DP, bool EXACT>
__global__ void __launch_bounds__(kScoreThreads, DP >= 128 && TYPE == CODEGEMM_KV_FP16 ? 2 : 3) score_few_kernel(const ScoreParams p)
{
    constexpr int TILES = score_tiles(DP), PARTS = DP / 32, BLOCK = 16 * TILES, VALUES = 4 * TILES;
    const int D = EXACT ? DP : p.c.D, tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave), col = lane & 15, g = lane >> 4;
    const int seq = blockIdx.x / p.c.Hk, head = blockIdx.x % p.c.Hk;
    const Queries qs = queries_of(p, seq);
    const int stride = p.slots * kScoreWaves * BLOCK;
    int t0 = ((int)blockIdx.y * kScoreWaves + wave) * BLOCK;
    if (t0 >= qs.len) return;
    const int rows = qs.n * p.r, lowest = first_seen(p, qs.at), fresh = p.first ? p.first[seq] : qs.at;
    const float* earlier = p.earlier ? p.earlier : p.scores;        // (where nothing says so: what lies in its place, which is not looked at)
    const int tile_of = (col >> 2) & (TILES - 1), in_tile = 4 * g + (col & 3);
    Codes<TYPE, DP, EXACT> codes;
    size_t place_next;
    float had_next;
    auto ask = [&](int from) {
        codes.load(p, seq, head, from, qs.len, col, g);
        place_next = codes.token[0];
#pragma unroll
        for (int n = 1; n < TILES; ++n) place_next = tile_of == n ? codes.token[n] : place_next;
        place_next += in_tile;
        had_next = earlier[place_next];
    };
    ask(t0);
    // The lane's row: its operands, where it stands, what its weights' logarithms lie below and 1 / their sum.
    // (Behind the last row this again, without weight: a row of zeros would meet infinite keys.)
    const int row = col < rows ? col : rows > 0 ? rows - 1 : 0, query = row / p.r, at = qs.at + query;
    half8_t q[PARTS];
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        half8_t x = {0, 0, 0, 0, 0, 0, 0, 0};
        const int d = operand_dim<TYPE, DP>(i, g);
        if (rows > 0 && d < D) x = *reinterpret_cast<const half8_t*>(p.q + (size_t)(qs.row0 + query) * p.q_stride + (size_t)(head * p.r + row - query * p.r) * D + d);
        q[i] = x;
    }
    Pair st = {0.0f, 0.0f};
    if (rows > 0) st = p.stats[(size_t)(qs.row0 + query) * (p.c.Hk * p.r) + head * p.r + row - query * p.r];
    if (col >= rows) st.b = 0.0f;
    const int seen_from = first_seen(p, qs.at + (qs.n > 0 ? qs.n - 1 : 0));                 // by all rows, up to the first one's position
    size_t place_last = 0;
    float last = 0.0f;
    bool to_store = false;
    for (; t0 < qs.len; t0 += stride) {
        const Codes<TYPE, DP, EXACT> now = codes;
        const size_t place = place_next;
        const float had = had_next;
        const int t = t0 + 16 * tile_of + in_tile, ok = now.ok;
        // (after the wait for the codes, so that it is not one for this store too)
        if (to_store) p.scores[place_last] = last;
        if (qs.len - t0 > stride) ask(t0 + stride);
        float sum[VALUES];
#pragma unroll
        for (int i = 0; i < VALUES; ++i) sum[i] = 0.0f;
        if (t0 + BLOCK > lowest && rows > 0) {
            Keys<TYPE, DP, EXACT> keys;
            keys.take(now, p, g);
            float4_t s[TILES];
#pragma unroll
            for (int n = 0; n < TILES; ++n) s[n] = float4_t{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < PARTS; ++i)
#pragma unroll
                for (int n = 0; n < TILES; ++n) s[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(keys.k[n][i], q[i], s[n], 0, 0, 0);
            const bool whole = ok == (1 << TILES) - 1 && t0 + BLOCK - 1 <= qs.at && t0 >= seen_from;
#pragma unroll
            for (int n = 0; n < TILES; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[4 * n + r] = __builtin_amdgcn_exp2f(s[n][r] * keys.by[n][r] - st.a) * st.b;
            if (!whole) {
                const Seen<TILES> seen = seen_of<TILES>(p, qs, at, t0, ok, g, st.b != 0.0f);
#pragma unroll
                for (int n = 0; n < TILES; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[4 * n + r] = seen(n, r) ? sum[4 * n + r] : 0.0f;
            }
        }
        over_columns<VALUES>(sum, col);
        to_store = t < qs.len && col < VALUES && (ok >> tile_of & 1);
        place_last = place;
        last = (p.earlier && t < fresh ? had : 0.0f) + sum[0];
    }
    if (to_store) p.scores[place_last] = last;
}

namespace {

struct ScorePlan {
    int slots, sum_slots, few_slots, z, rows;
    int most;               // rows of a sequence and key head, at most
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
    if (rows > 1ll << 30) return CODEGEMM_UNSUPPORTED;                                     // (a workgroup steps on from row to row in 32 bits)
    if (too_many(items, kScoreThreads)) return CODEGEMM_UNSUPPORTED;
    const int held = cache->max_pages * cache->page_size, longest = d->max_kv < held ? d->max_kv : held;
    const int block = 16 * score_tiles(d->head_dim > 128 ? 256 : 128) * kScoreWaves;
    const int dp = d->head_dim > 128 ? 256 : d->head_dim > 64 ? 128 : 64, at_once = rows_at_once(dp, true);
    const long long mean = (rows / d->kv_heads + d->num_seqs - 1) / d->num_seqs;           // rows of a sequence and key head
    p->z = (int)((mean + at_once - 1) / at_once);
    p->z = p->z < 1 ? 1 : p->z > 256 ? 256 : p->z;
    const long long blocks = ceil_div(longest, block), most = single ? d->q_heads / d->kv_heads : rows / d->kv_heads;
    auto share = [&](long long groups, long long of) { const long long n = (groups + of - 1) / of; return blocks < n ? blocks : n; };
    long long slots = share(kStatsGroups, items * p->z);
    if (!single && (size_t)slots * rows * sizeof(Pair) > kMostParts) slots = kMostParts / (rows * sizeof(Pair));
    p->slots = slots < 1 ? 1 : (int)slots;
    p->sum_slots = (int)share(kSumGroups, items);
    p->few_slots = (int)share(kFewGroups, items);
    p->most = most < 1024 ? (int)most : 1024;
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
    p.scale = log2_scale(d->scale);
    return p;
}

template <int TYPE, int DP, bool EXACT>
int launch_scores_one(ScoreParams p, const ScorePlan& plan, bool stats, hipStream_t s)
{
    const dim3 threads(kScoreThreads);
    const unsigned items = (unsigned)(p.c.seqs * p.c.Hk);
    const int rows = ceil_div(plan.most, kPairRows) * kPairRows;
    if (stats) {
        p.slots = plan.slots;
        p.many = rows < rows_at_once(DP, true) ? rows : rows_at_once(DP, true);
        auto fn = score_stats_kernel<TYPE, DP, EXACT>;
        const size_t lds = RowSpace<DP>::bytes(p.many, kScoreWaves) + RowSpace<DP>::lane_bytes(p.many);
        const int st = set_max_lds(reinterpret_cast<const void*>(fn), lds);
        if (st) return st;
        hipLaunchKernelGGL(fn, dim3(items, (unsigned)plan.slots, (unsigned)plan.z), threads, lds, s, p);
        hipLaunchKernelGGL(score_join_kernel, dim3((unsigned)ceil_div(p.rows, kScoreThreads)), threads, 0, s, p);
    }
    if (plan.most <= 16) {
        p.slots = plan.few_slots;
        hipLaunchKernelGGL((score_few_kernel<TYPE, DP, EXACT>), dim3(items, (unsigned)p.slots), threads, 0, s, p);
        return hipGetLastError() == hipSuccess ? CODEGEMM_OK : CODEGEMM_LAUNCH_FAILED;
    }
    p.slots = plan.sum_slots;
    p.many = rows < rows_at_once(DP, false) ? rows : rows_at_once(DP, false);
    auto fn = score_sum_kernel<TYPE, DP, EXACT>;
    const size_t lds = RowSpace<DP>::bytes(p.many, 1);
    const int st = set_max_lds(reinterpret_cast<const void*>(fn), lds);
    if (st) return st;
    hipLaunchKernelGGL(fn, dim3(items, (unsigned)plan.sum_slots), threads, lds, s, p);
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
