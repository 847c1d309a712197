// Eviction: of every sequence and key head the tokens with the highest scores go, in order, to pages of another table.
//
// Selecting: a workgroup for a sequence and key head looks for the lowest score that stays, digit by digit of its bits (11, 11 and 10) from the top, with a
// histogram in LDS; scores are there too, up to kKeptKeys of them.  The bin in which the budget ends is the digit, and once all of a bin's tokens stay, lower digits make no
// difference.  Then it writes down the positions that stay, each wavefront a stretch of them behind those of the wavefronts before it: no atomics but on counts, so the
// same list whenever it runs.  A selection reads 4 bytes a token and is bound by its steps behind one another: 9 us for 8 heads of 1111 tokens, 14 us for 40 of 8192.
// Long sequences of few heads are shared by several workgroups, with their histograms in memory between four launches: 43 us for 24 heads of 100 001 (130 by one each).
//
// Moving: a workgroup takes 64 or 256 places of a head (or a block's, where those are more), keys or values.  Keys are rows of whole tokens and go as they are.  A
// value's row holds 16 tokens of a dimension: a lane has a dimension (4 bits: two) of 16 places and picks their codes out of up to 16 rows, which ones is the same for the whole
// wavefront, so rows, words and shifts are in scalar registers, and tokens that follow each other in a row share its load.  The move is bound by what it reads
// around a token that stays (a row of 16 for one value) and, where most stay, by the picking.  Three documents of 100 001 to 33 333 (4 bits, 24 heads): 82 us, 115 MB
// of tokens that stay read and written, 2.8 TB/s; of five prompts of 8192 to 2048 (8 bits): 20 us.
#include "attn_common.h"

namespace cg {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / kWave;
constexpr int kKeptKeys = 32768;            // 128 KB, at most
constexpr int kBins = 2048, kDigits = 3;    // two for each thread
constexpr int kDigitAt[kDigits] = {21, 10, 0};
// More than kLongKeys positions are shared by workgroups of kPartKeys each, up to kSelectGroups in all: one sequence of 100 000 tokens, 8 heads, is evicted from and gathered in
// 104 us, by one workgroup each in 178.  Fewer positions stay in one workgroup's LDS, in one launch.
constexpr int kLongKeys = 16384, kPartKeys = 8192, kPartKept = 12288, kSelectGroups = 256;
constexpr int kMoveThreads = 256;
// Places of a workgroup that moves: few, so that there are workgroups for every CU, or, where there are more than kManyUnits of these, many, whose rows come with fewer waits.
// With the gather of what stays: 32 sequences of 8 heads, 8192 tokens to 4096, 4 bits, 281 us with kManyTokens and 318 with kFewTokens; one of 1111 to 701, fp16, 26.7 and 15.9.
constexpr int kFewTokens = 64, kManyTokens = 256, kManyUnits = 4096;

// Between the launches of a selection by several workgroups.
struct PartState {
    unsigned always;        // tokens of the part that stay whatever they have
    uint32_t kind;          // kSome, kAll or kNone of the others
    uint32_t prefix;        // kSome: of the least key that stays, as far as it is known
    unsigned room;          // how many stay of the keys that begin with it
    unsigned before;        // tokens of the parts ahead that stay, as far as is known
};

enum { kSome = 0, kAll = 1, kNone = 2 };

struct EvictParams {
    CacheView from, to;
    const float* scores;
    float* to_scores;
    const int32_t* shift;
    int32_t *to_lens, *to_shift;
    int32_t* list;          // [sequence][head][most]: positions that stay
    int2* info;             // [sequence][head]: tokens that stay, the sequence's length
    int budget, first, last, most;
    int kept_keys;          // in LDS, a multiple of 4
    int parts;              // workgroups of a sequence and key head that select
    uint32_t* part_bins;    // [sequence][head][part][digit][kBins]
    PartState* states;      // [sequence][head][part]
    uint32_t by_pieces, by_runs;        // 2^32 over the pieces of a key, rounded up, and over its runs: i / n is the upper half of the product (0: n is 1)
    int unit;               // places of a workgroup that moves
    int units;              // .. of a sequence
};

// Scores as numbers that order as they do: NaN below all, -0 as 0.  0 is for what is no candidate.
__device__ __forceinline__ uint32_t key_of(float score)
{
    const uint32_t w = __builtin_bit_cast(uint32_t, score + 0.0f);
    const uint32_t k = w & 0x80000000u ? ~w : w | 0x80000000u;
    return score == score ? k : 1u;
}

// What is common to the workgroups that select: positions begin .. end - 1 of a sequence and key head.
struct Selector {
    const EvictParams& p;
    uint32_t *kept_keys, *bins, *shared;        // LDS: [p.kept_keys], [kBins], [2 kSelectWaves]
    int seq, head, tid, lane, wave;
    int len, n, last;                           // the sequence's length, positions there are, the last tokens' first one
    int begin, end;

    __device__ __forceinline__ Selector(const EvictParams& params, unsigned char* smem, int item) : p(params)
    {
        kept_keys = reinterpret_cast<uint32_t*>(smem);
        bins = kept_keys + p.kept_keys;
        shared = bins + kBins;
        const CacheView& c = p.from;
        seq = item / c.Hk; head = item % c.Hk;
        tid = threadIdx.x; lane = tid & (kWave - 1); wave = __builtin_amdgcn_readfirstlane(tid / kWave);
        const int held = c.max_pages << c.page_shift, given = c.lens[seq];
        len = given < 0 ? 0 : given;
        n = len < held ? len : held;
        last = len > p.last ? len - p.last : 0;
        begin = 0;
        end = n;
    }

    // The four tokens from t on (a multiple of 4): their keys; ~0 for those that stay whatever they have, 0 for those that are none.
    __device__ __forceinline__ u32x4_t look(int t) const
    {
        const CacheView& c = p.from;
        const int at = t < end ? t : begin, page = page_of(c, seq, at >> c.page_shift);         // (no branches: loads of several places are under way together)
        const float4_t x = *reinterpret_cast<const float4_t*>(p.scores + ((((size_t)(page < 0 ? 0 : page) * c.Hk + head) << c.page_shift) + (at & ((1 << c.page_shift) - 1))));
        u32x4_t k;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool always = t + i < p.first || t + i >= last;
            k[i] = page < 0 || t + i >= end ? 0u : always ? ~0u : key_of(x[i]);
        }
        return k;
    }
    __device__ __forceinline__ u32x4_t keys_at(int t) const
    {
        if (t - begin + 4 <= p.kept_keys) return *reinterpret_cast<const u32x4_t*>(kept_keys + (t - begin));
        return look(t);
    }
    __device__ __forceinline__ void clear_bins() const
    {
        for (int i = tid; i < kBins / 4; i += kSelectThreads) reinterpret_cast<u32x4_t*>(bins)[i] = u32x4_t{0, 0, 0, 0};
    }
    __device__ __forceinline__ static bool candidate(uint32_t k) { return k != 0u && k != ~0u; }

    // take(t, get(t)) for the thread's places t, several of which are under way at once.
    template <class Get, class Take>
    __device__ __forceinline__ void each(Get get, Take take) const
    {
        constexpr int AT_ONCE = 4;
        for (int t0 = begin + 4 * tid; t0 < end; t0 += 4 * AT_ONCE * kSelectThreads) {
            u32x4_t k[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) k[i] = t0 + 4 * i * kSelectThreads < end ? get(t0 + 4 * i * kSelectThreads) : u32x4_t{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
                if (t0 + 4 * i * kSelectThreads < end) take(t0 + 4 * i * kSelectThreads, k[i]);
        }
    }

    // Keys into LDS, the histogram of their first digit, and how many stay anyhow (to all threads).
    __device__ __forceinline__ unsigned first_digit() const
    {
        clear_bins();
        if (tid == 0) shared[0] = 0;
        __syncthreads();
        unsigned always = 0;
        each([&](int t) { return look(t); }, [&](int t, const u32x4_t& k) {
            if (t - begin + 4 <= p.kept_keys) *reinterpret_cast<u32x4_t*>(kept_keys + (t - begin)) = k;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                always += k[i] == ~0u;
                if (candidate(k[i])) atomicAdd(&bins[k[i] >> kDigitAt[0]], 1u);
            }
        });
        if (always) atomicAdd(&shared[0], always);
        __syncthreads();
        return shared[0];
    }
    // .. of a further one, among the keys that begin with `prefix`.
    __device__ __forceinline__ void further_digit(int digit, uint32_t prefix) const
    {
        clear_bins();
        __syncthreads();
        const uint32_t mask = ~0u << kDigitAt[digit - 1];
        each([&](int t) { return keys_at(t); }, [&](int, const u32x4_t& k) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (candidate(k[i]) && (k[i] & mask) == prefix) atomicAdd(&bins[k[i] >> kDigitAt[digit] & (kBins - 1)], 1u);
        });
        __syncthreads();
    }

    // The sum of x over the threads up to this one.
    __device__ __forceinline__ unsigned upto(unsigned x) const
    {
        x = wave_scan(x);
        __syncthreads();
        if (lane == kWave - 1) shared[wave] = x;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kSelectWaves - 1; ++w) x += w < wave ? shared[w] : 0u;
        return x;
    }
    // Thread i has the numbers of keys in bins kBins - 1 - 2 i and the one below.  The bin in which the first `room` keys from the top end, and how many of its own are among them.
    struct Found {
        int bin;
        unsigned room, all;     // all: in all bins
        unsigned count;         // in that bin
    };
    __device__ __forceinline__ Found find(unsigned c0, unsigned c1, unsigned room) const
    {
        const int b0 = kBins - 1 - 2 * tid;
        const unsigned to = upto(c0 + c1), before = to - c0 - c1;
        if (before < room && room <= to) {                                              // one thread
            const bool second = room > before + c0;
            shared[kSelectWaves] = (uint32_t)(second ? b0 - 1 : b0);
            shared[kSelectWaves + 1] = room - before - (second ? c0 : 0u);
            shared[kSelectWaves + 3] = second ? c1 : c0;
        }
        if (tid == kSelectThreads - 1) shared[kSelectWaves + 2] = to;
        __syncthreads();
        return Found{(int)shared[kSelectWaves], shared[kSelectWaves + 1], shared[kSelectWaves + 2], shared[kSelectWaves + 3]};
    }

    // Writes down the positions whose keys are above `least`, and of those that have it the first `equal` behind `sames` of others; the first as the `places`-th.
    // The number of those that stay.
    __device__ __forceinline__ unsigned write_down(uint32_t least, unsigned equal, unsigned places, unsigned sames) const
    {
        int32_t* list = p.list + ((size_t)seq * p.from.Hk + head) * p.most;
        // each wavefront's stretch: how many are above, and are, the least; then their places
        const int stretch = ceil_div(ceil_div(end - begin, 4 * kWave), kSelectWaves) * 4 * kWave, from = begin + wave * stretch, to = from + stretch < end ? from + stretch : end;
        unsigned above = 0, same = 0;
        for (int t = from + 4 * lane; t < to; t += 4 * kWave) {
            const u32x4_t k = keys_at(t);
#pragma unroll
            for (int i = 0; i < 4; ++i) { above += k[i] > least; same += least != 0u && k[i] == least; }
        }
        above = wave_sum(above);
        same = wave_sum(same);
        __syncthreads();
        if (lane == 0) { shared[wave] = above; shared[kSelectWaves + wave] = same; }
        __syncthreads();
        unsigned all = places, seen = sames;
#pragma unroll
        for (int w = 0; w < kSelectWaves; ++w) {
            const unsigned a = shared[w], s = shared[kSelectWaves + w], taken = seen >= equal ? 0u : equal - seen < s ? equal - seen : s;
            if (w == wave) { places = all; sames = seen; }
            all += a + taken;
            seen += s;
        }
        for (int t0 = from; t0 < to; t0 += 4 * kWave) {
            const int t = t0 + 4 * lane;
            u32x4_t k = {0, 0, 0, 0};
            if (t < to) k = keys_at(t);
            unsigned s4 = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) s4 += least != 0u && k[i] == least;
            // (both counts of a wavefront's 256 tokens in one sum)
            unsigned a4 = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) a4 += k[i] > least;
            const unsigned both = wave_scan(s4 << 16 | a4);
            unsigned s_before = sames + (both >> 16) - s4, a_before = (both & 0xffffu) - a4;
            auto taken_of = [&](unsigned upto_same) { return (upto_same < equal ? upto_same : equal) - (sames < equal ? sames : equal); };      // since the wavefront's first
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool is_above = k[i] > least, is_same = least != 0u && k[i] == least;
                const unsigned at = places + a_before + taken_of(s_before);
                if ((is_above || (is_same && s_before < equal)) && at < (unsigned)p.most) list[at] = t + i;
                a_before += is_above;
                s_before += is_same;
            }
            const unsigned whole = (unsigned)__builtin_amdgcn_readlane((int)both, kWave - 1);
            places += (whole & 0xffffu) + taken_of(sames + (whole >> 16));
            sames += whole >> 16;
        }
        return all;
    }
};

// A sequence and key head by one workgroup.
__global__ void __launch_bounds__(kSelectThreads) kv_select_kernel(const EvictParams p)
{
    extern __shared__ __align__(16) unsigned char smem[];
    const Selector s(p, smem, blockIdx.x);
    const unsigned always = s.first_digit();
    unsigned room = (unsigned)p.budget - always;
    const int b0 = kBins - 1 - 2 * s.tid;
    Selector::Found f = s.find(s.bins[b0], s.bins[b0 - 1], room);
    uint32_t least = 0;                                                                 // all stay
    unsigned equal = 0;
    if (always + f.all > (unsigned)p.budget) {
        least = ~0u - 1;                                                                // (no candidate's key is that: none stays)
        if (room != 0) {
            least = (uint32_t)f.bin << kDigitAt[0];
            equal = f.room;
            bool all_of_bin = f.room == f.count;
#pragma unroll
            for (int digit = 1; digit < kDigits; ++digit) {
                if (all_of_bin) continue;                                               // (uniform) what is left to find out makes no difference
                s.further_digit(digit, least);
                f = s.find(s.bins[b0], s.bins[b0 - 1], equal);
                least |= (uint32_t)f.bin << kDigitAt[digit];
                equal = f.room;
                all_of_bin = f.room == f.count;
            }
            if (all_of_bin && least != 0u) { least -= 1; equal = 0; }                     // all keys from the bin on
        }
    }
    const unsigned all = s.write_down(least, equal, 0, 0);
    if (s.tid == 0) p.info[blockIdx.x] = int2{(int)all, s.len};
}

// .. by several, each with its part of the positions, in four launches: the histogram of the first digit, of the second, of the third, and what stays.  Every workgroup adds up
// the histograms of the digit before, and of those of the parts ahead of its own what is above the bin that was found.
template <int PASS>
__global__ void __launch_bounds__(kSelectThreads) kv_select_part_kernel(const EvictParams p)
{
    extern __shared__ __align__(16) unsigned char smem[];
    const int item = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
    Selector s(p, smem, item);
    const int size = ceil_div(ceil_div(s.n, 4), p.parts) * 4;
    s.begin = part * size < s.n ? part * size : s.n;
    s.end = s.begin + size < s.n ? s.begin + size : s.n;
    uint32_t* bins_of = p.part_bins + (size_t)item * p.parts * kDigits * kBins;         // [part][digit][kBins]
    PartState* states = p.states + (size_t)item * p.parts;
    if constexpr (PASS == 0) {
        const unsigned always = s.first_digit();
        for (int i = s.tid; i < kBins; i += kSelectThreads) bins_of[(size_t)part * kDigits * kBins + i] = s.bins[i];
        if (s.tid == 0) states[part] = PartState{always, kSome, 0, 0, 0};
        return;
    }
    // of the item: what came out of the digits before, the same in all parts
    unsigned always = 0, always_before = 0;
    for (int i = s.lane; i < p.parts; i += kWave) {
        const unsigned x = states[i].always;
        always += x;
        always_before += i < part ? x : 0u;
    }
    always = wave_sum(always);
    always_before = wave_sum(always_before);
    if constexpr (PASS == kDigits)                                                      // the part's keys, for what follows
        s.each([&](int t) { return s.look(t); }, [&](int t, const u32x4_t& k) {
            if (t - s.begin + 4 <= p.kept_keys) *reinterpret_cast<u32x4_t*>(s.kept_keys + (t - s.begin)) = k;
        });
    const unsigned room = PASS == 1 ? (unsigned)p.budget - always : states[part].room;
    uint32_t least = PASS == 1 ? 0u : states[part].prefix;
    unsigned before = PASS == 1 ? always_before : states[part].before;                  // what stays ahead of this part, of what is known
    const int b0 = kBins - 1 - 2 * s.tid;
    unsigned c0 = 0, c1 = 0, ahead0 = 0, ahead1 = 0;
#pragma unroll 8
    for (int i = 0; i < p.parts; ++i) {
        const u32x2_t x = *reinterpret_cast<const u32x2_t*>(bins_of + ((size_t)i * kDigits + PASS - 1) * kBins + b0 - 1);
        c0 += x[1];
        c1 += x[0];
        ahead0 += i < part ? x[1] : 0u;
        ahead1 += i < part ? x[0] : 0u;
    }
    const Selector::Found f = s.find(c0, c1, room);
    const uint32_t kind = PASS != 1 ? states[part].kind : always + f.all <= (unsigned)p.budget ? kAll : room == 0u ? kNone : kSome;
    const bool all_stay = kind == kAll, none = kind == kNone;
    unsigned equal = 0, sames = 0;
    {
        const unsigned mine = all_stay ? (PASS == 1 ? ahead0 + ahead1 : 0u) : none ? 0u : (b0 > f.bin ? ahead0 : 0u) + (b0 - 1 > f.bin ? ahead1 : 0u);
        const unsigned same = all_stay || none ? 0u : (b0 == f.bin ? ahead0 : 0u) + (b0 - 1 == f.bin ? ahead1 : 0u);
        const unsigned sum = s.upto(mine);
        __syncthreads();
        if (s.tid == kSelectThreads - 1) s.shared[kSelectWaves] = sum;
        if (s.tid == 0) s.shared[kSelectWaves + 1] = 0;
        __syncthreads();
        if (same) atomicAdd(&s.shared[kSelectWaves + 1], same);
        __syncthreads();
        before += s.shared[kSelectWaves];
        sames = s.shared[kSelectWaves + 1];
    }
    if (all_stay) least = 0;
    else if (none) least = ~0u - 1;
    else {
        least |= (uint32_t)f.bin << kDigitAt[PASS - 1];
        equal = f.room;
    }
    if constexpr (PASS < kDigits) {
        if (!all_stay && !none) {
            s.further_digit(PASS, least);
            for (int i = s.tid; i < kBins; i += kSelectThreads) bins_of[((size_t)part * kDigits + PASS) * kBins + i] = s.bins[i];
        }
        __syncthreads();
        // (every part reads its own state only, but for `always`, which stays)
        if (s.tid == 0) {
            states[part].kind = kind;
            states[part].prefix = least;
            states[part].room = equal;
            states[part].before = before;
        }
    } else {
        const unsigned all = s.write_down(least, equal, before + (sames < equal ? sames : equal), sames);
        if (part == p.parts - 1 && s.tid == 0) p.info[item] = int2{(int)all, s.len};
    }
}

// 8 bits: a code in another scale.
template <int TYPE>
__device__ __forceinline__ uint32_t again(uint32_t code, float ratio)
{
    if constexpr (TYPE == CODEGEMM_KV_INT8) return (uint32_t)(uint8_t)(int8_t)(int)rintf(__builtin_amdgcn_fmed3f((float)(int8_t)code * ratio, -127.0f, 127.0f));
    else {
        const float x = __builtin_amdgcn_fmed3f((float)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)code, 1.0f, false)[0] * ratio, -448.0f, 448.0f);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 255u;
    }
}

// The four bits of token j of a word's eight.
__device__ __forceinline__ constexpr int bit_of(int j) { return 4 * (j >> 1) + 16 * (j & 1); }

// i / n for i < 2^16 and n < 2^8, by 2^32 / n rounded up.
__device__ __forceinline__ int over(int i, uint32_t by) { return by != 0 ? (int)__umulhi((uint32_t)i, by) : i; }

// Units of places of a sequence and key head, keys or values.  (Values in fp16: a load for each token; sharing rows' loads as the others do took 116 us where this takes 63.)
template <int TYPE>
__global__ void __launch_bounds__(kMoveThreads) kv_move_kernel(const EvictParams p)
{
    constexpr bool FOUR = TYPE == CODEGEMM_KV_INT4, SCALED = TYPE == CODEGEMM_KV_INT8 || TYPE == CODEGEMM_KV_FP8;
    __shared__ int2 source[kMoveThreads];                       // [token]: page and slot
    __shared__ u32x2_t value_row[kMoveThreads];                 // [token]: where its 16 tokens' values begin in the pool, in bytes, and above bit 60 which of them it is
    __shared__ int page_to[kMoveThreads / 16];                  // [16 tokens]: the page that they go to, or -1
    __shared__ float old[kMoveThreads];                         // [token]: its scale so far
    __shared__ uint32_t largest[kMoveThreads];                  // [block]: the bits of its scale
    const CacheView &a = p.from, &b = p.to;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave), D = a.D;
    const int head = blockIdx.x % a.Hk, item = blockIdx.x / a.Hk, seq = item / p.units;
    const bool values = blockIdx.y != 0;
    // (the first unit's positions are asked for beside the counts, which say what of them there is)
    const int32_t* list = p.list + ((size_t)seq * a.Hk + head) * p.most;
    auto listed = [&](int unit) { const int i = unit * p.unit + tid; return tid < p.unit && i < p.most ? list[i] : 0; };
    int mine = listed(item % p.units);
    const int2 info = p.info[(size_t)seq * a.Hk + head];
    if (item % p.units == 0 && head == 0 && !values && tid == 0) {
        p.to_lens[seq] = info.x;
        if (p.to_shift) p.to_shift[seq] = (p.shift ? p.shift[seq] : 0) + info.y - info.x;
    }
    const int mask = (1 << a.page_shift) - 1;
    for (int unit = item % p.units;; unit += p.units) {
        const int first = unit * p.unit, count = info.x - first < p.unit ? info.x - first : p.unit;
        if (count <= 0) return;
        __syncthreads();
        if (SCALED) {
            if (tid < p.unit) largest[tid] = 0;
            __syncthreads();
        }
        if (tid < kMoveThreads / 16) page_to[tid] = 16 * tid < count ? page_of(b, seq, (first + 16 * tid) >> b.page_shift) : -1;
        if (tid < count) {
            const int t = mine, page = page_of(a, seq, t >> a.page_shift), slot = t & mask;       // (there is a page)
            source[tid] = int2{page, slot};
            const unsigned long long row = page_at(a, page, head) + (size_t)(slot & ~15) * D, at = FOUR ? row / 2 : TYPE == CODEGEMM_KV_FP16 ? row * 2 : row;
            value_row[tid] = u32x2_t{(uint32_t)at, (uint32_t)(at >> 32) | (uint32_t)(slot & 15) << 28};
            if constexpr (SCALED) {
                const float s = (values ? a.v_scales : a.k_scales)[scales_at(a, page, head) + (slot >> a.block_shift)];
                old[tid] = s;
                atomicMax(&largest[tid >> a.block_shift], __builtin_bit_cast(uint32_t, s));         // (bits order as scales do, a NaN above all)
            }
            if (!values && p.to_scores) {
                const int to = page_of(b, seq, (first + tid) >> b.page_shift);
                if (to >= 0)
                    p.to_scores[(((size_t)to * b.Hk + head) << b.page_shift) + ((first + tid) & mask)] = p.scores[(((size_t)page * a.Hk + head) << a.page_shift) + slot];
            }
        }
        mine = listed(unit + p.units);
        __syncthreads();
        auto ratio_of = [&](int token) {                        // 1: codes stay
            const float s = old[token], now = __builtin_bit_cast(float, largest[token >> a.block_shift]);
            return s == now ? 1.0f : s > 0.0f && s < now ? s / now : 0.0f;
        };
        if constexpr (SCALED) {
            const int block = tid << b.block_shift, to = block < count ? page_to[block >> 4] : -1;
            if (to >= 0) (values ? b.v_scales : b.k_scales)[scales_at(b, to, head) + (((first + block) & mask) >> b.block_shift)] = __builtin_bit_cast(float, largest[tid]);
        }
        if (!values) {
            const int pieces = TYPE == CODEGEMM_KV_FP16 ? D / 8 : FOUR ? D / 32 : D / 16;           // of 16 bytes, of a token
            constexpr int AT_ONCE = 4;
            for (int i0 = tid; i0 < count * pieces; i0 += AT_ONCE * kMoveThreads) {
                u32x4_t x[AT_ONCE];
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) {
                    const int i = i0 + k * kMoveThreads, token = over(i, p.by_pieces);
                    if (i < count * pieces) x[k] = reinterpret_cast<const u32x4_t*>(a.k)[((((size_t)source[token].x * a.Hk + head) << a.page_shift) + source[token].y) * pieces + (i - token * pieces)];
                }
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) {
                    const int i = i0 + k * kMoveThreads, token = over(i, p.by_pieces), t = first + token;
                    const int to = i < count * pieces ? page_to[token >> 4] : -1;
                    if (to < 0) continue;
                    if constexpr (SCALED) {
                        const float ratio = ratio_of(token);
                        if (ratio != 1.0f) {
#pragma unroll
                            for (int w = 0; w < 4; ++w) {
                                uint32_t y = 0;
#pragma unroll
                                for (int e = 0; e < 4; ++e) y |= again<TYPE>(x[k][w] >> (8 * e) & 255u, ratio) << (8 * e);
                                x[k][w] = y;
                            }
                        }
                    }
                    reinterpret_cast<u32x4_t*>(b.k)[((((size_t)to * b.Hk + head) << b.page_shift) + (t & mask)) * pieces + (i - token * pieces)] = x[k];
                }
            }
            if constexpr (FOUR) {
                for (int i = tid; i < count * a.runs; i += kMoveThreads) {
                    const int token = over(i, p.by_runs), run = i - token * a.runs, t = first + token, to = page_to[token >> 4];
                    if (to >= 0)
                        reinterpret_cast<uint32_t*>(b.k_scales)[runs_at(b, to, head, t & mask) + run] =
                            reinterpret_cast<const uint32_t*>(a.k_scales)[runs_at(a, source[token].x, head, source[token].y) + run];
                }
            }
            continue;
        }
        for (int group = wave; 16 * group < count; group += kMoveThreads / kWave) {
            const int t = first + 16 * group, here = count - 16 * group < 16 ? count - 16 * group : 16;
            const int to = __builtin_amdgcn_readfirstlane(page_to[group]);
            if (to < 0) continue;
            // Lane j has the group's j-th token: where its row begins, and which of the row's 16 it is.  Tokens that follow each other in a row share its load: `heads` are those
            // that begin one.
            const u32x2_t row_of = value_row[16 * group + ((lane & 15) < here ? lane & 15 : 0)];
            const uint32_t before_lo = (uint32_t)__shfl_up((int)row_of[0], 1), before_hi = (uint32_t)__shfl_up((int)row_of[1], 1);
            const uint32_t heads = (uint32_t)__ballot(lane < here && (lane == 0 || before_lo != row_of[0] || (before_hi ^ row_of[1]) << 4 != 0));
            float ratio = 1.0f;                                 // of the lane's token
            if constexpr (SCALED) ratio = ratio_of(16 * group + ((lane & 15) < here ? lane & 15 : 0));
            // .. and how a code goes from its row to its place: bits 0 to 4 where it is in its word, 8 to 12 where it comes, 16 on which word (4 bits: its own, its place's; 8: two bits each)
            const uint32_t in_row = row_of[1] >> 28, place = lane & 15;
            const uint32_t how_of = FOUR ? (uint32_t)bit_of(in_row & 7) | (uint32_t)bit_of(place & 7) << 8 | in_row >> 3 << 16 | place >> 3 << 17
                                         : 8 * (in_row & 3) | 8 * (place & 3) << 8 | in_row >> 2 << 16 | place >> 2 << 18;
            const size_t at = page_at(b, to, head) + (size_t)(t & mask) * D;
            constexpr int WORDS = TYPE == CODEGEMM_KV_FP16 ? 8 : 4, ROWS = 4;            // of a lane's part of a row; rows that are asked for at once
            for (int d = lane; d < (FOUR ? D / 2 : D); d += kWave) {                               // (4 bits: two dimensions a lane)
                uint32_t w[WORDS] = {0};
                if constexpr (TYPE == CODEGEMM_KV_FP16) {       // a load for each token: of one row, they are of the same lines
                    uint32_t x[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)row_of[0], j), hi = (uint32_t)__builtin_amdgcn_readlane((int)row_of[1], j);
                        x[j] = reinterpret_cast<const uint16_t*>(a.v + ((unsigned long long)(hi & 0x0fffffffu) << 32 | lo) + 2 * (hi >> 28))[(uint32_t)d * 16];
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j >> 1] |= j < here ? x[j] << (16 * (j & 1)) : 0u;
                }
                for (uint32_t left = TYPE == CODEGEMM_KV_FP16 ? 0u : heads; left != 0;) {
                    u32x4_t x[ROWS][WORDS / 4];
                    int from[ROWS + 1];
#pragma unroll
                    for (int k = 0; k < ROWS; ++k) {
                        from[k] = left != 0 ? __builtin_ctz(left) : here;
                        if (left != 0) {
                            const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)row_of[0], from[k]), hi = (uint32_t)__builtin_amdgcn_readlane((int)row_of[1], from[k]);
                            const u32x4_t* row = reinterpret_cast<const u32x4_t*>(a.v + ((unsigned long long)(hi & 0x0fffffffu) << 32 | lo));
#pragma unroll
                            for (int i = 0; i < WORDS / 4; ++i) x[k][i] = row[d * (WORDS / 4) + i];
                        }
                        left &= left - 1;
                    }
                    from[ROWS] = left != 0 ? __builtin_ctz(left) : here;
#pragma unroll
                    for (int k = 0; k < ROWS; ++k)
                        for (int j = from[k]; j < from[k + 1]; ++j) {
                            const uint32_t how = (uint32_t)__builtin_amdgcn_readlane((int)how_of, j), to_bit = how >> 8 & 31u;
                            // (which word a code is in and comes into by conditions and masks that are the same for all lanes: chosen by branches, words
                            // are copied about)
                            const u32x4_t y = x[k][0];
                            auto mask_of = [&](uint32_t is) { return is != 0 ? ~0u : 0u; };
                            if constexpr (FOUR) {
                                const bool upper = how & 0x10000u;
                                const uint32_t second = mask_of(how & 0x20000u), c0 = __builtin_amdgcn_ubfe(upper ? y[1] : y[0], how, 4) << to_bit, c1 = __builtin_amdgcn_ubfe(upper ? y[3] : y[2], how, 4) << to_bit;
                                w[0] |= c0 & ~second;
                                w[1] |= c0 & second;
                                w[2] |= c1 & ~second;
                                w[3] |= c1 & second;
                            } else if constexpr (SCALED) {
                                const bool odd = how & 0x10000u, upper = how & 0x20000u;
                                uint32_t code = upper ? (odd ? y[3] : y[2]) : (odd ? y[1] : y[0]);
                                code = __builtin_amdgcn_ubfe(code, how, 8);
                                const float by = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, ratio), j));
                                if (by != 1.0f) code = again<TYPE>(code, by);
                                code <<= to_bit;
                                const uint32_t to_word = how >> 18 & 3u;
#pragma unroll
                                for (int i = 0; i < 4; ++i) w[i] |= code & mask_of(to_word == (uint32_t)i ? 1u : 0u);
                            }
                        }
                }
                u32x4_t* dst = reinterpret_cast<u32x4_t*>(b.v + (FOUR ? at / 2 : at * (WORDS / 4))) + (size_t)d * (WORDS / 4);
#pragma unroll
                for (int i = 0; i < WORDS / 4; ++i) {
                    u32x4_t y = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
                    if (here < 16) {                            // the group's other places stay as they are
                        const u32x4_t was = dst[i];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            constexpr int PER = FOUR ? 8 : TYPE == CODEGEMM_KV_FP16 ? 2 : 4;      // tokens of a word
                            const int first_of = FOUR ? 8 * (e & 1) : PER * (4 * i + e);
                            uint32_t taken = 0;
#pragma unroll
                            for (int q = 0; q < PER; ++q) taken |= first_of + q < here ? (FOUR ? 15u << bit_of(q) : PER == 2 ? 0xffffu << (16 * q) : 255u << (8 * q)) : 0u;
                            y[e] |= was[e] & ~taken;
                        }
                    }
                    dst[i] = y;
                }
            }
        }
        if constexpr (FOUR) {
            for (int i = tid; i < count * a.runs; i += kMoveThreads) {
                const int token = over(i, p.by_runs), run = i - token * a.runs, t = first + token, to = page_to[token >> 4], slot = source[token].y;
                if (to < 0) continue;
                const uint16_t* src = reinterpret_cast<const uint16_t*>(a.v_scales) + 2 * runs_at(a, source[token].x, head, slot & ~15) + 32 * run + (slot & 15);
                uint16_t* dst = reinterpret_cast<uint16_t*>(b.v_scales) + 2 * runs_at(b, to, head, t & mask & ~15) + 32 * run + (t & 15);
                dst[0] = src[0];
                dst[16] = src[16];
            }
        }
    }
}

namespace {

constexpr size_t kFixedArea = (size_t)kCounterAreaWords * sizeof(uint32_t) + kPairAreaBytes;       // that other calls keep their counters in

struct EvictPlan {
    int most, unit, units, kept_keys, parts;
    size_t info, part_bins, states, bytes;
};

int evict_plan(const codegemm_kv_cache* from, const codegemm_evict_desc* d, EvictPlan* p)
{
    const int st = check_cache(from, false);
    if (st) return st;
    if (!d || d->budget < 1 || d->keep_first < 0 || d->keep_last < 0 || (long long)d->keep_first + d->keep_last > d->budget || d->max_kv < 1) return CODEGEMM_INVALID_ARG;
    const long long items = (long long)from->num_seqs * from->kv_heads;
    if (too_many(items, kSelectThreads)) return CODEGEMM_UNSUPPORTED;
    const int held = from->max_pages * from->page_size, known = d->max_kv < held ? d->max_kv : held;
    p->most = d->budget < held ? d->budget : held;
    const bool scaled = from->dtype == CODEGEMM_KV_INT8 || from->dtype == CODEGEMM_KV_FP8;
    const int kept = p->most < known ? p->most : known;
    const int tokens = 2 * items * ceil_div(kept, kFewTokens) > kManyUnits ? kManyTokens : kFewTokens;
    p->unit = scaled && from->scale_block > tokens ? from->scale_block : tokens;
    p->units = ceil_div(kept, p->unit);
    // (whatever the host knows: fewer workgroups have more units each)
    const long long room = 0xffffffffll / kMoveThreads / items;
    if (p->units > room) p->units = (int)room;
    p->kept_keys = known < kKeptKeys ? ceil_div(known, 4) * 4 : kKeptKeys;
    // Long sequences of few heads: several workgroups, which takes four launches.
    const long long parts = known <= kLongKeys ? 1 : kSelectGroups / items < ceil_div(known, kPartKeys) ? kSelectGroups / items : ceil_div(known, kPartKeys);
    p->parts = parts < 1 ? 1 : (int)parts;
    p->info = kFixedArea + ((size_t)items * p->most * sizeof(int32_t) + 255) / 256 * 256;
    p->part_bins = p->info + ((size_t)items * sizeof(int2) + 255) / 256 * 256;
    const size_t many = p->parts > 1 ? (size_t)items * p->parts : 0;
    p->states = p->part_bins + many * kDigits * kBins * sizeof(uint32_t);
    p->bytes = many ? p->states + many * sizeof(PartState) : p->info + (size_t)items * sizeof(int2);
    return CODEGEMM_OK;
}

template <int TYPE>
void launch_move(const EvictParams& p, hipStream_t s)
{
    hipLaunchKernelGGL(kv_move_kernel<TYPE>, dim3((unsigned)p.units * (unsigned)(p.from.seqs * p.from.Hk), 2), dim3(kMoveThreads), 0, s, p);
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" size_t codegemm_kv_evict_workspace_bytes(const codegemm_kv_cache* from, const codegemm_evict_desc* desc)
{
    EvictPlan plan;
    return evict_plan(from, desc, &plan) ? 0 : plan.bytes;
}

extern "C" int codegemm_kv_evict(const codegemm_kv_cache* from, const codegemm_kv_cache* to, const codegemm_evict_desc* desc, const float* scores, const int32_t* shift,
                                 float* to_scores, int32_t* to_lens, int32_t* to_shift, void* workspace, size_t workspace_bytes, void* stream)
{
    EvictPlan plan;
    int st = evict_plan(from, desc, &plan);
    if (!st) st = check_cache(from, true);
    if (!st) st = check_cache(to, true);
    if (st) return st;
    if (from->kv_heads != to->kv_heads || from->head_dim != to->head_dim || from->page_size != to->page_size || from->dtype != to->dtype || from->num_seqs != to->num_seqs ||
        (from->dtype != CODEGEMM_KV_FP16 && from->scale_block != to->scale_block))
        return CODEGEMM_INVALID_ARG;
    if (!scores || !to_lens || !workspace || misaligned(scores) || misaligned(workspace) || (to_scores && misaligned(to_scores))) return CODEGEMM_INVALID_ARG;
    if (misaligned_ints(to_lens) || (shift && misaligned_ints(shift)) || (to_shift && misaligned_ints(to_shift))) return CODEGEMM_INVALID_ARG;
    if (workspace_bytes < plan.bytes) return CODEGEMM_WORKSPACE_TOO_SMALL;
    EvictParams p;
    p.from = cache_view(*from);
    p.to = cache_view(*to);
    p.scores = scores;
    p.to_scores = to_scores;
    p.shift = shift;
    p.to_lens = to_lens;
    p.to_shift = to_shift;
    p.list = reinterpret_cast<int32_t*>(static_cast<unsigned char*>(workspace) + kFixedArea);
    p.info = reinterpret_cast<int2*>(static_cast<unsigned char*>(workspace) + plan.info);
    p.budget = desc->budget; p.first = desc->keep_first; p.last = desc->keep_last;
    p.most = plan.most; p.kept_keys = plan.kept_keys; p.unit = plan.unit; p.units = plan.units;
    const int pieces = from->head_dim / (from->dtype == CODEGEMM_KV_FP16 ? 8 : from->dtype == CODEGEMM_KV_INT4 ? 32 : 16);
    auto inverse = [](int n) { return n > 1 ? (uint32_t)(((1ull << 32) + (unsigned)n - 1) / (unsigned)n) : 0u; };
    p.by_pieces = inverse(pieces);
    p.by_runs = inverse(p.from.runs);
    p.parts = plan.parts;
    p.part_bins = reinterpret_cast<uint32_t*>(static_cast<unsigned char*>(workspace) + plan.part_bins);
    p.states = reinterpret_cast<PartState*>(static_cast<unsigned char*>(workspace) + plan.states);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const unsigned items = (unsigned)(p.from.seqs * p.from.Hk);
    if (plan.parts > 1) {
        p.kept_keys = 0;
        const size_t lds = ((size_t)kBins + 2 * kSelectWaves) * sizeof(uint32_t);
        const dim3 grid(items * (unsigned)plan.parts), threads(kSelectThreads);
        hipLaunchKernelGGL(kv_select_part_kernel<0>, grid, threads, lds, s, p);
        hipLaunchKernelGGL(kv_select_part_kernel<1>, grid, threads, lds, s, p);
        hipLaunchKernelGGL(kv_select_part_kernel<2>, grid, threads, lds, s, p);
        p.kept_keys = kPartKept;
        hipLaunchKernelGGL(kv_select_part_kernel<3>, grid, threads, lds + (size_t)p.kept_keys * sizeof(uint32_t), s, p);
    } else {
        const size_t lds = ((size_t)plan.kept_keys + kBins + 2 * kSelectWaves) * sizeof(uint32_t);
        st = set_max_lds(reinterpret_cast<const void*>(kv_select_kernel), lds);
        if (st) return st;
        hipLaunchKernelGGL(kv_select_kernel, dim3(items), dim3(kSelectThreads), lds, s, p);
    }
    if (from->dtype == CODEGEMM_KV_FP16) launch_move<CODEGEMM_KV_FP16>(p, s);
    else if (from->dtype == CODEGEMM_KV_INT8) launch_move<CODEGEMM_KV_INT8>(p, s);
    else if (from->dtype == CODEGEMM_KV_INT4) launch_move<CODEGEMM_KV_INT4>(p, s);
    else launch_move<CODEGEMM_KV_FP8>(p, s);
    return hipGetLastError() == hipSuccess ? CODEGEMM_OK : CODEGEMM_LAUNCH_FAILED;
}
