// Attention of one query token per sequence over the paged cache.
//
// An item is a sequence and up to 16 query heads that share a key head; its keys are steps of 32 tokens.  The workgroups look at all lengths
// and cut the items into pieces such that each has about one, whatever the lengths are; the last workgroup of an item to finish joins its
// pieces.
//
// Each wavefront works on its own on every NW-th step (of 8, 4 or 2 wavefronts): scores as S^T = K Q^T on the matrix cores (rows: tokens, columns: query heads),
// the softmax's running maximum and sum per column, and O^T += V^T P^T.  The right operand of the second product is what the score tiles
// leave in the lanes, because a step's tokens are dealt out to the four lane groups g in runs of 8: row 4 g + r of score tile n is
// token 8 g + 4 n + r, so lane group g holds 8 consecutive tokens of P^T, and the value pool has them next to each other for every
// dimension.  The memory pipeline writes keys, values and scales of the next steps into a ring in LDS (global_load .. lds), where every lane
// finds its own operands again; no wavefront waits for another before the end of an item.
// 8-bit codes become fp16 exactly on the way into the matrix cores; a key's scale multiplies its score, a value's scale its weight.
//
// Bound by: the cache's bytes, where there are many.  32 sequences of 206 376 tokens, 64 and 8 heads of 128, 8 bits: 82 us, 5.2 TB/s; 3 of 240 551,
// fp8: 86 us, 5.7 TB/s (a large copy: 4.85, read and written); loads that nothing is computed with take 81 and 87.  13 of twenty heads of 64 in fp16
// with a window of 1500: 22.5 us, 4.0 TB/s.  Steps held in registers instead of LDS took 93 and 136 us at best.
// Shortest: 700 tokens of one sequence, 10.3 us, of which 6.3 are one step of every wavefront (of 100 tokens) and 4 the exchange between workgroups;
// three steps in one workgroup take 11.3.  8000 tokens: 15.2.
// Farthest from the bytes: long sequences with few key heads, whose pieces are as many as there are workgroups and are added up by one of them, 8 at a time:
// 100 000 tokens with 8, 2 and 1 key heads take 45.7, 33.2 and 44.0 us for 205, 51 and 26 MB, 32 000 tokens 23.6, 26.6 and 25.7.
// Heads of 80 are worked on as 128: 32 sequences of 206 376 tokens take 70 us for 265 MB, 3.8 TB/s; of 256, one wavefront a SIMD: 240 us for 848 MB, 3.5 TB/s.
// 4 bits: a code is (code + 16) scale + offset in fp16 on the way into the matrix cores, two instructions for a pair of codes and one multiply-add, which is exact to
// the cached value's one rounding; scales and offsets come with the codes into the ring.  The running maximum is not followed from step to step, but only where a
// weight would pass 2^15.5: the largest lies between 2^10 and that.  Bound by the codes' way into operands as much as by bytes: 32 sequences of 206 000 tokens,
// 58.7 us, 4.1 TB/s (of loads alone 52, of what is computed alone 55); three of 250 000 70.7 us, 4.5 TB/s; 13 of twenty heads of 64 with a window of 1500 19.2 us;
// one of 701 9.3.
#include <cmath>
#include <type_traits>

#include "attn_common.h"

namespace cg {

constexpr int kDecodeRows = 16;             // query heads of a workgroup
constexpr int kDecodeUnits = 256;           // compute units
constexpr int kJoinSteps = 1;               // what joining pieces takes, in steps of a wavefront: an item that is longer by less stays whole
constexpr int kRoundSteps = 10;             // .. and a second piece for the same workgroup
constexpr int kJoined = 8;                  // pieces that are joined at a time
constexpr int kMostGroups = 1 << 20;        // workgroups of a launch, which has fewer than 2^32 threads
constexpr float kLeastLog = -40.0f;         // of a scale's logarithm in the running maximum
// The largest weight is 2^kLift, so that fp16 holds weights down to 2^-28 of it with all their places and down to 2^-38 at all: behind one key that has most of
// the weight and values near zero, thousands of others with little weight each make the result.  (With 1 for the largest, the weights of the keys that share
// a wavefront with such a key were off by 2.6 % at 15 nats below it, by 44 % at 17, and zero at 18.)  Not from scores of kFine on, which may have no place for it.
constexpr float kLift = 14.0f, kFine = 1048576.0f;
// 4 bits: the largest weight lies between 2^10 and 2^15.5, so that sums are seldom rescaled (below).  In the worst case fp16 holds weights with all their places down to 2^-24 of it, 16.6
// nats below the largest score instead of 19.4, and at all down to 2^-34.
constexpr float kLowLift = 10.0f, kReach = 5.5f;

struct DecodeParams {
    CacheView c;
    const _Float16* q;
    _Float16* out;
    float* part;            // [piece of an item that has several][16 (D + 2)]: [D / 16][64 lanes][4] sums, [16] maximum and weight
    uint32_t* counters;     // of such an item: that of its first piece
    Pair* stats;            // [sequence][query head], or NULL: what scores are a weight's logarithm above, and 1 / the weights' sum
    int slots;              // workgroups that run at once
    int r;                  // query heads of a key head
    int tiles;              // items of 16 of them
    int q_stride, out_stride;
    int window;
    float scale;            // times log2(e)
};

typedef __attribute__((address_space(3))) u32x4_t lds_words4;
typedef __attribute__((address_space(3))) u32x2_t lds_words2;
typedef __attribute__((address_space(3))) uint32_t lds_word;
typedef __attribute__((address_space(3))) float4_t lds_float4;
typedef __attribute__((address_space(3))) float lds_float1;
typedef __attribute__((address_space(4))) const int32_t const_int;

// A step in LDS, per wavefront: keys, values, the tokens' scales.  A workgroup has a compute unit to itself, or, NARROW, half of one.
template <int TYPE, int DP, bool NARROW>
struct DecodeStep {
    static constexpr bool kHalf = TYPE == CODEGEMM_KV_FP16, kFour = TYPE == CODEGEMM_KV_INT4;
    static constexpr bool kScaled = !kHalf && !kFour;                // scales go to scores and weights
    static constexpr int kSize = kHalf ? 2 : 1;
    static constexpr int kTokens = 32, kRun = 8, kTiles = 2;
    static constexpr int kPart = kTokens * DP * kSize / (kFour ? 2 : 1);       // bytes of the keys, and of the values
    static constexpr int kRuns = DP / 32;                            // 4 bits: scales and offsets of a token, at most
    static constexpr int kRunBytes = 64 * kRuns;                     // .. of 16 tokens
    static constexpr int kScaleBytes = kHalf ? 0 : !kFour ? 256 : DP == 256 ? 2048 : 1024;     // [keys, values][32] fp32; [keys, values][2][kRunBytes], and some more
    static constexpr int kBytes = 2 * kPart + kScaleBytes;
    static constexpr int kRequests = 2 * kPart / 1024 + (kHalf ? 0 : kFour ? kScaleBytes / 1024 : 1);
    static constexpr int kStages = 2;
    static constexpr int kPerCu = NARROW && kBytes <= 20 * 1024 ? 2 : 1;
    // (4 bits, heads of 64, 32 sequences of 8 heads: 12 wavefronts 21.5 us, 8 23.3, 16 22.6; 13 of twenty heads: 2 x 8 19.6, 2 x 4 20.5.  Heads of 128: 12 hide no more than 8,
    // 56.4 for 58.8 us at 206 000 tokens, and cost short sequences 1.4 us; 2 x 6 are slower than 2 x 4, 78 for 62.)
    static constexpr int kWaves = kFour && DP == 64 ? (NARROW ? 8 : 12) : (kBytes > 20 * 1024 ? 2 : kBytes > 9 * 1024 ? 4 : 8) / kPerCu;
    static constexpr int kRing = kWaves * kStages * kBytes;
    static constexpr int kSums = kWaves * kDecodeRows * 8;           // the wavefronts' maxima and weights
    static constexpr int kLds = kRing + kSums + 16;
    static constexpr int kBlocks = DP / 16 / kWaves > 0 ? DP / 16 / kWaves : 1;    // of 16 dimensions that a wavefront sums up in the end
    static_assert(kStages * kBytes >= kDecodeRows * DP * 4, "a wavefront's sums fit into its part of the ring");
};

__device__ __forceinline__ unsigned wave_max(unsigned x)
{
    for (int o = 1; o < kWave; o <<= 1) {
        const unsigned w = (unsigned)__shfl_xor((int)x, o);
        x = x > w ? x : w;
    }
    return (unsigned)__builtin_amdgcn_readfirstlane((int)x);
}

// A sequence's tokens lo .. len - 1; its steps start at multiples of their length.  One without tokens has a step all the same, in
// which nothing counts, and so gets its zeros.
struct Span {
    int lo, len, first, steps;
};
__device__ __forceinline__ Span span_of(const DecodeParams& p, int n)
{
    const int held = p.c.max_pages << p.c.page_shift;
    Span s;
    s.len = n < 0 ? 0 : n < held ? n : held;
    s.lo = p.window > 0 && n > p.window ? n - p.window : 0;
    if (s.lo >= s.len) s.lo = s.len = 0;                             // none at all, or a window behind the table's end
    s.first = s.lo & ~31;
    s.steps = s.len > s.lo ? (s.len - s.first + 31) / 32 : 1;
    return s;
}

// 16 bytes per lane (LANES of them), each from its own address, to LDS byte address lds + 16 lane; 4 bytes, lds + 4 lane.
__device__ __forceinline__ void request16(uint32_t lds, const unsigned char* from)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" :: "{m0}"(lds), "v"(from) : "memory");
}
// .. the lane's address as 32 bits from a common one
__device__ __forceinline__ void request16(uint32_t lds, const unsigned char* base, uint32_t from)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "{m0}"(lds), "v"(from), "s"(base) : "memory");
}
__device__ __forceinline__ void request4(uint32_t lds, const float* from)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" :: "{m0}"(lds), "v"(from) : "memory");
}

// TYPE: of the cache.  DP: head_dim rounded up to 64, 128 or 256; EXACT: it is head_dim.
// SUMS: of weights as they are, not as they are rounded, also in fp16 (there are `stats`).
template <int TYPE, int DP, bool EXACT, bool NARROW, bool SUMS>
__global__ void __launch_bounds__((DecodeStep<TYPE, DP, NARROW>::kWaves * kWave), (DecodeStep<TYPE, DP, NARROW>::kWaves * DecodeStep<TYPE, DP, NARROW>::kPerCu > 12 ? 4 : DecodeStep<TYPE, DP, NARROW>::kWaves * DecodeStep<TYPE, DP, NARROW>::kPerCu > 8 ? 3 : DecodeStep<TYPE, DP, NARROW>::kWaves * DecodeStep<TYPE, DP, NARROW>::kPerCu > 4 ? 2 : 1))
attn_decode_kernel(const DecodeParams p)
{
    typedef DecodeStep<TYPE, DP, NARROW> T;
    constexpr int NW = T::kWaves;
    extern __shared__ __align__(16) unsigned char smem[];
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char*)smem);
    const uint32_t ml_at = lds0 + T::kRing;
    volatile uint32_t* flag = reinterpret_cast<volatile uint32_t*>(smem + T::kRing + T::kSums);     // whether this workgroup is an item's last

    const CacheView& cv = p.c;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int col = lane & 15, g = lane >> 4;
    const int D = EXACT ? DP : cv.D;
    const int items = cv.Hk * p.tiles;                               // of a sequence

    // The most steps of a piece: such that there are no more pieces than workgroups, if that is little more than an even share of all steps;
    // else that share, and some workgroups have a second piece.
    int tokens = 0;                                                  // of the lane's sequence
    auto steps_at = [&](int i) {
        tokens = i < cv.seqs ? cv.lens[i] : 0;
        return i < cv.seqs ? (unsigned)span_of(p, tokens).steps : 0u;
    };
    unsigned mine = steps_at(lane), sum = mine, longest = mine;
    for (int i = kWave; i < cv.seqs; i += kWave) {
        const unsigned n = steps_at(i + lane);
        sum += n;
        longest = longest > n ? longest : n;
    }
    longest = wave_max(longest);
    const unsigned groups = gridDim.x, all_items = (unsigned)(cv.seqs * items), total = wave_sum(sum) * (unsigned)items;
    unsigned share = (total + (unsigned)p.slots - 1) / (unsigned)p.slots;
    share = share > (unsigned)NW ? share : (unsigned)NW;
    unsigned most = longest;
    if (all_items <= groups) {
        const unsigned each = groups / all_items;
        most = (longest + each - 1) / each;                          // does for any lengths
        if (cv.seqs <= kWave) {                                      // less may do for these
            unsigned from = share;
            for (int i = 0; i < 5 && from < most; ++i) {
                const unsigned mid = (from + most) / 2;
                if (wave_sum((mine + mid - 1) / mid) * (unsigned)items <= groups) most = mid;
                else from = mid + 1;
            }
        }
        most = most > (unsigned)NW ? most : (unsigned)NW;
    }
    if (most > share + kRoundSteps * NW) most = share;
    if (longest <= most + kJoinSteps * NW) most = longest;

    const_int* table = (const_int*)(uintptr_t)cv.table;
    const uint32_t codes_at = T::kFour ? code_mask() : 0u;

    // where the lane's own operands lie in a stage
    const uint32_t ring = lds0 + (uint32_t)(wave * T::kStages * T::kBytes);
    const uint32_t k_read = ring + lane * 16;
    const uint32_t v_read = T::kHalf ? k_read + T::kPart
                          : T::kFour ? ring + T::kPart + (uint32_t)((g >> 1) * DP * 8 + col * 8 + (g & 1) * 4)
                                     : ring + T::kPart + (uint32_t)((g >> 1) * 512 + col * 16 + (g & 1) * 8);
    // .. its scales; 4 bits: those of its token's keys (tile 0), and of its 8 tokens' values
    const uint32_t s_read = ring + 2 * T::kPart + (T::kFour ? (uint32_t)((col >> 3) * T::kRunBytes + (8 * ((col >> 2) & 1) + (col & 3)) * cv.runs * 4) : (uint32_t)(g * 32));
    // 4 bits: what lanes ask for, from where a step's keys, values and scales begin in its page (as request_four does for groups of 16 tokens)
    uint32_t k_from[T::kFour ? T::kPart / 1024 : 1] = {0}, v_from[T::kFour ? T::kPart / 1024 : 1] = {0};
    long long s_from = 0;
    if constexpr (T::kFour) {
        const int token = 8 * (col >> 2) + (col & 3);
#pragma unroll
        for (int i = 0; i < T::kPart / 1024; ++i) {
            const int n = DP == 64 ? g >> 1 : i / ((DP + 127) / 128), d = DP == 64 ? 32 * (g & 1) : 128 * (i % ((DP + 127) / 128)) + 32 * g;
            k_from[i] = (uint32_t)((token + 4 * n) * (D / 2) + (EXACT || d < D ? d : 0) / 2);
            const int at = i * kWave + lane, x = at / (DP / 2), dv = 2 * (at % (DP / 2));
            v_from[i] = (uint32_t)(x * 8 * D + (EXACT || dv < D ? dv : 0) * 8);
        }
        constexpr int kLanes = T::kRunBytes / 16;
        const int at = lane / kLanes & 3, word = 4 * (lane % kLanes), last = 16 * cv.runs - 4;
        s_from = 4 * ((at & 1) * 16 * cv.runs + (word < last ? word : last));
        if (T::kScaleBytes == 1024 && (at & 2)) s_from += (long long)(reinterpret_cast<uintptr_t>(cv.v_scales) - reinterpret_cast<uintptr_t>(cv.k_scales));
    }
    const uint32_t vs_read = ring + 2 * T::kPart + (uint32_t)((2 + (g >> 1)) * T::kRunBytes + (g & 1) * 16);

    for (unsigned piece = blockIdx.x;; piece += groups) {
        // Its sequence and item, and steps begin .. s_end - 1: the k-th of the item's `parts`.
        int seq = -1, item = 0, begin = 0, s_end = 0, k_part = 0, parts = 1;
        Span sp = {};
        unsigned kept = 0;                                           // pieces of cut items before this item's: their sums are kept apart
        for (unsigned i = 0, before = 0; i < (unsigned)cv.seqs; i += kWave) {
            if (cv.seqs > kWave) mine = steps_at((int)i + lane);
            const unsigned n = (mine + most - 1) / most, several = n > 1 ? n : 0;
            const unsigned past = before + wave_scan(n) * (unsigned)items, kept_past = kept + wave_scan(several) * (unsigned)items;
            const unsigned long long in = __ballot(piece < past);
            if (in) {
                const int l = __builtin_ctzll(in);
                const unsigned of_item = (unsigned)__builtin_amdgcn_readlane((int)n, l), length = (unsigned)__builtin_amdgcn_readlane((int)mine, l);
                const unsigned local = piece - ((unsigned)__builtin_amdgcn_readlane((int)past, l) - of_item * (unsigned)items), size = (length + of_item - 1) / of_item;
                seq = (int)i + l;
                sp = span_of(p, __builtin_amdgcn_readlane(tokens, l));
                item = __builtin_amdgcn_readfirstlane((int)(local / of_item));
                k_part = __builtin_amdgcn_readfirstlane((int)(local % of_item));
                parts = (int)of_item;
                begin = __builtin_amdgcn_readfirstlane(k_part * (int)size);
                s_end = __builtin_amdgcn_readfirstlane(begin + (int)size < (int)length ? begin + (int)size : (int)length);
                kept = (unsigned)__builtin_amdgcn_readlane((int)kept_past, l) - (unsigned)(items - item) * of_item;
                break;
            }
            kept = (unsigned)__builtin_amdgcn_readlane((int)kept_past, kWave - 1);
            before = (unsigned)__builtin_amdgcn_readlane((int)past, kWave - 1);
        }
        if (seq < 0) return;
        const int head = item / p.tiles, row0 = item % p.tiles * kDecodeRows;
        const int rows = p.r - row0 < kDecodeRows ? p.r - row0 : kDecodeRows;

        int page[2];
        // A step's pages: those of its two groups of 16 tokens (one page, where pages are longer), by scalar loads ahead of their use.
        // Groups past the end take the last one's place: what is loaded there does not count.
        const_int* pages = table + (size_t)seq * cv.max_pages;
        auto find = [&](int step) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                int t = sp.first + step * 32 + 16 * x;
                t = t < sp.len ? t : sp.len > 0 ? sp.len - 1 : 0;
                page[x] = pages[t >> cv.page_shift];
            }
        };
        // 4 bits.  Keys: as below, lane (col, g) reads dimensions 128 j + 32 g .. + 31; heads of up to 64: a lane both tiles' half of a token.  Values: the
        // groups of 16 tokens as they lie.  Scales and offsets: those of keys and of values, 16 tokens' at a time; lanes past the last read that again.
        auto request_four = [&](uint32_t to, const unsigned char* const (&kp)[2], const unsigned char* const (&vp)[2], const float* const (&ks)[2], const float* const (&vs)[2]) {
            const unsigned char* k = (col >= 8 ? kp[1] : kp[0]) + (8 * ((col >> 2) & 1) + (col & 3)) * (D / 2);
            if constexpr (DP == 64) {
                const int d = 32 * (g & 1);
                request16(to, k + (4 * (g >> 1) * D + (EXACT || d < D ? d : 0)) / 2);
            } else {
#pragma unroll
                for (int n = 0; n < T::kTiles; ++n)
#pragma unroll
                    for (int j = 0; j < DP / 128; ++j) {
                        const int d = 128 * j + 32 * g;
                        request16(to + (uint32_t)((n * (DP / 128) + j) * 1024), k + (4 * n * D + (EXACT || d < D ? d : 0)) / 2);
                    }
            }
#pragma unroll
            for (int i = 0; i < T::kPart / 1024; ++i) {
                const int at = i * kWave + lane, x = at / (DP / 2), d = 2 * (at % (DP / 2));
                request16(to + (uint32_t)(T::kPart + i * 1024), (x ? vp[1] : vp[0]) + (EXACT || d < D ? d : 0) * 8);
            }
            constexpr int kLanes = T::kRunBytes / 16;               // of 16 tokens' scales
#pragma unroll
            for (int i = 0; i < T::kScaleBytes / 1024; ++i) {
                const int at = (i * kWave + lane) / kLanes & 3, word = 4 * (lane % kLanes), last = 16 * cv.runs - 4;
                const float* s = at & 2 ? (at & 1 ? vs[1] : vs[0]) : (at & 1 ? ks[1] : ks[0]);
                request16(to + (uint32_t)(2 * T::kPart + i * 1024), reinterpret_cast<const unsigned char*>(s + (word < last ? word : last)));
            }
        };
        // .. where a page has a step's 32 tokens (those behind the last one lie in it too, and do not count)
        auto request_page = [&](int step, int stage) {
            const int t = sp.len > 0 ? sp.first + step * 32 : 0;
            const bool in = (unsigned)page[0] < (unsigned)cv.pages;
            const size_t token = (((size_t)(in ? page[0] : 0) * cv.Hk + head) << cv.page_shift) + (size_t)(t & ((1 << cv.page_shift) - 1));
            const size_t at = token * (size_t)(D / 2), runs_from = token * (size_t)cv.runs * 4;
            const uint32_t to = ring + (uint32_t)(stage * T::kBytes);
#pragma unroll
            for (int i = 0; i < T::kPart / 1024; ++i) request16(to + (uint32_t)(i * 1024), cv.k + at, k_from[i]);
#pragma unroll
            for (int i = 0; i < T::kPart / 1024; ++i) request16(to + (uint32_t)(T::kPart + i * 1024), cv.v + at, v_from[i]);
            if constexpr (T::kScaleBytes == 1024) {
                const unsigned char* both = reinterpret_cast<const unsigned char*>(cv.k_scales) + runs_from;
                request16(to + (uint32_t)(2 * T::kPart), both + s_from);
            } else {
                request16(to + (uint32_t)(2 * T::kPart), reinterpret_cast<const unsigned char*>(cv.k_scales) + runs_from, (uint32_t)s_from);
                request16(to + (uint32_t)(2 * T::kPart + 1024), reinterpret_cast<const unsigned char*>(cv.v_scales) + runs_from, (uint32_t)s_from);
            }
            return in ? 3 : 0;
        };
        // bit x: group x has a page
        auto request = [&](int step, int stage) {
            if constexpr (T::kFour) {
                if (cv.page_shift >= 5) return request_page(step, stage);
            }
            const unsigned char *kp[2], *vp[2];
            const float *ks[2], *vs[2];
            int ok = 0;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                int t = sp.first + step * 32 + 16 * x;
                t = t < sp.len ? t : sp.len > 0 ? (sp.len - 1) & ~15 : 0;
                const bool in = (unsigned)page[x] < (unsigned)cv.pages;
                ok |= in ? 1 << x : 0;
                const int pg = in ? page[x] : 0, slot = t & ((1 << cv.page_shift) - 1);
                if constexpr (T::kFour) {
                    const size_t at = (page_at(cv, pg, head) + (size_t)slot * D) / 2;
                    kp[x] = cv.k + at;
                    vp[x] = cv.v + at;
                    ks[x] = cv.k_scales + runs_at(cv, pg, head, slot);
                    vs[x] = cv.v_scales + runs_at(cv, pg, head, slot);
                    continue;
                }
                kp[x] = cv.k + (page_at(cv, pg, head) + (size_t)slot * D) * T::kSize;
                vp[x] = cv.v + (page_at(cv, pg, head) + (size_t)slot * D) * T::kSize;
                if constexpr (T::kScaled) {
                    ks[x] = cv.k_scales + scales_at(cv, pg, head) + (slot >> cv.block_shift);
                    vs[x] = cv.v_scales + scales_at(cv, pg, head) + (slot >> cv.block_shift);
                }
            }
            const uint32_t to = ring + (uint32_t)(stage * T::kBytes);
            if constexpr (T::kFour) {
                request_four(to, kp, vp, ks, vs);
                return ok;
            }
            // keys: lane (col, g) reads dimensions 64 j + 16 g .. + 15 of token 8 (col / 4) + 4 n + col % 4
            const unsigned char* k = (col >= 8 ? kp[1] : kp[0]) + (size_t)((8 * ((col >> 2) & 1) + (col & 3)) * D) * T::kSize;
#pragma unroll
            for (int n = 0; n < T::kTiles; ++n)
#pragma unroll
                for (int j = 0; j < DP / 64; ++j) {
                    const int d = 64 * j + 16 * g;
#pragma unroll
                    for (int h = 0; h < T::kSize; ++h)
                        request16(to + (uint32_t)(((n * (DP / 64) + j) * T::kSize + h) * 1024), k + (4 * n * D + (EXACT || d < D ? d : 0)) * T::kSize + 16 * h);
                }
            if constexpr (T::kHalf) {
                // values: lane (col, g) reads tokens 8 g .. 8 g + 7 of dimension 16 b + col
                const unsigned char* v = (g >= 2 ? vp[1] : vp[0]) + col * 32 + (g & 1) * 16;
#pragma unroll
                for (int b = 0; b < DP / 16; ++b) request16(to + (uint32_t)(T::kPart + b * 1024), v + (EXACT || 16 * b < D ? b : 0) * 512);
            } else {
                // .. lane l reads the 16 tokens of group l / 32 of dimension 32 b + l % 32
                const unsigned char* v = (lane >= 32 ? vp[1] : vp[0]);
#pragma unroll
                for (int b = 0; b < DP / 32; ++b) {
                    const int d = 32 * b + (lane & 31);
                    request16(to + (uint32_t)(T::kPart + b * 1024), v + (EXACT || d < D ? d : 0) * 16);
                }
                // scales: lane l reads that of token l % 32's key, or from 32 on value
                const float* s = lane & 16 ? (lane & 32 ? vs[1] : ks[1]) : (lane & 32 ? vs[0] : ks[0]);
                request4(to + 2 * T::kPart, s + ((lane & 15) >> cv.block_shift));
            }
            return ok;
        };

        // Q^T: column `col`, for product i the 8 dimensions that a lane has of a key; zeros beyond the head's rows and dimensions.
        half8_t qf[DP / 32];
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) {
            half8_t w = {0, 0, 0, 0, 0, 0, 0, 0};
            const int d = operand_dim<TYPE, DP>(i, g);
            if (col < rows && d < D) w = *reinterpret_cast<const half8_t*>(p.q + (size_t)seq * p.q_stride + (size_t)(head * p.r + row0 + col) * D + d);
            qf[i] = w;
        }

        float4_t o[DP / 16];
#pragma unroll
        for (int b = 0; b < DP / 16; ++b) o[b] = float4_t{0, 0, 0, 0};
        float m = -INFINITY, l = 0.0f;

        // WHOLE: all its tokens count
        auto compute_as = [&](auto is_whole, int step, int stage, int ok) {
            constexpr bool whole = decltype(is_whole)::value;
            const uint32_t off = (uint32_t)(stage * T::kBytes);
            float4_t s[T::kTiles];
#pragma unroll
            for (int n = 0; n < T::kTiles; ++n) {
                s[n] = float4_t{0, 0, 0, 0};
                if constexpr (T::kFour) {
#pragma unroll
                    for (int j = 0; j < (DP + 127) / 128; ++j) {
                        constexpr int kEach = DP < 128 ? DP / 32 : 4;       // words of a lane
                        const int d = DP < 128 ? 16 * g : 128 * j + 32 * g;
                        const bool in = EXACT || d < D;
                        const uint32_t so = *(const lds_word*)(uintptr_t)(s_read + off + (uint32_t)(4 * n * cv.runs * 4 + ((in ? d : 0) >> cv.run_shift) * 4));
                        const half2_t scale = both_low(so), offset = both_high(so);
                        uint32_t w[kEach];
                        if constexpr (DP < 128) {
                            const u32x2_t x = *(const lds_words2*)(uintptr_t)(ring + off + (uint32_t)(((2 * n + (g >> 1)) * 16 + col) * 16 + (g & 1) * 8));
                            w[0] = x[0]; w[1] = x[1];
                        } else {
                            const u32x4_t x = *(const lds_words4*)(uintptr_t)(k_read + off + (uint32_t)((n * (DP / 128) + j) * 1024));
#pragma unroll
                            for (int a = 0; a < kEach; ++a) w[a] = x[a];
                        }
#pragma unroll
                        for (int a = 0; a < kEach; ++a) {
                            half8_t kf = four_bits(w[a], scale, offset, codes_at);
                            if (!EXACT && !in) kf = half8_t{0, 0, 0, 0, 0, 0, 0, 0};
                            s[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[kEach * j + a], s[n], 0, 0, 0);
                        }
                    }
                    continue;
                }
#pragma unroll
                for (int j = 0; j < DP / 64; ++j) {
                    const bool in = EXACT || 64 * j + 16 * g < D;
                    half8_t kf[2];
                    if constexpr (T::kHalf) {
#pragma unroll
                        for (int a = 0; a < 2; ++a) {
                            u32x4_t w = *(const lds_words4*)(uintptr_t)(k_read + off + (uint32_t)(((n * (DP / 64) + j) * 2 + a) * 1024));
                            if (!EXACT && !in) w = u32x4_t{0, 0, 0, 0};
                            kf[a] = __builtin_bit_cast(half8_t, w);
                        }
                    } else {
                        u32x4_t w = *(const lds_words4*)(uintptr_t)(k_read + off + (uint32_t)((n * (DP / 64) + j) * 1024));
                        if (!EXACT && !in) w = u32x4_t{0, 0, 0, 0};
                        kf[0] = codes_to_half<TYPE>(w[0], w[1]);
                        kf[1] = codes_to_half<TYPE>(w[2], w[3]);
                    }
                    s[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[0], qf[2 * j], s[n], 0, 0, 0);
                    s[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[1], qf[2 * j + 1], s[n], 0, 0, 0);
                }
            }
            const int t0 = sp.first + step * 32, t = t0 + 8 * g;
            // of the run's tokens, those that count
            const int vlo = sp.lo > t ? sp.lo - t : 0, vhi = !(ok >> (g >> 1) & 1) || t >= sp.len ? 0 : sp.len - t;
            float4_t vs[T::kTiles];
#pragma unroll
            for (int n = 0; n < T::kTiles; ++n) {
                if constexpr (!T::kScaled) s[n] *= p.scale;
                else {
                    s[n] *= *(const lds_float4*)(uintptr_t)(s_read + off + (uint32_t)(16 * n)) * p.scale;
                    vs[n] = *(const lds_float4*)(uintptr_t)(s_read + off + (uint32_t)(128 + 16 * n));
                }
            }
            if (!whole) {
#pragma unroll
                for (int n = 0; n < T::kTiles; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const bool seen = 4 * n + r >= vlo && 4 * n + r < vhi;
                        s[n][r] = seen ? s[n][r] : -INFINITY;
                        if constexpr (T::kScaled) vs[n][r] = seen ? vs[n][r] : 0.0f;
                    }
            }
            // The maximum is taken over score + log2 of the value's scale, so that weight times scale, rounded to fp16, is at most 2^kLift.
            float most = -INFINITY;
            if (!T::kScaled || (whole && cv.block_shift >= 3)) {           // one scale for the run
#pragma unroll
                for (int n = 0; n < T::kTiles; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) most = fmaxf(most, s[n][r]);
                if constexpr (T::kScaled) most += fmaxf(__builtin_amdgcn_logf(vs[0][0]), kLeastLog);
            } else if constexpr (T::kScaled) {
#pragma unroll
                for (int n = 0; n < T::kTiles; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) most = fmaxf(most, s[n][r] + fmaxf(__builtin_amdgcn_logf(vs[n][r]), kLeastLog));
            }
            most = over_groups(most, [](float a, float b) { return fmaxf(a, b); });
            float m_new;
            if constexpr (T::kFour) {
                // (Followed where a weight would pass 2^(kLowLift + kReach) only, so that sums are seldom rescaled: they are, in nearly every step, for one of the
                // heads or another, where every new maximum is followed.)
                const bool fine = fabsf(most) < kFine;
                const float from = most - (fine ? kLowLift : 0.0f);
                m_new = from > m + (fine ? kReach : 0.0f) ? from : m;
            } else {
                most -= fabsf(most) < kFine ? kLift : 0.0f;
                m_new = fmaxf(m, most);
            }
            const float base = m_new == -INFINITY ? 0.0f : m_new;
            const float keep = __builtin_amdgcn_exp2f(m - base);
            m = m_new;
            float add = 0.0f;
            half8_t pf;
#pragma unroll
            for (int n = 0; n < T::kTiles; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float w = __builtin_amdgcn_exp2f(s[n][r] - base);
                    pf[4 * n + r] = (_Float16)(T::kScaled ? w * vs[n][r] : w);
                    if constexpr (!T::kHalf || SUMS) add += w;           // (unrounded, as products have scales: off by 2^-11 at most)
                }
            if constexpr (T::kHalf && !SUMS) {                                    // the sum of the weights as they are rounded
#pragma unroll
                for (int i = 0; i < 8; i += 2) add = __builtin_amdgcn_fdot2(half2_t{pf[i], pf[i + 1]}, half2_t{(_Float16)1.0f, (_Float16)1.0f}, add, false);
            }
            l = l * keep + add;
            // values that do not count are zeros: what lies there may be a NaN
            u32x4_t mask = {~0u, ~0u, ~0u, ~0u};
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (!(i >= vlo && i < vhi)) {
                        if constexpr (!T::kScaled) mask[i / 2] &= i & 1 ? 0x0000ffffu : 0xffff0000u;
                        else mask[i / 4] &= ~(0xffu << (8 * (i & 3)));
                    }
            }
            if (!__all(keep == 1.0f)) {
#pragma unroll
                for (int b = 0; b < DP / 16; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[b][r] *= keep;
            }
            u32x4_t scale4, offset4;                                     // 4 bits: of the 8 tokens and 32 dimensions; without either, a code is zero
#pragma unroll
            for (int b = 0; b < DP / 16; ++b) {
                half8_t vf;
                if constexpr (T::kFour) {
                    if (b % 2 == 0) {
                        const uint32_t at = vs_read + off + (uint32_t)(((EXACT || 16 * b < D ? 16 * b : 0) >> cv.run_shift) * 64);
                        scale4 = *(const lds_words4*)(uintptr_t)at;
                        offset4 = *(const lds_words4*)(uintptr_t)(at + 32);
                        if (!whole) { scale4 &= mask; offset4 &= mask; }
                    }
                    vf = four_bits(*(const lds_word*)(uintptr_t)(v_read + off + (uint32_t)(b * 128)), scale4, offset4, codes_at);
                } else if constexpr (T::kHalf) {
                    u32x4_t w = *(const lds_words4*)(uintptr_t)(v_read + off + (uint32_t)(b * 1024));
                    if (!whole) w &= mask;
                    vf = __builtin_bit_cast(half8_t, w);
                } else {
                    u32x2_t w = *(const lds_words2*)(uintptr_t)(v_read + off + (uint32_t)((b >> 1) * 1024 + (b & 1) * 256));
                    if (!whole) w &= u32x2_t{mask[0], mask[1]};
                    vf = codes_to_half<TYPE>(w[0], w[1]);
                }
                o[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf, o[b], 0, 0, 0);
            }
        };

        auto compute = [&](int step, int stage, int ok) {
            const int t0 = sp.first + step * 32;
            if (t0 >= sp.lo && t0 + 32 <= sp.len && ok == 3) compute_as(std::true_type(), step, stage, ok);
            else compute_as(std::false_type(), step, stage, ok);
        };

        // The wavefront's steps: two stages, each asked for again as soon as it has been read.
        {
            int s = begin + wave, stage = 0, ok = 0, next = 0;
            if (s < s_end) {
                find(s);
                ok = request(s, 0);
            }
            if (s + NW < s_end) {
                find(s + NW);
                next = request(s + NW, 1);
            }
            if (s + 2 * NW < s_end) find(s + 2 * NW);
            // The queries are here before the loop: in it, the compiler's wait for them would be one for every request.
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) asm volatile("" : "+v"(qf[i]));
            for (; s < s_end; s += NW) {
                if (s + NW < s_end) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(T::kRequests) : "memory");
                else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                compute(s, stage, ok);
                ok = next;
                if (s + 2 * NW < s_end) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the stage has been read
                    next = request(s + 2 * NW, stage);
                    if (s + 3 * NW < s_end) find(s + 3 * NW);
                }
                stage ^= 1;
            }
        }
        l = over_groups(l, [](float a, float b) { return a + b; });

        // Every wavefront leaves its sums in its own part of the ring (its first stage; 4 bits: the beginning of its second too), whose last step has been read, then takes
        // some blocks of 16 dimensions and adds up all wavefronts' sums of them, each lane those of its own place.
#pragma unroll
        for (int b = 0; b < DP / 16; ++b) *(lds_float4*)(uintptr_t)(ring + (uint32_t)(b * 1024 + lane * 16)) = o[b];
        if (g == 0) {
            *(lds_float1*)(uintptr_t)(ml_at + (uint32_t)((wave * kDecodeRows + col) * 8)) = m;
            *(lds_float1*)(uintptr_t)(ml_at + (uint32_t)((wave * kDecodeRows + col) * 8 + 4)) = l;
        }
        __syncthreads();
        float top = -INFINITY, weight = 0.0f, by[NW];
        {
            float ls[NW];
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                by[w] = *(const lds_float1*)(uintptr_t)(ml_at + (uint32_t)((w * kDecodeRows + col) * 8));
                ls[w] = *(const lds_float1*)(uintptr_t)(ml_at + (uint32_t)((w * kDecodeRows + col) * 8 + 4));
                top = fmaxf(top, by[w]);
            }
            const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                by[w] = __builtin_amdgcn_exp2f(by[w] - base);
                weight += by[w] * ls[w];
            }
        }
        float4_t mine_o[T::kBlocks];
#pragma unroll
        for (int i = 0; i < T::kBlocks; ++i) {
            const int b = wave * T::kBlocks + i;
            mine_o[i] = float4_t{0, 0, 0, 0};
            if (16 * b >= DP) continue;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float4_t x = *(const lds_float4*)(uintptr_t)(lds0 + (uint32_t)(w * T::kStages * T::kBytes + b * 1024 + lane * 16));
#pragma unroll
                for (int r = 0; r < 4; ++r) mine_o[i][r] = __builtin_fmaf(by[w], x[r], mine_o[i][r]);
            }
        }
        auto store = [&](int b, const float4_t& x, float inv) {
            _Float16* out = p.out + (size_t)seq * p.out_stride + (size_t)(head * p.r + row0 + col) * D + 16 * b + 4 * g;
            if (col < rows && 16 * b < D) *reinterpret_cast<half4_t*>(out) = half4_t{(_Float16)(x[0] * inv), (_Float16)(x[1] * inv), (_Float16)(x[2] * inv), (_Float16)(x[3] * inv)};
        };
        auto tell = [&](float upto, float all, float inv) {
            if (p.stats && wave == 0 && g == 0 && col < rows) p.stats[(size_t)seq * cv.Hk * p.r + head * p.r + row0 + col] = Pair{all == 0.0f ? 0.0f : upto, inv};
        };
        if (parts == 1) {
            const float inv = weight == 0.0f ? 0.0f : 1.0f / weight;
            tell(top, weight, inv);
#pragma unroll
            for (int i = 0; i < T::kBlocks; ++i) store(wave * T::kBlocks + i, mine_o[i], inv);
        } else {
            // Stores acknowledged before the ticket is taken; the last workgroup of the item adds the pieces in order and leaves the counter at zero.
            const int each = kDecodeRows * (D + 2) * 4, own = k_part * each, ml_of = kDecodeRows * D * 4 + col * 8;
            const __amdgpu_buffer_rsrc_t sums = parts_of(p.part + (size_t)kept * kDecodeRows * (D + 2));        // the item's pieces
            if (col < rows) {
#pragma unroll
                for (int i = 0; i < T::kBlocks; ++i) {
                    const int b = wave * T::kBlocks + i;
                    if (16 * b >= D) continue;
                    put16(sums, own + (b * kWave + lane) * 16, mine_o[i]);
                }
                if (wave == 0 && g == 0) put8(sums, own + ml_of, top, weight);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tid == 0) {
                uint32_t* ctr = p.counters + (size_t)kept * kCounterAreaWords / (4 * kDecodeUnits);
                const bool last = __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(parts - 1);
                if (last) __hip_atomic_store(ctr, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                *flag = last ? 1u : 0u;
            }
            __syncthreads();
            if (*flag != 0u && col < rows) {
                for (int b = wave; 16 * b < D; b += NW) {
                    float4_t x = {0, 0, 0, 0};
                    float upto = -INFINITY, all = 0.0f;
                    for (int k0 = 0; k0 < parts; k0 += kJoined) {
                        float4_t w[kJoined];
                        Pair ml[kJoined];
#pragma unroll
                        for (int k = 0; k < kJoined; ++k) {
                            const int from = (k0 + k < parts ? k0 + k : k0) * each;         // (one that is there, with weight 0)
                            ml[k] = get8(sums, from + ml_of);
                            w[k] = get16(sums, from + (b * kWave + lane) * 16);
                        }
                        float m_new = upto;
#pragma unroll
                        for (int k = 0; k < kJoined; ++k) m_new = fmaxf(m_new, ml[k].a);
                        const float base = m_new == -INFINITY ? 0.0f : m_new, keep = __builtin_amdgcn_exp2f(upto - base);
                        upto = m_new;
                        all *= keep;
                        x *= keep;
#pragma unroll
                        for (int k = 0; k < kJoined; ++k) {
                            const float f = k0 + k < parts ? __builtin_amdgcn_exp2f(ml[k].a - base) : 0.0f;
                            all += f * ml[k].b;
                            x += f * w[k];
                        }
                    }
                    const float inv = all == 0.0f ? 0.0f : 1.0f / all;
                    if (b == wave) tell(upto, all, inv);
                    store(b, x, inv);
                }
            }
        }
        __syncthreads();                                              // the sums' places and the flag are free again
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
    int r, tiles, groups;
    bool narrow;
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
    // A workgroup counts all steps there are in 32 bits.
    if ((long long)cache->num_seqs * (((long long)cache->max_pages * cache->page_size + 31) / 32) * d->kv_heads * p->tiles >= 1ll << 31) return CODEGEMM_UNSUPPORTED;
    // Up to as many items as there are compute units, a unit works on one: a workgroup each, or for all the pieces of 4 steps that there may be as
    // far as the host knows (any number is right).  More items: two at a time.
    const long long items = (long long)d->num_seqs * d->kv_heads * p->tiles;
    const int held = cache->max_pages * cache->page_size, longest = d->max_kv < held ? d->max_kv : held;
    const int keys = d->window > 0 && d->window < longest ? d->window : longest;
    const long long pieces = (ceil_div(keys, 32) + 1ll) / 4 * items + items;
    p->narrow = items > kDecodeUnits;
    const int slots = p->narrow ? 2 * kDecodeUnits : kDecodeUnits;
    p->groups = (int)(items > kMostGroups ? kMostGroups : items > slots ? items : pieces < slots ? pieces : slots);
    // A cut item of x shares has at most 2 x pieces, and there are as many shares as workgroups that run at once.
    p->bytes = (size_t)kCounterAreaWords * sizeof(uint32_t) + kPairAreaBytes + 2 * (size_t)(p->groups < slots ? p->groups : slots) * kDecodeRows * (d->head_dim + 2) * sizeof(float);
    return CODEGEMM_OK;
}

template <int TYPE, int DP, bool EXACT, bool NARROW, bool SUMS>
int launch_decode_as(DecodeParams& p, int groups, hipStream_t s)
{
    typedef DecodeStep<TYPE, DP, NARROW> T;
    static_assert(T::kLds * T::kPerCu <= kMaxLds, "LDS");
    auto fn = attn_decode_kernel<TYPE, DP, EXACT, NARROW, SUMS>;
    const int st = set_max_lds(reinterpret_cast<const void*>(fn), T::kLds);
    if (st) return st;
    p.slots = groups < kDecodeUnits * T::kPerCu ? groups : kDecodeUnits * T::kPerCu;
    hipLaunchKernelGGL(fn, dim3((unsigned)groups), dim3(T::kWaves * kWave), T::kLds, s, p);
    return hipGetLastError() == hipSuccess ? CODEGEMM_OK : CODEGEMM_LAUNCH_FAILED;
}

template <int TYPE, int DP, bool EXACT, bool NARROW>
int launch_decode_one(DecodeParams& p, int groups, hipStream_t s)
{
    if constexpr (TYPE == CODEGEMM_KV_FP16) {
        if (p.stats) return launch_decode_as<TYPE, DP, EXACT, NARROW, true>(p, groups, s);
    }
    return launch_decode_as<TYPE, DP, EXACT, NARROW, false>(p, groups, s);
}

template <int TYPE, int DP>
int launch_decode(DecodeParams& p, bool narrow, int groups, hipStream_t s)
{
    if constexpr (DecodeStep<TYPE, DP, true>::kPerCu == 2) {
        if (narrow) return p.c.D == DP ? launch_decode_one<TYPE, DP, true, true>(p, groups, s) : launch_decode_one<TYPE, DP, false, true>(p, groups, s);
    }
    return p.c.D == DP ? launch_decode_one<TYPE, DP, true, false>(p, groups, s) : launch_decode_one<TYPE, DP, false, false>(p, groups, s);
}

template <int TYPE>
int launch_decode_of(DecodeParams& p, bool narrow, int groups, hipStream_t s)
{
    if (p.c.D <= 64) return launch_decode<TYPE, 64>(p, narrow, groups, s);
    if (p.c.D <= 128) return launch_decode<TYPE, 128>(p, narrow, groups, s);
    return launch_decode<TYPE, 256>(p, narrow, groups, s);
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" size_t codegemm_attn_decode_workspace_bytes(const codegemm_kv_cache* cache, const codegemm_attn_desc* desc)
{
    DecodePlan plan;
    return decode_plan(cache, desc, &plan) ? 0 : plan.bytes;
}

namespace cg {

// stats: as the kernel leaves them, or NULL.
int attn_decode(const codegemm_kv_cache* cache, const codegemm_attn_desc* desc, const void* q, void* out, Pair* stats, void* workspace, size_t workspace_bytes, void* stream)
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
    p.stats = stats;
    p.r = plan.r;
    p.tiles = plan.tiles;
    p.q_stride = row_stride(desc->q_stride, desc->q_heads * desc->head_dim);
    p.out_stride = row_stride(desc->out_stride, desc->q_heads * desc->head_dim);
    p.window = desc->window;
    p.scale = log2_scale(desc->scale);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (cache->dtype == CODEGEMM_KV_FP16) return launch_decode_of<CODEGEMM_KV_FP16>(p, plan.narrow, plan.groups, s);
    if (cache->dtype == CODEGEMM_KV_INT8) return launch_decode_of<CODEGEMM_KV_INT8>(p, plan.narrow, plan.groups, s);
    if (cache->dtype == CODEGEMM_KV_INT4) return launch_decode_of<CODEGEMM_KV_INT4>(p, plan.narrow, plan.groups, s);
    return launch_decode_of<CODEGEMM_KV_FP8>(p, plan.narrow, plan.groups, s);
}

}  // namespace cg

extern "C" int codegemm_attn_decode(const codegemm_kv_cache* cache, const codegemm_attn_desc* desc, const void* q, void* out, void* workspace,
                                    size_t workspace_bytes, void* stream)
{
    return attn_decode(cache, desc, q, out, nullptr, workspace, workspace_bytes, stream);
}
