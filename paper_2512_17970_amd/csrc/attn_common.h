// What the kernels around the paged cache share: its layout on the device, host checks, and the search for the sequence of a row.
#pragma once

#include <type_traits>

#include "cg_common.h"

namespace cg {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));

constexpr int kMaxHeads = 1024;
constexpr int kMaxHeadDim = 256;
constexpr int kMaxSeqs = 65535;
constexpr int kMaxTokens = 1 << 24;
constexpr int kMaxStride = 1 << 20;    // elements between tokens: 64 of them stay in a buffer's 32-bit offsets
constexpr int kTokenGroup = 16;        // tokens that lie innermost in the value pool

// A codegemm_kv_cache as the kernels take it.
struct CacheView {
    unsigned char *k, *v;
    float *k_scales, *v_scales;
    const int32_t *table, *lens;
    int Hk, D, pages, max_pages, seqs;
    int page_shift;      // log2 of the page size
    int block_shift;     // log2 of the tokens that share a scale
    int run_shift;       // 4 bits: log2 of the dimensions that share a token's scale and offset,
    int runs;            // .. and how many such runs a head has
};

// Page of a position's page index, or -1.
__device__ __forceinline__ int page_of(const CacheView& c, int seq, int index)
{
    if ((unsigned)index >= (unsigned)c.max_pages) return -1;
    const int page = c.table[(size_t)seq * c.max_pages + index];
    return (unsigned)page < (unsigned)c.pages ? page : -1;
}

// First element of a page's head, in elements; 64 bits.
__device__ __forceinline__ size_t page_at(const CacheView& c, int page, int head) { return (((size_t)page * c.Hk + head) << c.page_shift) * (size_t)c.D; }
// .. and its first scale.
__device__ __forceinline__ size_t scales_at(const CacheView& c, int page, int head) { return ((size_t)page * c.Hk + head) << (c.page_shift - c.block_shift); }

// The last i in 0..n-1 with first(i) <= x, or 0; first() ascends.  By a whole wavefront, 64 probes at a time, so that up to 64
// sequences take one load and 4096 take two.
template <class First>
__device__ __forceinline__ int last_at_most(int n, int x, First first)
{
    const int lane = threadIdx.x & (kWave - 1);
    int base = 0;
    while (n > 1) {
        const int step = (n + kWave - 1) / kWave;
        const int i = lane * step;
        const int below = __popcll(__ballot(i < n && first(base + i) <= x));
        const int at = below > 0 ? (below - 1) * step : 0;
        base += at;
        n = n - at < step ? n - at : step;
    }
    return __builtin_amdgcn_readfirstlane(base);
}

// The sum of the values up to the lane's own; all lanes' in the last lane.
__device__ __forceinline__ unsigned wave_scan(unsigned x)
{
    auto add = [&](auto ctrl, auto rows) { x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(rows)::value, 0xf, false); };
    typedef std::integral_constant<int, 0xf> all;
    add(std::integral_constant<int, 0x111>(), all());      // row_shr 1, 2, 4, 8
    add(std::integral_constant<int, 0x112>(), all());
    add(std::integral_constant<int, 0x114>(), all());
    add(std::integral_constant<int, 0x118>(), all());
    add(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());     // row_bcast 15 into rows 1 and 3
    add(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());     // row_bcast 31 into rows 2 and 3
    return x;
}
__device__ __forceinline__ unsigned wave_sum(unsigned x) { return (unsigned)__builtin_amdgcn_readlane((int)wave_scan(x), kWave - 1); }

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

// Sum, maximum over the four lanes of a column: lanes l, l ^ 16, l ^ 32, l ^ 48.
template <class Join>
__device__ __forceinline__ float over_groups(float x, Join join)
{
    const uint32_t w = __builtin_bit_cast(uint32_t, x);
    const auto a = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    const uint32_t y = __builtin_bit_cast(uint32_t, join(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1])));
    const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    return join(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}

// What workgroups hand to each other: device-scope accesses of 16 (8) bytes, `at` bytes from the base of `parts`.  (By 8-byte atomics, single tokens
// after 8000, 32 pieces, took 18.0 us, so 15.0.)
constexpr int kDeviceScope = 16;            // the cache policy bit that device-scope atomics have (sc1)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t parts_of(float* base) { return __builtin_amdgcn_make_buffer_rsrc(base, 0, 0x7fffffff, 0x00020000); }
__device__ __forceinline__ void put16(__amdgpu_buffer_rsrc_t parts, int at, const float4_t& x)
{
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, x), parts, at, 0, kDeviceScope);
}
__device__ __forceinline__ float4_t get16(__amdgpu_buffer_rsrc_t parts, int at)
{
    return __builtin_bit_cast(float4_t, __builtin_amdgcn_raw_buffer_load_b128(parts, at, 0, kDeviceScope));
}
__device__ __forceinline__ void put8(__amdgpu_buffer_rsrc_t parts, int at, float a, float b)
{
    const u32x2_t w = {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
    __builtin_amdgcn_raw_buffer_store_b64(w, parts, at, 0, kDeviceScope);
}
struct Pair {
    float a, b;
};
__device__ __forceinline__ Pair get8(__amdgpu_buffer_rsrc_t parts, int at)
{
    const u32x2_t w = __builtin_amdgcn_raw_buffer_load_b64(parts, at, 0, kDeviceScope);
    const uint32_t a = w[0], b = w[1];
    return Pair{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}

// 4 bits: eight codes of a word, code j in bits 4 (j / 2) + 16 (j % 2), so that shifts by whole words and one mask leave consecutive codes in the two
// halves, at the place of the four leading mantissa bits: with the exponent of 16 that is 16 + code in fp16, and one packed multiply-add makes the values.
// (The mask in a vector register: an instruction takes one constant, and mask and exponent are one instruction then.)
__device__ __forceinline__ uint32_t code_mask()
{
    uint32_t m = 0x03c003c0u;
    asm("" : "+v"(m));
    return m;
}
__device__ __forceinline__ half2_t code_pair(uint32_t w, int i, uint32_t mask)
{
    const uint32_t at = i == 0 ? w << 6 : i == 1 ? w << 2 : i == 2 ? w >> 2 : w >> 6;
    return __builtin_bit_cast(half2_t, (at & mask) | 0x4c004c00u);
}
__device__ __forceinline__ half2_t halves_of(uint32_t w) { return __builtin_bit_cast(half2_t, w); }
__device__ __forceinline__ half2_t both_low(uint32_t w) { return halves_of(__builtin_amdgcn_perm(w, w, 0x01000100u)); }
__device__ __forceinline__ half2_t both_high(uint32_t w) { return halves_of(__builtin_amdgcn_perm(w, w, 0x03020302u)); }
// .. of one scale and offset (a key's run of dimensions)
__device__ __forceinline__ half8_t four_bits(uint32_t w, half2_t scale, half2_t offset, uint32_t mask)
{
    half8_t x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const half2_t y = __builtin_elementwise_fma(code_pair(w, i, mask), scale, offset);
        x[2 * i] = y[0];
        x[2 * i + 1] = y[1];
    }
    return x;
}
// .. of eight (values of eight tokens)
__device__ __forceinline__ half8_t four_bits(uint32_t w, const u32x4_t& scale, const u32x4_t& offset, uint32_t mask)
{
    half8_t x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const half2_t y = __builtin_elementwise_fma(code_pair(w, i, mask), halves_of(scale[i]), halves_of(offset[i]));
        x[2 * i] = y[0];
        x[2 * i + 1] = y[1];
    }
    return x;
}
// The 8 dimensions that lane group g (of 16 lanes) has of a key in the i-th product of 32 dimensions, as one or two loads of 16 bytes leave them; heads are
// worked on as DP dimensions.
template <int TYPE, int DP>
__device__ __forceinline__ constexpr int operand_dim(int i, int g)
{
    return TYPE != CODEGEMM_KV_INT4 || DP < 128 ? 64 * (i / 2) + 16 * g + 8 * (i % 2) : 128 * (i / 4) + 32 * g + 8 * (i % 4);
}
// First scale-and-offset word of a token's keys (of 16 tokens' values) at slot `slot`, a multiple of 16 for values: as many for both.
__device__ __forceinline__ size_t runs_at(const CacheView& c, int page, int head, int slot) { return ((((size_t)page * c.Hk + head) << c.page_shift) + slot) * (size_t)c.runs; }

int attn_decode(const codegemm_kv_cache* cache, const codegemm_attn_desc* desc, const void* q, void* out, Pair* stats, void* workspace, size_t workspace_bytes, void* stream);
int set_max_lds(const void* fn, size_t bytes);                    // status; gemm.hip
int check_cache(const codegemm_kv_cache* c, bool pointers);     // status
int check_attn(const codegemm_attn_desc* d);                     // status
CacheView cache_view(const codegemm_kv_cache& c);

inline bool misaligned_ints(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
// The scale of scores times log2(e).  From 1e25 on all are the same, as any difference of scores of fp16 times that leaves the smaller no weight; and no score
// times that is infinite.
inline float log2_scale(float scale)
{
    const double s = scale > 1e25f ? 1e25 : scale < -1e25f ? -1e25 : (double)scale;
    return (float)(s * 1.4426950408889634);
}
// A launch has fewer than 2^32 threads in a dimension.
inline bool too_many(long long blocks, int threads) { return blocks * threads > 0xffffffffll; }
// A row stride of 0 stands for dense rows of `dense` elements.
inline int row_stride(int stride, int dense) { return stride ? stride : dense; }
inline bool bad_stride(int stride, int dense) { return stride != 0 && (stride < dense || stride > kMaxStride || (stride & 7) != 0); }

}  // namespace cg
