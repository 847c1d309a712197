// What the kernels around the paged cache share: its layout on the device, host checks, and the search for the sequence of a row.
#pragma once

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
