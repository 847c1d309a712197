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

int check_cache(const codegemm_kv_cache* c, bool pointers);     // status
int check_attn(const codegemm_attn_desc* d);                     // status
CacheView cache_view(const codegemm_kv_cache& c);

inline bool misaligned_ints(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
// A launch has fewer than 2^32 threads.
inline bool too_many(long long blocks, int threads) { return blocks * threads > 0xffffffffll; }
// A row stride of 0 stands for dense rows of `dense` elements.
inline int row_stride(int stride, int dense) { return stride ? stride : dense; }
inline bool bad_stride(int stride, int dense) { return stride != 0 && (stride < dense || stride > kMaxStride || (stride & 7) != 0); }

}  // namespace cg
