// The paged cache of 8-bit values: what its two kernels (cache_append_kernels.hip, cache_attention_kernels.hip) share.
#pragma once
#include "common.h"

namespace astra {

constexpr int kCacheMaxSeqs = 1024;
constexpr float kE4m3Max = 448.f;
constexpr int64_t kMaxGridThreads = 0xffffffff;      // of a launch, as the runtime takes it

// The arrays and sizes of a step.  What they say is checked where it is used: no entry of the table, no length and no row number
// takes an access out of its array.
struct CacheStep {
    const int32_t* table;
    const int32_t* lens;
    const int32_t* first;
    int32_t n_seqs, n_tokens, max_pages, table_stride, n_pages;
    int32_t page_shift;          // page_size = 1 << page_shift
    int32_t Hq, Hkv;

    __device__ __forceinline__ int32_t capacity() const { return max_pages << page_shift; }
};

// first row of sequence s, inside the rows that there are
__device__ __forceinline__ int32_t cache_row(const CacheStep& c, int s) { return min(max(c.first[s], 0), c.n_tokens); }
__device__ __forceinline__ int32_t cache_len(const CacheStep& c, int s) { return min(max(c.lens[s], 0), c.capacity()); }

int check_cache_desc(const astra_cache_desc* d);
CacheStep cache_step(const astra_cache_desc& d, const int32_t* table, const int32_t* lens, const int32_t* first);

}  // namespace astra
