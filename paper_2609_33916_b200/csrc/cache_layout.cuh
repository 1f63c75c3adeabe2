// Where the elements of a cache page are (include/moa_cache.h states the same in words).
#pragma once
#include "common.cuh"
#include "rotate.cuh"

namespace moa {

constexpr int kBlockKeys = 16;       // keys of a block of a 4-bit page

struct CachePool {
    int pages, page, Hkv, d, int4;
    long long page_stride;           // bytes
    long long page_bytes() const { return (long long)Hkv * page * (int4 ? d + d / 8 : 4 * d); }
};

// A 4-bit block of 16 keys: byte offsets of its parts
template <int D>
struct Block4 {
    static constexpr int kGroups = D / 32, kWords = D / 64;             // scale groups of a head; 32-bit words of V codes per key and lane
    static constexpr int offKS = 8 * D, offV = 9 * D, offVS = 17 * D, kBytes = 18 * D;
    __host__ __device__ static constexpr int k_word(int r, int t, int y) { return r * (D / 2) + 4 * (t * kGroups + y); }
    __host__ __device__ static constexpr int k_scale(int r, int y) { return offKS + 2 * ((2 * (r % 8) + r / 8) * kGroups + y); }
    // the word of elements 4 g .. 4 g + 3 of groups 2 h and 2 h + 1
    __host__ __device__ static constexpr int v_word(int r, int g, int h)
    {
        return offV + 128 * kGroups * (r / 8) + 4 * kGroups * (4 * g + r % 8 / 2) + 2 * kGroups * (r % 2) + 4 * h;
    }
    __host__ __device__ static constexpr int v_scale(int r, int y) { return offVS + 8 * kGroups * (r % 8 / 2) + 8 * y + 4 * (r / 8) + 2 * (r % 2); }
};

// Byte offset, from its page's start, of a bf16 row (v: 0 K, 1 V) and of a 4-bit block
__host__ __device__ __forceinline__ long long row16(int page, int d, int h, int v, int key) { return (((long long)h * 2 + v) * page + key) * (2LL * d); }
template <int D>
__host__ __device__ __forceinline__ long long block4(int page, int h, int blk) { return ((long long)h * (page / kBlockKeys) + blk) * Block4<D>::kBytes; }

// cache.cu
struct AppendProblem {
    CachePool pool;
    int T, H, d_rot, pairs;
    float factor;
    RopeStride sq, sk, sv, so;
};
cudaError_t kv_append(const AppendProblem &p, const void *q, const void *k, const void *v, const int *pos, const long long *slot,
                      const float *inv_freq, void *qo, void *pool, cudaStream_t st);
cudaError_t kv_gather(const CachePool &pool, int T, int dtype, const void *base, const long long *slot, void *k, void *v, RopeStride sk, RopeStride sv,
                      cudaStream_t st);

// paged_decode.cu
struct PagedProblem {
    CachePool pool;
    int B, H, max_pages;
    float scale;
    long long table_stride;
    RopeStride sq;
};
size_t paged_decode_workspace_bytes(const PagedProblem &p);
cudaError_t paged_decode(const PagedProblem &p, const void *q, const void *pool, const int *table, const int *lens, void *out, float *lse,
                         void *ws, cudaStream_t st);

}  // namespace moa
