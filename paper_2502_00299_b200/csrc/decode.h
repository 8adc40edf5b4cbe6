// Host-side declarations of the kernels that work on the decode cache (rotate.cu, attend.cu, evict.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace chunkkv {

// A paged cache [num_pages, page_size, Hkv, d] and the block tables of the sequences in it.
struct PagedCache {
    const int32_t* tables;      // [B, max_pages]
    int max_pages, page_size, num_pages;
    int cap;                    // max_pages * page_size: rows that a sequence can have
    uint32_t magic;             // row / page_size = (mulhi(magic, row) + row) >> shift for rows below 2^31
    int shift;
};
inline PagedCache paged_cache(const int32_t* tables, int max_pages, int page_size, int num_pages) {
    int shift = 0;
    while ((1LL << shift) < page_size) ++shift;
    const uint64_t over = (1ULL << shift) - static_cast<uint64_t>(page_size);
    return {tables, max_pages, page_size, num_pages, max_pages * page_size, static_cast<uint32_t>((over << 32) / page_size + 1), shift};
}

// Queries and keys normalised and rotated (rotate.cu): into out_q / out_k (token and head strides in elements), or, with a cache, keys and values
// into it.
struct RotateArgs {
    const __nv_bfloat16* qkv;
    long long row_elems;
    int T, Hq, Hkv;
    const __nv_bfloat16 *gain_q, *gain_k;     // [d]; NULL: no norm
    float eps;
    const float *cos_t, *sin_t;               // [n_pos, d / 2]
    int n_pos;
    const int32_t* positions;                 // [T]
    __nv_bfloat16 *out_q, *out_k;
    long long q_token, q_head, k_token, k_head;
    __nv_bfloat16 *cache_K, *cache_V;
    const int32_t* lengths;                   // [T, Hkv], the token's row included
    PagedCache cache;
    int steps;                                // set by the launch
};
cudaError_t launch_rotate(const RotateArgs& args, int d, int num_sms, cudaStream_t stream);

// Attention of one token a sequence over a paged cache (attend.cu).
constexpr size_t kAttNoScratch = 256;         // said of calls that need none
constexpr int kAttMaxCtas = 160;              // CTAs that leave records, at most
struct AttendArgs {
    const __nv_bfloat16 *q, *K, *V;
    const int32_t* lengths;                   // [B, Hkv]
    PagedCache cache;
    int B, Hq, Hkv;
    float scale_log2;                         // log2(e) / sqrt(d)
    float* weights;                           // [B, Hkv, cap] or NULL
    __nv_bfloat16* out;
    int groups, group;                        // groups of query heads of a KV head, and heads of one; these and what follows are set by the launch
    int blocks, block;                        // blocks of KV heads that a CTA takes together, and heads of one
    int tile, tile_shift;                     // rows that are dealt together; log2 where it is a power of two, else -1
    float2 *part_ml, *whole_ml;
    int2* shared_by;                          // first and last CTA with rows of a unit
    float *part_o, *logits;
    long long logit_stride;
    int small_rows;                           // rows of a CTA of a cluster, at most
};
struct AttendPlan {
    int nh, groups, group, blocks, block, tile, tile_shift, max_ctas;
    int cluster, warps, small_rows;           // CTAs of a cluster of the form for short caches (0: the other form), warps and rows of one
    long long logit_stride;
    size_t off_o, off_whole, off_shared, off_logits, bytes;
};
// wide: clusters of 16 CTAs can be launched (more than the eight that every device takes).
AttendPlan attend_plan(int B, int Hq, int Hkv, int d, int cap, bool sums, bool wide);
bool attend_wide_clusters();                  // on the current device
cudaError_t launch_attend(const AttendArgs& args, const AttendPlan& plan, int d, char* scratch, int num_sms, int device, cudaStream_t stream);

// Eviction from a paged cache by sums of attention (evict.cu).
struct EvictArgs {
    float* weights;                           // [B, Hkv, cap]
    int32_t* lengths;                         // [B, Hkv]
    uint4 *K, *V;
    PagedCache cache;
    int Hkv, w, c, budget;
    int32_t* out_idx;                         // [B, Hkv, budget]
    int list_cap, key_cap;                    // set by the launch
};
struct EvictPlan {
    bool fits;
    int list_cap, key_cap, smem_bytes;
};
EvictPlan evict_plan(int cap, int c, int smem_limit);
cudaError_t launch_evict(const EvictArgs& args, const EvictPlan& plan, int B, int d, int num_sms, cudaStream_t stream);

}  // namespace chunkkv
