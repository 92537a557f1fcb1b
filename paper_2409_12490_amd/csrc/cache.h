// What the kernels around the paged cache share: the parameter block, where a token's row lies, the 8-bit format.
#pragma once
#include "kernels.h"

namespace cp {

// The parameter block of the cache operators, checked.
struct CacheShape {
    int hq, hkv, group;                       // group = hq / hkv
    int dtype;                                // 0 fp32, 1 bf16
    int mxfp8;                                // the cache holds e4m3 elements and a scale per 32 channels, else elements of dtype
    int page, page_shift, n_pages;            // tokens of a page, a power of two of at least 16
    int tokens, n_seqs, max_pages, max_q;
    long long max_kv;
    int rotary, interleaved;
    float eps, scale;                         // of the norm, of the logits
    int64_t qs[2], ks[2], vs[2], os[2], kos[2];   // element strides: token, head
};

// A cache: K and V pages [n_pages][hkv][page][128], and with mxfp8 the scales [n_pages][hkv][page][4], one byte e for 2^(e - 127).
struct CachePtr {
    void *k, *v;
    uint8_t *ks, *vs;
};

bool cache_call_streams(const CacheShape& sh, int rows, int held);
hipError_t launch_norm_rope(const CacheShape& sh, const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight,
                            const double* inv_freq, const int32_t* positions, const int32_t* slots, void* q_out, void* k_out, const CachePtr* cache, hipStream_t st);
hipError_t launch_cache_write(const CacheShape& sh, const void* k, const void* v, const int32_t* slots, const CachePtr& cache, hipStream_t st);
hipError_t launch_cache_read(const CacheShape& sh, const int32_t* slots, const CachePtr& cache, void* k, void* v, hipStream_t st);

// Attention of new tokens over the pages: a fixed number of workgroups share the key steps of all (sequence, KV head, row tile) units evenly.
struct PagedRoute {
    int chunk;                                // 0: the kernel whose waves split the keys, 1: the one whose waves split 256 rows
    int rows;                                 // rows (token, query head of the group) of a tile
    int tile_shift;                           // log2 of the tokens of a tile
    int step_shift;                           // log2 of the keys of a step
    int workgroups;
    int least;                                // steps that a workgroup takes at least
    int setup;                                // what a unit takes beside its steps, in steps
    int whole;                                // units are not cut: sequences are known to be short, and there is nothing to join
};
PagedRoute paged_route(const CacheShape& sh);
size_t paged_workspace(const CacheShape& sh);
hipError_t launch_paged_attn(const CacheShape& sh, const void* q, const CachePtr& cache, const int32_t* table, const int32_t* q_start, const int32_t* kv_len, void* out,
                             float* lse, void* workspace, hipStream_t st);

}  // namespace cp
