// C ABI of the operators around the paged cache: argument checks, then kernel launches on the caller's stream.
#include "../../include/critiprefill.h"
#include "cache.h"

#include <cmath>

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// What every entry point needs.  `uses`: which of the sizes below it reads.
enum { USES_Q = 1, USES_PAGES = 2, USES_SEQS = 4, USES_TURN = 8 };

int make_cache_shape(const critiprefill_cache_params* p, int uses, cp::CacheShape* sh) {
    if (!p) return CP_ERR_NULL;
    if (p->n_kv_heads <= 0 || p->tokens < 0) return CP_ERR_SHAPE;
    if ((uses & USES_Q) && (p->n_q_heads <= 0 || p->n_q_heads % p->n_kv_heads != 0)) return CP_ERR_SHAPE;
    if (p->head_dim != cp::kHeadDim) return CP_ERR_UNSUPPORTED;
    if (p->dtype != CP_DTYPE_FP32 && p->dtype != CP_DTYPE_BF16) return CP_ERR_UNSUPPORTED;
    *sh = cp::CacheShape{};
    sh->hkv = p->n_kv_heads;
    sh->hq = (uses & USES_Q) ? p->n_q_heads : p->n_kv_heads; sh->group = sh->hq / sh->hkv;     // without USES_Q the field may hold anything
    sh->dtype = p->dtype; sh->tokens = p->tokens;
    if (sh->hq > 65535 || sh->hkv > 65535) return CP_ERR_UNSUPPORTED;
    if (uses & USES_PAGES) {
        if (p->n_pages <= 0 || p->page_size <= 0) return CP_ERR_SHAPE;
        if (p->cache_format != CP_CACHE_PLAIN && p->cache_format != CP_CACHE_MXFP8 && p->cache_format != CP_CACHE_MXFP4) return CP_ERR_UNSUPPORTED;
        if (p->page_size < 16 || (p->page_size & (p->page_size - 1))) return CP_ERR_UNSUPPORTED;
        if ((long long)p->n_pages * p->page_size >= (1ll << 31)) return CP_ERR_UNSUPPORTED;    // a slot is an int32
        sh->held = p->cache_format == CP_CACHE_MXFP4 ? cp::HELD_MXFP4 : p->cache_format == CP_CACHE_MXFP8 ? cp::HELD_MXFP8 : cp::HELD_PLAIN;
        sh->page = p->page_size; sh->n_pages = p->n_pages;
        while ((1 << sh->page_shift) < sh->page) ++sh->page_shift;
    }
    if (uses & USES_TURN) {
        if (p->rotary_dim < 0 || p->rotary_dim > cp::kHeadDim || !(p->norm_eps >= 0.f)) return CP_ERR_SHAPE;
        if (p->rotary_dim % 16) return CP_ERR_UNSUPPORTED;
        sh->rotary = p->rotary_dim; sh->interleaved = p->rotary_interleaved != 0; sh->eps = p->norm_eps;
    }
    if (uses & USES_SEQS) {
        if (p->n_seqs < 0 || p->max_pages < 0 || p->max_q_len < 0 || p->max_kv_len < 0 || !(p->attn_scale >= 0.f)) return CP_ERR_SHAPE;
        if (sh->group > 64) return CP_ERR_UNSUPPORTED;
        sh->n_seqs = p->n_seqs; sh->max_pages = p->max_pages; sh->max_q = p->max_q_len > 0 ? p->max_q_len : p->tokens;
        sh->scale = p->attn_scale > 0.f ? p->attn_scale : 1.0f / std::sqrt((float)p->head_dim);
        const long long keys = (long long)p->max_pages * p->page_size;
        if (keys >= (1ll << 30)) return CP_ERR_UNSUPPORTED;
        sh->max_kv = p->max_kv_len > 0 ? p->max_kv_len : keys;
        // key steps are counted in 32 bits
        const cp::PagedRoute r = cp::paged_route(*sh);
        const double tiles = (double)(sh->tokens >> r.tile_shift) + sh->n_seqs, steps = (double)(keys >> r.step_shift) + 2 + r.setup;
        if (tiles * steps * sh->hkv >= 2147483648.0) return CP_ERR_UNSUPPORTED;
    }
    for (int i = 0; i < 2; ++i) {
        sh->qs[i] = p->q_stride[i]; sh->ks[i] = p->k_stride[i]; sh->vs[i] = p->v_stride[i]; sh->os[i] = p->o_stride[i]; sh->kos[i] = p->ko_stride[i];
    }
    return CP_OK;
}

int check_tensor(const void* p, const int64_t* stride) {
    if (!p) return CP_ERR_NULL;
    if (!aligned16(p)) return CP_ERR_ALIGN;
    for (int i = 0; i < 2; ++i)
        if (stride[i] < 0 || (stride[i] & 7)) return CP_ERR_ALIGN;
    return CP_OK;
}

// written tensors: rows must not share elements, so all heads of a token lie before the next token, or all tokens of a head before the next head
int check_output(const void* p, const int64_t* stride, int tokens, int heads) {
    const int e = check_tensor(p, stride);
    if (e != CP_OK) return e;
    if (stride[0] < cp::kHeadDim || stride[1] < cp::kHeadDim) return CP_ERR_SHAPE;
    const bool apart = tokens == 1 || heads == 1 || (stride[0] - cp::kHeadDim) / stride[1] >= heads - 1 || (stride[1] - cp::kHeadDim) / stride[0] >= tokens - 1;
    return apart ? CP_OK : CP_ERR_SHAPE;
}

int check_cache(const cp::CacheShape& sh, const void* k, const void* v, const uint8_t* ks, const uint8_t* vs) {
    const bool scaled = sh.held != cp::HELD_PLAIN;
    if (!k || !v || (scaled && (!ks || !vs))) return CP_ERR_NULL;
    if (!aligned16(k) || !aligned16(v) || (scaled && (!aligned16(ks) || !aligned16(vs)))) return CP_ERR_ALIGN;
    return CP_OK;
}

int check_turn(const cp::CacheShape& sh, const void* q_weight, const void* k_weight, const double* inv_freq, const int32_t* positions) {
    if (sh.rotary && (!inv_freq || !positions)) return CP_ERR_NULL;
    if ((q_weight && !aligned16(q_weight)) || (k_weight && !aligned16(k_weight))) return CP_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(inv_freq) & 7u) || (reinterpret_cast<uintptr_t>(positions) & 3u)) return CP_ERR_ALIGN;
    return CP_OK;
}

int check_ints(const int32_t* p) { return !p ? CP_ERR_NULL : (reinterpret_cast<uintptr_t>(p) & 3u) ? CP_ERR_ALIGN : CP_OK; }

int done(hipError_t e) { return e == hipSuccess ? CP_OK : CP_ERR_LAUNCH; }

}  // namespace

#define CP_TRY(x) do { const int e_ = (x); if (e_ != CP_OK) return e_; } while (0)

extern "C" {

int critiprefill_norm_rope(const critiprefill_cache_params* p, const void* q, const void* k, const void* q_weight, const void* k_weight,
                           const double* inv_freq, const int32_t* positions, void* q_out, void* k_out, void* hip_stream) {
    cp::CacheShape sh;
    CP_TRY(make_cache_shape(p, USES_Q | USES_TURN, &sh));
    if (sh.tokens == 0) return CP_OK;
    CP_TRY(check_tensor(q, sh.qs)); CP_TRY(check_tensor(k, sh.ks));
    CP_TRY(check_output(q_out, sh.os, sh.tokens, sh.hq)); CP_TRY(check_output(k_out, sh.kos, sh.tokens, sh.hkv));
    CP_TRY(check_turn(sh, q_weight, k_weight, inv_freq, positions));
    return done(cp::launch_norm_rope(sh, q, k, nullptr, q_weight, k_weight, inv_freq, positions, nullptr, q_out, k_out, nullptr, (hipStream_t)hip_stream));
}

int critiprefill_norm_rope_write(const critiprefill_cache_params* p, const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight,
                                 const double* inv_freq, const int32_t* positions, const int32_t* slots, void* q_out, void* k_cache, void* v_cache,
                                 uint8_t* k_scale, uint8_t* v_scale, void* hip_stream) {
    cp::CacheShape sh;
    CP_TRY(make_cache_shape(p, USES_Q | USES_PAGES | USES_TURN, &sh));
    if (sh.tokens == 0) return CP_OK;
    CP_TRY(check_tensor(q, sh.qs)); CP_TRY(check_tensor(k, sh.ks)); CP_TRY(check_tensor(v, sh.vs));
    CP_TRY(check_output(q_out, sh.os, sh.tokens, sh.hq));
    CP_TRY(check_turn(sh, q_weight, k_weight, inv_freq, positions));
    CP_TRY(check_ints(slots));
    CP_TRY(check_cache(sh, k_cache, v_cache, k_scale, v_scale));
    const cp::CachePtr cache = {k_cache, v_cache, k_scale, v_scale};
    return done(cp::launch_norm_rope(sh, q, k, v, q_weight, k_weight, inv_freq, positions, slots, q_out, nullptr, &cache, (hipStream_t)hip_stream));
}

int critiprefill_cache_write(const critiprefill_cache_params* p, const void* k, const void* v, const int32_t* slots, void* k_cache, void* v_cache,
                             uint8_t* k_scale, uint8_t* v_scale, void* hip_stream) {
    cp::CacheShape sh;
    CP_TRY(make_cache_shape(p, USES_PAGES, &sh));
    if (sh.tokens == 0) return CP_OK;
    CP_TRY(check_tensor(k, sh.ks)); CP_TRY(check_tensor(v, sh.vs));
    CP_TRY(check_ints(slots));
    CP_TRY(check_cache(sh, k_cache, v_cache, k_scale, v_scale));
    const cp::CachePtr cache = {k_cache, v_cache, k_scale, v_scale};
    return done(cp::launch_cache_write(sh, k, v, slots, cache, (hipStream_t)hip_stream));
}

int critiprefill_cache_read(const critiprefill_cache_params* p, const int32_t* slots, const void* k_cache, const void* v_cache, const uint8_t* k_scale,
                            const uint8_t* v_scale, void* k, void* v, void* hip_stream) {
    cp::CacheShape sh;
    CP_TRY(make_cache_shape(p, USES_PAGES, &sh));
    if (sh.tokens == 0) return CP_OK;
    CP_TRY(check_output(k, sh.ks, sh.tokens, sh.hkv)); CP_TRY(check_output(v, sh.vs, sh.tokens, sh.hkv));
    CP_TRY(check_ints(slots));
    CP_TRY(check_cache(sh, k_cache, v_cache, k_scale, v_scale));
    const cp::CachePtr cache = {const_cast<void*>(k_cache), const_cast<void*>(v_cache), const_cast<uint8_t*>(k_scale), const_cast<uint8_t*>(v_scale)};
    return done(cp::launch_cache_read(sh, slots, cache, k, v, (hipStream_t)hip_stream));
}

size_t critiprefill_paged_workspace_bytes(const critiprefill_cache_params* p) {
    cp::CacheShape sh;
    if (make_cache_shape(p, USES_Q | USES_PAGES | USES_SEQS, &sh) != CP_OK) return 0;
    return cp::paged_workspace(sh);
}

int critiprefill_paged_attn(const critiprefill_cache_params* p, const void* q, const void* k_cache, const void* v_cache, const uint8_t* k_scale,
                            const uint8_t* v_scale, const int32_t* page_table, const int32_t* q_start, const int32_t* kv_len, void* out, float* lse,
                            void* workspace, size_t workspace_bytes, void* hip_stream) {
    cp::CacheShape sh;
    CP_TRY(make_cache_shape(p, USES_Q | USES_PAGES | USES_SEQS, &sh));
    if (sh.tokens == 0 || sh.n_seqs == 0) return CP_OK;
    CP_TRY(check_tensor(q, sh.qs));
    CP_TRY(check_output(out, sh.os, sh.tokens, sh.hq));
    CP_TRY(check_ints(q_start)); CP_TRY(check_ints(kv_len));
    if (sh.max_pages) CP_TRY(check_ints(page_table));
    if (lse && (reinterpret_cast<uintptr_t>(lse) & 3u)) return CP_ERR_ALIGN;
    CP_TRY(check_cache(sh, k_cache, v_cache, k_scale, v_scale));
    if (!workspace) return CP_ERR_NULL;
    if (!aligned16(workspace)) return CP_ERR_ALIGN;
    if (workspace_bytes < cp::paged_workspace(sh)) return CP_ERR_WORKSPACE;
    const cp::CachePtr cache = {const_cast<void*>(k_cache), const_cast<void*>(v_cache), const_cast<uint8_t*>(k_scale), const_cast<uint8_t*>(v_scale)};
    return done(cp::launch_paged_attn(sh, q, cache, page_table, q_start, kv_len, out, lse, workspace, (hipStream_t)hip_stream));
}

}  // extern "C"
