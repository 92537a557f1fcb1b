// Attention of the new tokens of each sequence over the pages of a cache, for few rows a KV head (single tokens above all) and for fp32:
//
//   o_t = sum_u p_tu v_u / sum_u p_tu,  p_tu = exp(q_t k_u scale - m_t),  u <= keys - tokens + t;  no such u: o_t = 0, lse_t = -inf
//
// A tile has up to 16 * NQ rows (a token's query heads of one KV head lie next to each other) and its keys are read once for all of them.  The four waves
// of a workgroup split the keys: a step gives each wave 32 (bf16; fp32: 16) of its own, with a running maximum, sum and output of its own, merged
// through LDS when the unit or the workgroup's run ends.  How the steps are dealt to workgroups: paged.h.
//
//   S^T[key][row]  = K . Q^T      16x16 MFMA, A = K straight from memory (a lane has one key's 32 neighbouring channels), B = Q in registers
//   softmax                       one row per lane column
//   O^T[ch][row]  += V^T . P^T    A = V straight from memory, 8 channels of a token to a lane (whole rows per instruction); the pairs of tokens that a bf16
//                                 operand wants come from v_perm, and the channel that an operand row stands for is the lane's own choice: lane c, operand
//                                 n is channel 8 c + n.  B = P^T, the S^T accumulators as they stand.
// Nothing goes through LDS and no wave waits for another in the key loop: K of the next step is asked for when QK has read this one's, V when PV has, and the other wave
// of the SIMD works meanwhile (both a whole step ahead in registers of their own: as fast for one token, 20 % slower for 32 rows, where a second wave then has no room).
// 8-bit keys and values become bf16 (exact: their scales are powers of two) or fp32 in registers.
//
// What bounds it, 32/8 heads: the memory, with all of K and V read once: one token after 131071 in bf16 95 us and 5.7 TB/s (reads past the caches reach 7.0), 48 single tokens
// of up to 32769 each over 8-bit pages 74 us and 5.3 TB/s; MFMA and vector units are busy for a twentieth of that.  After 1999 tokens it is latency: 7 us, of which an empty launch
// takes 3, then lengths, page table, keys and the join's launch one after another (4 more).  fp32, 4/2 heads: the matrix units (16x16x4 fp32 MFMAs, 154 TFLOP/s in a large product)
// for two thirds of 20 x 200 tokens after 8000 (684 us); of 3 x up to 200 after 3000 (32 us) for 15, the rest are the beginnings and ends of runs of eight steps.  Two workgroups of
// 32 fp32 rows to a compute unit, within 256 registers: no faster for 20 x 200 after 8000, up to 40 % slower for less.
#include "paged.h"

#include <algorithm>
#include <cmath>

namespace cp {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef const __attribute__((address_space(4))) int32_t* scalar_list;   // read through scalar loads: wave-uniform addresses

constexpr float kLazyLog2 = 8.0f;             // how far a row's max may outgrow its reference point before O is rescaled
constexpr int kThreads = 256;

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { union { u32x4 u; bf16x8 b; } c; c.u = v; return c.b; }
__device__ __forceinline__ unsigned as_u32(bf16x2 v) { union { bf16x2 b; unsigned u; } c; c.b = v; return c.u; }

// max and sum over the four lanes that share a column: l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float column_max(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float column_sum(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ float mx_scale(unsigned byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ u32x2 widen4(unsigned w, float scale) {      // four e4m3 to bf16
    u32x2 r;
    r[0] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
    r[1] = as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
    return r;
}
__device__ __forceinline__ f32x4 widen4f(unsigned w, float scale) {     // to fp32
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
    return f32x4{lo[0], lo[1], hi[0], hi[1]};
}

// What a wave has of a step: K and V as they come from memory.
template <bool F32, bool MX> struct Raw;
template <> struct Raw<false, false> { u32x4 k[2][4]; u32x4 v[8]; };                           // [16 keys][64 bytes]; [token]
template <> struct Raw<false, true> { u32x4 k[2][2]; u32x2 v[8]; unsigned ks[2]; u32x4 vs[2]; };
template <> struct Raw<true, false> { f32x4 k[8]; f32x4 v[4][2]; };
template <> struct Raw<true, true> { u32x4 k[2]; unsigned v[4][2]; unsigned ks; u32x4 vs; };

template <bool F32, bool MX, int NQ>
__global__ __launch_bounds__(kThreads, NQ == 1 || !F32 ? 2 : 1) void paged_rows_kernel(PagedArgs a) {
    constexpr int kRows = 16 * NQ, kWaveKeys = F32 ? 16 : 32, kGroups = kWaveKeys / 16;
    constexpr int kRowBytes = MX ? kHeadDim : (F32 ? 512 : 256);
    extern __shared__ __attribute__((aligned(16))) float merge[];              // [wave][row][128], then (max, sum) [wave][row]
    float* const wave_stats = merge + 4 * kRows * kHeadDim;

    const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, kg = lane >> 4;
    const int wave = first_lane(tid >> 6);
    Run<false> run;
    const bool any = run.find(a, blockIdx.x, lane);
    if (blockIdx.x == 0 && tid == 0) a.record[0] = (int)run.used;
    if (run.logical < run.used && tid == 0) a.record[4 + 4 * run.logical + 3] = 0;
    if (!any) return;
    const unsigned home = run.logical;
    const float c = a.scale_log2e, lazy_raw = fminf(kLazyLog2 / c, 3e38f);      // not infinite, whatever the scale: no maximum would be taken over then
    const int page_mask = (1 << a.page_shift) - 1;

    while (true) {
        const Sequence seq = run.now;
        const int tile_tokens = 1 << a.tile_shift, t0 = run.tile << a.tile_shift;
        const int live = min(tile_tokens, seq.tokens - t0);                    // tokens of the tile
        unsigned first, count, unit;
        run.piece(a, first, count, unit);
        const int head = run.head;
        const scalar_list table = (scalar_list)(unsigned long long)(a.table + (int64_t)run.seq * a.max_pages);
        const int past = seq.keys - seq.tokens;                                // position of the sequence's first new token
        const int low = min(past + t0, seq.keys - 1), high = min(past + t0 + live, seq.keys) - 1;   // last keys that its first and its last row see

        // ---- Q: lane's column is a row, 8 channels at 32 kg + 8 ks (fp32: 32 at 32 kg)
        bf16x8 qf[F32 ? 1 : NQ][4];
        f32x4 qw[F32 ? NQ : 1][8];
        int last[NQ];                                                          // the last key that the row sees
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            const int r = 16 * nq + c16, of = (int)a.by_group.div((unsigned)r), t = min(of, live - 1), g = r - of * a.group;
            last[nq] = min(past + t0 + t, seq.keys - 1);
            const int64_t at = (seq.start + t0 + t) * a.qs0 + (int64_t)(head * a.group + g) * a.qs1 + 32 * kg;
            if (F32) {
#pragma unroll
                for (int x = 0; x < 8; ++x) qw[F32 ? nq : 0][x] = *(const f32x4*)((const float*)a.q + at + 4 * x);
            } else {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) qf[F32 ? 0 : nq][ks] = *(const bf16x8*)((const __bf16*)a.q + at + 8 * ks);
            }
        }

        f32x4 o[NQ][8];
        float m_run[NQ], l_run[NQ];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            m_run[nq] = -INFINITY; l_run[nq] = 0.f;
#pragma unroll
            for (int n = 0; n < 8; ++n) o[nq][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        // ---- loads.  Pages are looked up a step ahead; one that is not in the pool holds nothing: its keys are hidden, and read from page 0
        int entry[kGroups];
        bool odd = false;                                                      // see the loop
        auto key_of = [&](unsigned step) { return (int)(step << a.step_shift) + wave * kWaveKeys; };
        auto look_up = [&](unsigned step) __attribute__((always_inline)) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int u = key_of(step) + 16 * g;
                entry[g] = table[max(min(u, high), 0) >> a.page_shift];        // no branch; whether the keys are there is asked in load
            }
        };
        Raw<F32, MX> raw;
        int seen[kGroups], seen_next[kGroups];                                 // keys of a group that exist, of this step and the next
        int64_t at[kGroups];                                                   // first row of the groups asked for last
        auto load_k = [&](unsigned step) __attribute__((always_inline)) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int u = key_of(step) + 16 * g;
                const bool there = (unsigned)entry[g] < (unsigned)a.n_pages && u <= high;
                seen_next[g] = there ? seq.keys - u : 0;
                at[g] = (((int64_t)(there ? entry[g] : 0) * a.hkv + head) << a.page_shift) + (u & page_mask);
                const char* kp = (const char*)a.cache.k + at[g] * kRowBytes;
                if constexpr (!F32) {
                    const int per = MX ? 32 : 64;
#pragma unroll
                    for (int x = 0; x < (MX ? 2 : 4); ++x) raw.k[g][x] = *(const u32x4*)(kp + c16 * kRowBytes + kg * per + 16 * x);
                    if constexpr (MX) raw.ks[g] = (a.cache.ks + at[g] * 4)[c16 * 4 + kg];
                } else if constexpr (MX) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) raw.k[x] = *(const u32x4*)(kp + c16 * kRowBytes + kg * 32 + 16 * x);
                    raw.ks = (a.cache.ks + at[g] * 4)[c16 * 4 + kg];
                } else {
#pragma unroll
                    for (int x = 0; x < 8; ++x) raw.k[x] = *(const f32x4*)(kp + c16 * kRowBytes + kg * 128 + 16 * x);
                }
            }
        };
        auto load_v = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const char* vp = (const char*)a.cache.v + at[g] * kRowBytes;
                if constexpr (!F32) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (MX) raw.v[4 * g + i] = *(const u32x2*)(vp + (4 * kg + i) * kRowBytes + 8 * c16);
                        else raw.v[4 * g + i] = *(const u32x4*)(vp + (4 * kg + i) * kRowBytes + 16 * c16);
                    }
                    if constexpr (MX) raw.vs[g] = *(const u32x4*)(a.cache.vs + at[g] * 4 + 16 * kg);   // of four tokens
                } else if constexpr (MX) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int x = 0; x < 2; ++x) raw.v[i][x] = *(const unsigned*)(vp + (4 * kg + i) * kRowBytes + 4 * c16 + 64 * x);
                    raw.vs = *(const u32x4*)(a.cache.vs + at[g] * 4 + 16 * kg);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int x = 0; x < 2; ++x) raw.v[i][x] = *(const f32x4*)(vp + (4 * kg + i) * kRowBytes + 16 * c16 + 256 * x);
                }
            }
        };
        // ---- the loop.  K of the next step is asked for when QK has read this one's, V when PV has: each has half a step and the other wave of the SIMD to land in
        look_up(first); load_k(first); load_v();
        look_up(first + 1);
        for (unsigned x = 0; x < count; ++x) {
            const int u0 = key_of(first + x);
            const bool more = x + 1 < count;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) seen[g] = seen_next[g];
            f32x4 s[NQ][kGroups];
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                for (int g = 0; g < kGroups; ++g) s[nq][g] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (!F32) {
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) {
                        u32x4 kw;
                        if constexpr (MX) {
                            const float scale = mx_scale(raw.ks[g]);
                            const u32x2 lo = widen4(raw.k[g][ks >> 1][2 * (ks & 1)], scale), hi = widen4(raw.k[g][ks >> 1][2 * (ks & 1) + 1], scale);
                            kw = u32x4{lo[0], lo[1], hi[0], hi[1]};
                        } else kw = raw.k[g][ks];
#pragma unroll
                        for (int nq = 0; nq < NQ; ++nq) s[nq][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kw), qf[nq][ks], s[nq][g], 0, 0, 0);
                    }
            } else {
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    f32x4 kw;
                    if constexpr (MX) kw = widen4f(raw.k[x >> 2][x & 3], mx_scale(raw.ks));
                    else kw = raw.k[x];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int nq = 0; nq < NQ; ++nq) s[nq][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(kw[e], qw[nq][x][e], s[nq][0], 0, 0, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) load_k(first + x + 1);
            __builtin_amdgcn_sched_barrier(0);
            // Hidden keys: behind the row's own, or without a page.  Their values may hold anything, and a weight of 0 does not keep an infinity or NaN out of a
            // sum: rows of V that no row sees become 0, and so does what is not finite in those that some rows do not see (only with more than one token); `odd`
            // says that there was any, and the unit's end adds it for the rows that see it.
            bool whole = u0 + kWaveKeys - 1 <= low;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) whole = whole && seen[g] > 0;
            if (!whole) {
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq) {
                        const int lim = seen[g] > 0 ? last[nq] - u0 - 16 * g - 4 * kg : -1;
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[nq][g][i] = i > lim ? -INFINITY : s[nq][g][i];
                    }
                    const int lim = seen[g] > 0 ? high - u0 - 16 * g - 4 * kg : -1, sure = low - u0 - 16 * g - 4 * kg;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        bool any = false;
                        auto clean32 = [&](float x) { const bool bad = (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; any = any || bad; return bad ? 0.f : x; };
                        auto clean8 = [&](unsigned x) {                        // e4m3: 0x7f of either sign
                            unsigned keep = 0;
#pragma unroll
                            for (int e = 0; e < 4; ++e) keep |= ((x >> (8 * e)) & 0x7f) == 0x7f ? 0u : 0xffu << (8 * e);
                            any = any || ~keep;
                            return x & keep;
                        };
                        if constexpr (!F32 && MX) {
                            if (i > lim) { raw.v[4 * g + i] = u32x2{0, 0}; raw.vs[g][i] = 0x7f7f7f7fu; }
                            else if (i > sure) { raw.v[4 * g + i][0] = clean8(raw.v[4 * g + i][0]); raw.v[4 * g + i][1] = clean8(raw.v[4 * g + i][1]); }
                        } else if constexpr (!F32) {
                            if (i > lim) raw.v[4 * g + i] = u32x4{0, 0, 0, 0};
                            else if (i > sure) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const unsigned x = raw.v[4 * g + i][e];
                                    const unsigned keep = ((x & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u) | ((x & 0x7f80u) == 0x7f80u ? 0u : 0xffffu);
                                    any = any || ~keep;
                                    raw.v[4 * g + i][e] = x & keep;
                                }
                            }
                        } else if constexpr (MX) {
                            if (i > lim) { raw.v[i][0] = raw.v[i][1] = 0; raw.vs[i] = 0x7f7f7f7fu; }
                            else if (i > sure) { raw.v[i][0] = clean8(raw.v[i][0]); raw.v[i][1] = clean8(raw.v[i][1]); }
                        } else {
                            if (i > lim) raw.v[i][0] = raw.v[i][1] = f32x4{0.f, 0.f, 0.f, 0.f};
                            else if (i > sure) {
#pragma unroll
                                for (int e = 0; e < 8; ++e) raw.v[i][e >> 2][e & 3] = clean32(raw.v[i][e >> 2][e & 3]);
                            }
                        }
                        if (any) odd = true;
                    }
                }
            }
            bf16x8 pf[F32 ? 1 : NQ];
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) {
                float mx = fmaxf(fmaxf(s[nq][0][0], s[nq][0][1]), fmaxf(s[nq][0][2], s[nq][0][3]));
                if constexpr (!F32) mx = fmaxf(fmaxf(fmaxf(s[nq][1][0], s[nq][1][1]), fmaxf(s[nq][1][2], s[nq][1][3])), mx);
                mx = column_max(mx);
                // the reference point moves only when the maximum has outgrown it by 2^kLazyLog2: P <= 2^8 meanwhile, the same factor in O and l
                const float m_new = mx > m_run[nq] + lazy_raw ? mx : m_run[nq];
                const float m_safe = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = __builtin_amdgcn_exp2f((m_run[nq] - m_safe) * c);
                const float ms = m_safe * c;
                m_run[nq] = m_new;
                float sum = 0.f;
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(s[nq][g][i], c, -ms));
                        sum += p;                                              // before P is rounded for the product: lse is as exact as fp32 allows
                        if constexpr (F32) s[nq][g][i] = p;
                        else pf[nq][4 * g + i] = (__bf16)p;
                    }
                l_run[nq] = l_run[nq] * alpha + sum;
                if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
                    for (int n = 0; n < 8; ++n) o[nq][n] *= alpha;
                }
            }
            if constexpr (!F32) {
                u32x4 v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if constexpr (MX) {
                        const float scale = mx_scale((raw.vs[j >> 2][j & 3] >> (8 * (c16 >> 2))) & 0xff);
                        const u32x2 lo = widen4(raw.v[j][0], scale), hi = widen4(raw.v[j][1], scale);
                        v[j] = u32x4{lo[0], lo[1], hi[0], hi[1]};
                    } else v[j] = raw.v[j];
                }
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    u32x4 w;                                                   // channel n of the lane's 8 tokens
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_perm(v[2 * e + 1][n >> 1], v[2 * e][n >> 1], n & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq) o[nq][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), pf[nq], o[nq][n], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4 v[2];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if constexpr (MX) v[x] = widen4f(raw.v[i][x], mx_scale((raw.vs[i] >> (16 * x + 8 * (c16 >> 3))) & 0xff));
                        else v[x] = raw.v[i][x];
                    }
#pragma unroll
                    for (int n = 0; n < 8; ++n)
#pragma unroll
                        for (int nq = 0; nq < NQ; ++nq) o[nq][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[n >> 2][n & 3], s[nq][0][i], o[nq][n], 0, 0, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) { load_v(); look_up(first + x + 2); }
        }

        if (__builtin_amdgcn_ballot_w64(odd) != 0) {
            for (unsigned x = 0; x < count; ++x)
                for (int i = 0; i < kWaveKeys; ++i) {                          // once in a blue moon: a key after another, from memory
                    const int u = key_of(first + x) + i;
                    if (u <= low || u > high) continue;
                    const int page = table[u >> a.page_shift];
                    if ((unsigned)page >= (unsigned)a.n_pages) continue;
                    const int64_t row = (((int64_t)page * a.hkv + head) << a.page_shift) + (u & page_mask);
#pragma unroll
                    for (int n = 0; n < 8; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {                          // o[][n][e] is this channel's
                            const int ch = F32 ? 64 * (n >> 2) + 4 * (4 * kg + e) + (n & 3) : 8 * (4 * kg + e) + n;
                            float v;
                            if constexpr (MX) {
                                const unsigned b = ((const uint8_t*)a.cache.v)[row * kRowBytes + ch];
                                v = (b & 0x7f) == 0x7f ? NAN : 0.f;
                            } else if constexpr (F32) v = ((const float*)((const char*)a.cache.v + row * kRowBytes))[ch];
                            else v = __uint_as_float((unsigned)((const uint16_t*)((const char*)a.cache.v + row * kRowBytes))[ch] << 16);
                            const bool bad = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u;
#pragma unroll
                            for (int nq = 0; nq < NQ; ++nq)
                                if (bad && u <= last[nq]) o[nq][n][e] += v;
                        }
                }
        }

        // ---- merge the four waves: sum_w 2^(c (m_w - M)) O_w; 16-byte pieces of a row swizzled by the row
        __syncthreads();                                                       // the unit before has been read
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            const int r = 16 * nq + c16;
            const float l = column_sum(l_run[nq]);
            if (kg == 0) { wave_stats[2 * (wave * kRows + r)] = m_run[nq]; wave_stats[2 * (wave * kRows + r) + 1] = l; }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int half = 0; half < 2; ++half) {                         // channels 8 (4 kg + i) + 4 half ..; fp32: 64 half + 4 (4 kg + i) ..
                    const int piece = F32 ? 16 * half + 4 * kg + i : 2 * (4 * kg + i) + half;
                    f32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = o[nq][4 * half + e][i];
                    *(f32x4*)(merge + (wave * kRows + r) * kHeadDim + 4 * (piece ^ c16)) = w;
                }
        }
        __syncthreads();
        const bool began = first == 0, ended = first + count == unit;
        const int64_t slot = 2 * (int64_t)home + (began ? 1 : 0);
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            const int r = 16 * nq + (tid >> 4), piece = tid & 15;              // 8 channels
            const int t = (int)a.by_group.div((unsigned)r), g = r - t * a.group;
            if (t >= live) continue;
            float M = -INFINITY, L = 0.f, sum[8];
#pragma unroll
            for (int w = 0; w < 4; ++w) M = fmaxf(M, wave_stats[2 * (w * kRows + r)]);
            const float M_safe = M == -INFINITY ? 0.f : M;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = __builtin_amdgcn_exp2f((wave_stats[2 * (w * kRows + r)] - M_safe) * c);
                L = fmaf(f, wave_stats[2 * (w * kRows + r) + 1], L);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const f32x4 v = *(const f32x4*)(merge + (w * kRows + r) * kHeadDim + 4 * ((2 * piece + half) ^ (r & 15)));
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[4 * half + e] = fmaf(f, v[e], sum[4 * half + e]);
                }
            }
            if (began && ended) {
                const float inv = L == 0.f ? 0.f : 1.0f / L;
                const int64_t row = seq.start + t0 + t;
                const int h = head * a.group + g;
                const int64_t at = row * a.os0 + h * a.os1 + 8 * piece;
                if (F32) {
                    *(f32x4*)((float*)a.out + at) = f32x4{sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv};
                    *(f32x4*)((float*)a.out + at + 4) = f32x4{sum[4] * inv, sum[5] * inv, sum[6] * inv, sum[7] * inv};
                } else {
                    bf16x8 w;
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = (__bf16)(sum[e] * inv);
                    *(bf16x8*)((__bf16*)a.out + at) = w;
                }
                if (a.lse && piece == 0) a.lse[row * a.hq + h] = L == 0.f ? -INFINITY : M * a.scale + logf(L);
            } else {
                float* to = a.parts + (slot * kRows + r) * kHeadDim + 8 * piece;
                *(f32x4*)to = f32x4{sum[0], sum[1], sum[2], sum[3]};
                *(f32x4*)(to + 4) = f32x4{sum[4], sum[5], sum[6], sum[7]};
                if (piece == 0) *(f32x2*)(a.stats + 2 * (slot * kRows + r)) = f32x2{M, L};
            }
        }
        if (began && !ended && tid == 0) {
            const unsigned rest = unit - first - count;                        // of whole runs, the last perhaps not whole
            int32_t* rec = a.record + 4 + 4 * home;
            rec[0] = seq.start + t0; rec[1] = live; rec[2] = head; rec[3] = 1 + (int)((rest + run.share - 1) / run.share);
        }
        if (!run.next_steps(a)) break;
    }
}

template <bool F32, bool MX, int NQ>
hipError_t launch(const PagedArgs& a, hipStream_t st) {
    constexpr int smem = 4 * 16 * NQ * (kHeadDim + 2) * 4;
    if (smem > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)paged_rows_kernel<F32, MX, NQ>, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((paged_rows_kernel<F32, MX, NQ>), dim3(a.workgroups), dim3(kThreads), smem, st, a);
    return hipGetLastError();
}

int log2_of(int x) { int s = 0; while ((2 << s) <= x) ++s; return s; }        // rounded down

}  // namespace

PagedRoute paged_route(const CacheShape& sh) {
    PagedRoute r;
    const bool f32 = sh.dtype == 0;
    // All of these lines were measured at 32/8 heads (fp32: 4/2), and go by rows, units and keys alone.
    // Tiles of 256 rows pay from more than 16 rows on, 8-bit pages from 32; up to 32 rows not for few units and keys (and not where a token alone has more than 16).  us, 32/8 heads, waves that split the keys / tiles of 256 rows:
    // 1 x 4 tokens of 2000 10.8 / 16.1, of 60000 44 / 56, 8 x 4 of 2000 23.6 / 26.3, of 16000 102 / 105; 1 x 8 of 2000 14.1 / 16.3, of 16000 24.6 / 29.1, of 60000 78 / 57, 8 x 8 of 2000
    // 32.5 / 26.3, of 16000 127 / 104; 8 bits: 1 x 8 of 16000 19.9 / 28.9, 8 x 8 55 / 106, 8 x 16 114 / 112.
    const long long want = (long long)sh.max_q * sh.group;
    const double heads = (double)sh.n_seqs * sh.hkv;
    r.chunk = !f32 && want > (sh.mxfp8 ? 32 : 16) && !(sh.group <= 16 && want <= 32 && heads <= 8 && sh.max_kv <= 24576);
    // Sequences known to be short: units are not cut, and nothing is joined.  us, cut / whole, 32/8 heads: 1 token after 255 10.1 / 7.8, after 509 10.2 / 10.1, after 999 10.2 / 14.7;
    // fp32 (steps of half as many keys, and slower) 8 x 1 of up to 512 12.2 / 17.1.  With units for a quarter of the chip the join has more to read and longer units pay: 8 x 1 of 760
    // 13.0 / 12.5, of 1000 15.6 / 15.9, 32 x 1 of 760 26.0 / 19.5, 8 bits 8 x 1 of 760 12.6 / 10.7, of 1000 14.0 / 12.3, of 1500 14.2 / 16.4, 32 x 1 of 1000 22.2 / 15.8 (a single long
    // one among short ones: 20 % lost).  Tiles of 256 rows: 8 units (1 x 64) of 250 keys 16.4 / 15.9, of 510 17.0 / 21.6; 16 (2 x 64) of 510 22.2 / 21.7, of 760 24.6 / 27.5; 80 (2 x 300)
    // of 510 25.9 / 22.3, of 760 31.7 / 28.0, of 1000 34.2 / 33.0.
    // (Eight waves to a workgroup, half as many steps: no faster; a unit's 56 GB/s are what one compute unit reads.)
    const int brief = f32 ? 128 : heads < 64 ? 512 : sh.mxfp8 ? 1024 : 768;
    if (r.chunk) {
        r.rows = 256; r.tile_shift = log2_of(256 / sh.group); r.step_shift = 6; r.workgroups = 256; r.least = 2; r.setup = 5;
        const double units = heads * (((long long)sh.max_q + (1 << r.tile_shift) - 1) >> r.tile_shift);
        r.whole = sh.max_kv <= (units < 16 ? 256 : units < 64 ? 512 : 768);
        return r;
    }
    // The smallest tile that holds a sequence's new tokens, up to 16 rows, in bf16 over 8-bit pages (K and V converted once) and fp32 over plain ones (K and V read once) 32.  Of fp32
    // with 32 rows one workgroup has room on a compute unit, and few steps are better shared by twice as many of 16: us, 32 / 16 rows (4/2 heads): 1 x 9 tokens after 3000
    // 16.2 / 13.0, 1 x 16 after 8000 26.4 / 21.1, 1 x 50 after 600 15.5 / 13.2, after 3000 20.4 / 21.6, 8 x 16 after 3000 28.7 / 36.2, 1 x 500 after 8000 99 / 117; 8-bit pages 1 x 50 after
    // 600 15.3 / 12.8, 3 x 200 after 3000 56 / 52, 20 x 200 after 8000 720 / 645.
    int most = sh.mxfp8 ? 2 : 1;
    if (f32) {
        const int shift = log2_of(std::max(1, 32 / sh.group));
        const double steps = (double)sh.n_seqs * sh.hkv * (((long long)sh.max_q + (1 << shift) - 1) >> shift) * ((double)(sh.max_kv >> 6) + 1);
        most = !sh.mxfp8 && steps > 256 ? 2 : 1;
    }
    int nq = 1;
    while (nq < most && (16 * nq < sh.group || (1 << log2_of(16 * nq / sh.group)) < sh.max_q)) nq *= 2;
    while (16 * nq < sh.group) nq *= 2;                             // fp32: 33 to 64 query heads a KV head
    r.rows = 16 * nq;
    r.tile_shift = log2_of(r.rows / sh.group);
    r.step_shift = f32 ? 6 : 7;
    r.workgroups = nq == 1 || !f32 ? 512 : 256;                     // two to a compute unit, where their registers allow it
    r.least = 1;
    r.setup = 1;
    r.whole = sh.max_kv <= brief;
    return r;
}

// No more workgroups than there can be runs, from what the host knows of the lengths: any number is right, and those without a run take time to begin and end, in the
// join above all.  A multiple of 8, see Run.
static double most_units(const CacheShape& sh, const PagedRoute& r) { return (double)sh.hkv * ((sh.tokens >> r.tile_shift) + (double)sh.n_seqs); }
static unsigned useful_workgroups(const CacheShape& sh, const PagedRoute& r) {
    const double units = most_units(sh, r), steps = (double)(sh.max_kv >> r.step_shift) + 2 + r.setup;
    const double runs = r.whole ? units : units * steps / r.least;
    return (unsigned)std::min<double>(r.workgroups, 8.0 * std::ceil(runs / 8));
}

size_t paged_workspace(const CacheShape& sh) {
    CacheShape many = sh;                                          // the larger of what the number of sequences decides between
    many.n_seqs = 1 << 20;
    const PagedRoute r = paged_route(many);                         // fp32: 512 workgroups of 16 rows or 256 of 32, the same bytes but for the records
    return (size_t)r.workgroups * 2 * r.rows * (kHeadDim + 2) * 4 + (4 + 4 * (size_t)512) * 4;
}

hipError_t launch_paged_rows(const CacheShape& sh, const PagedRoute& route, const PagedArgs& a, hipStream_t st) {
    const int nq = route.rows / 16;
    if (sh.dtype == 0) {
        if (sh.mxfp8) return nq == 1 ? launch<true, true, 1>(a, st) : nq == 2 ? launch<true, true, 2>(a, st) : launch<true, true, 4>(a, st);
        return nq == 1 ? launch<true, false, 1>(a, st) : nq == 2 ? launch<true, false, 2>(a, st) : launch<true, false, 4>(a, st);
    }
    if (sh.mxfp8) return nq == 1 ? launch<false, true, 1>(a, st) : launch<false, true, 2>(a, st);
    return launch<false, false, 1>(a, st);
}

hipError_t launch_paged_attn(const CacheShape& sh, const void* q, const CachePtr& cache, const int32_t* table, const int32_t* q_start, const int32_t* kv_len, void* out,
                             float* lse, void* workspace, hipStream_t st) {
    const PagedRoute route = paged_route(sh);
    PagedArgs a;
    a.q = q; a.cache = cache; a.table = sh.max_pages ? table : kv_len; a.q_start = q_start; a.kv_len = kv_len; a.out = out; a.lse = lse;
    a.parts = (float*)workspace;
    a.stats = a.parts + (size_t)route.workgroups * 2 * route.rows * kHeadDim;
    a.record = (int32_t*)(a.stats + (size_t)route.workgroups * 2 * route.rows * 2);
    a.tokens = sh.tokens; a.n_seqs = sh.n_seqs; a.max_pages = sh.max_pages; a.n_pages = sh.n_pages; a.hq = sh.hq; a.hkv = sh.hkv; a.group = sh.group;
    a.page_shift = sh.page_shift; a.tile_shift = route.tile_shift; a.step_shift = route.step_shift;
    a.workgroups = useful_workgroups(sh, route); a.cut_units = (unsigned)std::min<double>(a.workgroups, most_units(sh, route)); a.least = route.least; a.setup = route.setup; a.whole = route.whole; a.mxfp8 = sh.mxfp8;
    a.by_group = FastDiv(sh.group);
    a.scale = sh.scale; a.scale_log2e = sh.scale * 1.4426950408889634f;
    a.qs0 = sh.qs[0]; a.qs1 = sh.qs[1]; a.os0 = sh.os[0]; a.os1 = sh.os[1];
    if (route.chunk) return launch_paged_chunk(sh, a, st);
    hipError_t e = launch_paged_rows(sh, route, a, st);
    if (e != hipSuccess) return e;
    if (route.whole) return hipSuccess;
    // A workgroup of the join takes a row with eight groups of threads, or two with four; more rows than its grid has, where a chunk is longer than was said, come in
    // turn.  Eight and four: 1 x 4 tokens after 5000 (16 rows, 64 parts) 16.1 and 17.2 us; 8 x 8 after 16000 over 8-bit pages (32 rows) 70 and 67, fp32 4/2 heads 3 x 200 40.6 and 38.7.
    const int rows = (int)std::min<long long>(route.rows, (long long)std::min(sh.max_q, 1 << route.tile_shift) * sh.group);
    const dim3 grid(a.cut_units, (unsigned)(rows <= 16 ? rows : (rows + 1) / 2));
    if (sh.dtype == 0) {
        if (rows <= 16) hipLaunchKernelGGL((join_kernel<float, false, 8>), grid, dim3(256), 0, st, a, route.rows, grid.y);
        else hipLaunchKernelGGL((join_kernel<float, false, 4>), grid, dim3(256), 0, st, a, route.rows, grid.y);
    } else {
        if (rows <= 16) hipLaunchKernelGGL((join_kernel<__bf16, false, 8>), grid, dim3(256), 0, st, a, route.rows, grid.y);
        else hipLaunchKernelGGL((join_kernel<__bf16, false, 4>), grid, dim3(256), 0, st, a, route.rows, grid.y);
    }
    return hipGetLastError();
}

}  // namespace cp
