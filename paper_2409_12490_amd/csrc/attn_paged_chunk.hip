// Attention of chunks of new tokens over the pages of a cache: bf16, for tiles of 256 rows, which multiply more than they read.  The units, how they are dealt
// to workgroups and how the parts of a unit are joined: paged.h.
//
// A workgroup of 8 waves takes 256 rows, 32 a wave; a row is a token's query head, so a KV head's query heads read its keys together.  The waves and their key
// loop are those of the 256-row kernel over contiguous keys (attn_bf16.hip, where the reasons stand): S^T = K . Q^T and O^T += V^T . P^T in 32x32x16 MFMA, two waves to
// a SIMD half a period apart, K and V in rings of four tiles of 64 keys in LDS, 16-byte pieces swizzled by the row.  What differs: a tile's rows come from up to
// four pages, looked up by scalar loads a step ahead (pages are whole multiples of 16 tokens, so the rows of one load lie together); rows past the sequence's end lie in
// its last page and may hold anything, so rows of V that no row sees are zeroed in LDS; the row sum adds P before it is rounded, since the log-sum-exp is an
// output in its own right here (32 additions a step for 16 dot products).
// Pages of 8 and 4 bits: the 512 threads share a tile out, take their 16 bytes of it into registers a step ahead, and write them to LDS as bf16 (exact: the scales are powers of two), where
// conversion at the reads from LDS would have each wave convert all of it.  8 bits: 16 channels of a row of K and of V; 4 bits: the 32 channels of one scale, of K or of V.
//
// What bounds it, 32/8 heads: the matrix units under the clock that they leave, as in attn_bf16.hip: 8192 new tokens of 32768 3.16 ms, 1.22 PFLOP/s, where a large product of the
// library reaches 1.24; the MFMA pipe is busy for 55 % of the launch, the vector units for 43 %, 96 % of the reads come from L2.  Over 8-bit pages 3.38 ms: 14 % more vector
// instructions; over pages of 4 bits 3.23 ms, and 4096 of 32768 1.73 ms, 1.19 PFLOP/s.  512 after 16384: 138 us, 1.01 PFLOP/s, 64 units in 314 pieces and 10 us to join them.  Mixed batches and short follow-ups: the beginnings and ends of pieces, 5 steps' worth each
// (12 sequences of 1 to 300 new tokens, 32/4 heads, 8 bits: 388 pieces for 156 units, 98 us and 9.5 to join; 20 of these, 4 bits: 478 pieces for 232 units, 121 us and 11 to join; 1 x 64 of 2000 21 us in all, MFMA busy for a twentieth of it).
// Not kept: 8-bit bytes by way of LDS, three tiles in flight (no faster at 109 us for 8 x 4 tokens after 16000, 4 % slower in mixed batches); conversion that writes to LDS without bank
// conflicts at the price of selections (257 conflict cycles a step less, 3 % slower); the places of the key loops within 32 bytes (1 % between the best and the worst).
#include "attn_bf16.h"
#include "paged.h"

#include <algorithm>

namespace cp {
namespace {

constexpr int kChunkRows = 256, WQ = 32, TK = 64, NBUF = 4;
constexpr int kTileBytes = TK * 256;
constexpr int kVOff = 0, kKOff = NBUF * kTileBytes, kOddOff = 2 * NBUF * kTileBytes, kSmem = kOddOff + 16;
constexpr int kOutPitch = 272;                        // epilogue staging: one output row + 16 B, in bytes
static_assert(8 * WQ * kOutPitch <= kSmem, "epilogue staging reuses the tile rings");

__device__ __forceinline__ unsigned packed(bf16x2 v) { union { bf16x2 b; unsigned u; } c; c.b = v; return c.u; }
__device__ __forceinline__ u32x4 widen8(unsigned w0, unsigned w1, float scale) {      // eight e4m3 to bf16
    u32x4 r;
    r[0] = packed(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false));
    r[1] = packed(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true));
    r[2] = packed(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false));
    r[3] = packed(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true));
    return r;
}

__device__ __forceinline__ u32x4 widen8(unsigned w, float scale) {                    // eight e2m1 to bf16; a scale of 255 makes them NaN
    u32x4 r;
    r[0] = packed(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    r[1] = packed(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    r[2] = packed(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    r[3] = packed(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    return r;
}

// 4 bits: a thread has the four 16-byte pieces of a scale's 32 channels, and neighbouring threads those of the next, so that piece w of 32-channel block b lies at 4 w + b of its row and not at
// 4 b + w, swizzled by the row as below: eight lanes that write, two rows of four blocks, meet all 32 banks, and so do those that read (257 conflict cycles a step with the other
// kernels' order).
__device__ __forceinline__ unsigned k_turn(int row) { return (unsigned)((row & 1) << 2 | (row >> 1 & 3) | (row & 8)); }     // of row & 15
__device__ __forceinline__ unsigned v_turn(int row) { return (unsigned)(row | (row & 1) << 2); }                           // of row & 3

// All units of a workgroup's run, for waves 0-3 or (ROTATED, half a period behind) waves 4-7, each of which shares its SIMD with wave - 4.  The roles part here and not
// around their key loops: with both loops inside the one over the units the compiler spills 60 to 80 registers.  Both meet the same barriers.
// What is left of it: all forms keep 174 to 292 times a scalar in a lane of a vector register, and that over 8-bit pages of 16 one vector register in memory (8 bytes of scratch).
// RUNS: pages that a tile of 64 keys lies in: 1 (pages of 64 and more), 2 or 4 (of 16).  Four look-ups and what follows from them are 80 scalar instructions a step more than one:
// 8192 new tokens of 32768 (32/8 heads), pages of 64, 3571 us with four and 3310 with one.
template <int HELD, int RUNS, bool ROTATED>
__device__ __forceinline__ void work(const PagedArgs& a, Run<true, HELD == HELD_MXFP4>& run, unsigned home, unsigned lds0) {
    constexpr bool MX = HELD != HELD_PLAIN, MX4 = HELD == HELD_MXFP4;
    constexpr int kRowBytes = row_bytes(HELD, 2);                  // of 4 bits
    const float c = a.scale_log2e, lazy_raw = fminf(kLazyLog2 / c, 3e38f);      // not infinite, whatever the scale: no maximum would be taken over then
    if (thread_id() == 0) *LDS_PTR(unsigned, lds0 + kOddOff) = 0;
    __syncthreads();
    while (true) {
        // What follows from the thread's number is worked out for each unit: kept from one to the next it would be spilled, 60 registers of it.
        int tid = thread_id();
        asm volatile("" : "+v"(tid));
        const int lane = tid & 63, l32 = lane & 31, hh = lane >> 5, r4 = lane >> 4, pch = lane & 15;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        // ---- per-lane LDS addresses (bytes, ring slot 0), see attn_bf16.hip
        const unsigned k_base = (lds0 + kKOff + l32 * 256) | (MX4 ? (k_turn(l32 & 15) ^ (unsigned)hh << 2) << 4 : (unsigned)(((l32 & 15) ^ hh) << 4));
        const int i16 = lane & 15, gbit = (lane >> 4) & 1;
        unsigned v_addr[4];
    #pragma unroll
        for (int dt = 0; dt < 4; ++dt)
            v_addr[dt] = MX4 ? lds0 + kVOff + (4 * hh + (i16 >> 2)) * 256 + (((unsigned)(((2 * gbit + ((i16 & 3) >> 1)) << 2) + dt) ^ v_turn(i16 >> 2)) << 4) + (i16 & 1) * 8
                             : lds0 + kVOff + (4 * hh + (i16 >> 2)) * 256 + ((((unsigned)(dt ^ (i16 >> 2)) << 2) + 2 * gbit + ((i16 & 3) >> 1)) << 4) + (i16 & 1) * 8;
        // copies: wave w fills rows 4 w .. 4 w + 3 and 32 + 4 w .. of a tile; physical chunk pch of row r4
        const unsigned lane_k = (unsigned)r4 * 256 + (unsigned)(pch ^ ((4 * wave + r4) & 15)) * 16, lane_v = (unsigned)r4 * 256 + (unsigned)(pch ^ (4 * r4)) * 16;
        // 8 bits: thread tid has 16 channels 16 * (tid & 7) of row tid >> 3 of K and V.  4 bits: the 32 channels 32 * (tid & 3), those of a scale, of row tid / 4, of K (waves 0-3) or V (4-7).
        const int xrow = MX4 ? (tid & 255) >> 2 : tid >> 3, xpiece = MX4 ? tid & 3 : tid & 7;

        const Sequence seq = run.now;
        const int t0 = run.tile << a.tile_shift, live = min(1 << a.tile_shift, seq.tokens - t0), head = run.head;
        unsigned first, count, unit;
        run.piece(a, first, count, unit);
        const int ntiles = (int)count, base0 = (int)first * TK;
        const scalar_list table = (scalar_list)(unsigned long long)uniform_ptr(a.table + (int64_t)run.seq * a.max_pages);
        const int past = seq.keys - seq.tokens;
        const int high = min(past + t0 + live, seq.keys) - 1;        // the last key that any row sees
        const int rows_live = live * a.group;
        auto sees = [&](int r) { return min(past + t0 + (int)a.by_group.div((unsigned)min(r, rows_live - 1)), seq.keys - 1); };   // last key of row r
        const int qpos = sees(WQ * wave + l32);
        int wq_lo = sees(WQ * wave);
        asm("" : "+v"(wq_lo));                                       // a vector register, see attn_bf16.hip
        int wq_last = WQ * wave < rows_live ? sees(WQ * wave + WQ - 1) : -1;
        asm("" : "+v"(wq_last));

        // ---- Q as whole rows to LDS, where tiles 2 and 3 come later, and from there into registers
        const unsigned q_lds = lds0 + (wave < 4 ? kVOff : kKOff) + 2 * kTileBytes + (wave & 3) * (WQ * 256);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned r = (unsigned)min(WQ * wave + 4 * i + r4, rows_live - 1), t = a.by_group.div(r);
            const uint16_t* row = (const uint16_t*)a.q + (int64_t)(seq.start + t0 + (int)t) * a.qs0 + (int64_t)(head * a.group + (int)(r - t * a.group)) * a.qs1;
            dma16_far((const char*)row + (((unsigned)(pch ^ r4) << 4) ^ (64 * (i & 3))), q_lds + i * 1024);
        }

        // ---- pages: of tile x the entries of its runs of keys, and what follows from them
        constexpr int kRunKeys = TK / RUNS, kRunBits = (1 << (4 / RUNS)) - 1;
        const int mask = (1 << a.page_shift) - 1;
        int entry[RUNS];
        auto look_up = [&](int x) __attribute__((always_inline)) {
#pragma unroll
            for (int g = 0; g < RUNS; ++g)
                entry[g] = table[max(min(base0 + x * TK + kRunKeys * g, high), 0) >> a.page_shift];     // no branch; whether the key is there is asked in describe
        };
        int ok[4] = {0, 0, 0, 0};                                    // of tiles t .. t + 3: which runs of 16 keys are there, a bit each
        int64_t at[2], v_at[2];                                      // first rows of the wave's two loads of the tile described last; V is issued a step later
        auto describe = [&](int x) __attribute__((always_inline)) {  // from `entry`
            v_at[0] = at[0]; v_at[1] = at[1];
            ok[0] = ok[1]; ok[1] = ok[2]; ok[2] = ok[3]; ok[3] = 0;
            int page[RUNS];
#pragma unroll
            for (int g = 0; g < RUNS; ++g) {
                const bool there = (unsigned)entry[g] < (unsigned)a.n_pages && base0 + x * TK + kRunKeys * g <= high;
                ok[3] |= there ? kRunBits << (g * (4 / RUNS)) : 0;
                page[g] = there ? entry[g] : 0;                      // keys that are not there are read from page 0 and hidden
            }
            // the wave's rows: 4 * wave .. + 3 and 32 + 4 * wave .. + 3, or 8 * wave .. + 7
            if constexpr (MX4) {                                     // rows 16 * (wave & 3) .. + 15
                int p = page[0];
#pragma unroll
                for (int g = 1; g < RUNS; ++g) p = (wave & 3) / (4 / RUNS) == g ? page[g] : p;
                at[0] = (((int64_t)p * a.hkv + head) << a.page_shift) + ((base0 + x * TK + 16 * (wave & 3)) & mask);
            } else if (MX) {
                int p = page[0];
#pragma unroll
                for (int g = 1; g < RUNS; ++g) p = wave / (8 / RUNS) == g ? page[g] : p;
                at[0] = (((int64_t)p * a.hkv + head) << a.page_shift) + ((base0 + x * TK + 8 * wave) & mask);
            } else if (RUNS == 1) {
                at[0] = (((int64_t)page[0] * a.hkv + head) << a.page_shift) + ((base0 + x * TK) & mask) + 4 * wave;
                at[1] = at[0] + 32;
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int p = RUNS == 2 ? page[i % RUNS] : wave < 4 ? page[2 * i % RUNS] : page[(2 * i + 1) % RUNS];
                    at[i] = (((int64_t)p * a.hkv + head) << a.page_shift) + ((base0 + x * TK + 32 * i + 4 * wave) & mask);
                }
            }
        };
        auto base = [&](int x) { return base0 + x * TK; };
        int high_v = high;
        asm("" : "+v"(high_v));                                      // like wq_lo
        auto in_vector = [](int x) { asm("" : "+v"(x)); return x; };
        // Tiles with keys that some rows do not see, or none: a weight of 0 does not keep an infinity or NaN of theirs out of a sum.  As V of such a tile comes in, keys that
        // no row sees become 0, and so does what is not finite in those that some rows do not see; where there was any, `odd` in LDS is set and the unit's end adds it for the rows that see it.
        int low_v = min(past + t0, seq.keys - 1);                    // the last key that the first row sees
        asm("" : "+v"(low_v));
        auto partly = [&](int x, int bits) { return base(x) + TK - 1 > low_v || in_vector(bits) != 15; };
        auto clean = [&](u32x4 v, int key, bool there) __attribute__((always_inline)) -> u32x4 {
            there = there && key <= high_v;
            const unsigned all_see = key <= low_v ? ~0u : 0u;
            unsigned any = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned keep = ((v[e] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u) | ((v[e] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | all_see;
                any |= ~keep;
                v[e] = there ? v[e] & keep : 0u;
            }
            if (there && any) *LDS_PTR(unsigned, lds0 + kOddOff) = 1;
            return v;
        };
        auto issue_k = [&](int slot) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                dma16(uniform_ptr((const char*)a.cache.k + at[i] * 256), lane_k, lds0 + kKOff + slot * kTileBytes + (32 * i + 4 * wave) * 256);
        };
        auto issue_v = [&](int slot, bool now) {                     // now: of the tile described last (prologue), else of the one before
#pragma unroll
            for (int i = 0; i < 2; ++i)
                dma16(uniform_ptr((const char*)a.cache.v + (now ? at[i] : v_at[i]) * 256), lane_v, lds0 + kVOff + slot * kTileBytes + (32 * i + 4 * wave) * 256);
        };
        auto clean_v = [&](int x, int bits, int slot) {              // the lane's own pieces
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = 32 * i + 4 * wave + r4;
                const unsigned at = lds0 + kVOff + slot * kTileBytes + (32 * i + 4 * wave) * 256 + lane * 16;
                *LDS_PTR(u32x4, at) = clean(*LDS_PTR(const u32x4, at), base(x) + row, (bits >> (row >> 4)) & 1);
            }
        };
        // 8 and 4 bits: the tile in flight; of 4 bits K or V are in raw_k
        u32x4 raw_k, raw_v; unsigned scale_k = 0, scale_v = 0;
        auto load_raw = [&]() __attribute__((always_inline)) {       // of the tile described last
            if constexpr (MX4) {
                const char* from = uniform_ptr((const char*)(ROTATED ? a.cache.v : a.cache.k) + at[0] * kRowBytes);
                const unsigned in_rows = (unsigned)lane * 16;
                raw_k = *(const u32x4*)(from + in_rows);
                scale_k = (uniform_ptr((ROTATED ? a.cache.vs : a.cache.ks) + at[0] * 4))[(unsigned)lane];
                return;
            }
            const unsigned in_rows = (unsigned)lane * 16, in_scales = (unsigned)(lane >> 3) * 4 + (unsigned)((lane & 7) >> 1);   // eight rows of a wave
            raw_k = *(const u32x4*)(uniform_ptr((const char*)a.cache.k + at[0] * 128) + in_rows);
            raw_v = *(const u32x4*)(uniform_ptr((const char*)a.cache.v + at[0] * 128) + in_rows);
            scale_k = (uniform_ptr(a.cache.ks + at[0] * 4))[in_scales];
            scale_v = (uniform_ptr(a.cache.vs + at[0] * 4))[in_scales];
        };
        auto store_raw = [&](int x, int bits, int slot) __attribute__((always_inline)) {
            if constexpr (MX4) {
                const float scale = __uint_as_float(scale_k << 23);
                const unsigned to = lds0 + (ROTATED ? kVOff : kKOff) + slot * kTileBytes + xrow * 256 + (((unsigned)xpiece ^ (ROTATED ? v_turn(xrow & 3) : k_turn(xrow & 15))) << 4);
                const bool part = ROTATED && partly(x, bits), there = ROTATED && ((bits >> (xrow >> 4)) & 1);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    u32x4 v = widen8(raw_k[w], scale);
                    if (part) v = clean(v, base(x) + xrow, there);
                    *LDS_PTR(u32x4, to ^ (w << 6)) = v;
                }
                return;
            }
            const float sk = __uint_as_float(scale_k << 23), sv = __uint_as_float(scale_v << 23);
            const unsigned row = lds0 + slot * kTileBytes + xrow * 256;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *LDS_PTR(u32x4, row + kKOff + (((2 * xpiece + h) ^ (xrow & 15)) << 4)) = widen8(raw_k[2 * h], raw_k[2 * h + 1], sk);
            __builtin_amdgcn_sched_barrier(0);                       // registers of one at a time
            u32x4 v2[2] = {widen8(raw_v[0], raw_v[1], sv), widen8(raw_v[2], raw_v[3], sv)};
            if (partly(x, bits)) {
                const bool there = (bits >> (xrow >> 4)) & 1;
                v2[0] = clean(v2[0], base(x) + xrow, there); v2[1] = clean(v2[1], base(x) + xrow, there);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) *LDS_PTR(u32x4, row + kVOff + (((2 * xpiece + h) ^ (4 * (xrow & 3))) << 4)) = v2[h];
        };

        bf16x8 qf[8];
        f32x16 o[4];
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
        float m_run = -INFINITY, l_run = 0.f;

        // ---- the phases, see attn_bf16.hip
        unsigned ka[8], va[4];
        int ka_slot = 0, va_slot = 0;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) ka[ks] = k_base ^ (MX4 ? ((ks & 1) << 3 | ks >> 1) << 4 : ks << 5);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) va[dt] = v_addr[dt];
        auto next_k_slot = [&]() {
            const unsigned d = ka_slot == NBUF - 1 ? (unsigned)(-(NBUF - 1) * kTileBytes) : (unsigned)kTileBytes;
            ka_slot = (ka_slot + 1) & (NBUF - 1);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) ka[ks] += d;
        };
        auto next_v_slot = [&]() {
            const unsigned d = va_slot == NBUF - 1 ? (unsigned)(-(NBUF - 1) * kTileBytes) : (unsigned)kTileBytes;
            va_slot = (va_slot + 1) & (NBUF - 1);
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) va[dt] += d;
        };
        constexpr int kLook = 3;
        bf16x8 ring[kLook + 1];
        auto read_k = [&](int ks, int kt, bf16x8& f) { f = as_bf16x8(*LDS_PTR(const u32x4, ka[ks] + kt * 32 * 256)); };
        auto read_v = [&](int t4, int dt, bf16x8& f) {
            const unsigned ad = va[dt] + t4 * 16 * 256;
            const v4bf16_lds lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(LDS_PTR(v4bf16_lds, ad));
            const v4bf16_lds hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(LDS_PTR(v4bf16_lds, ad + 8 * 256));
#pragma unroll
            for (int e = 0; e < 4; ++e) { f[e] = lo[e]; f[4 + e] = hi[e]; }
        };
        // fragment j of a matrix phase.  kind 0: QK alone (16), 1: PV alone (16), 2: PV of one tile interleaved with QK of the next (32)
        auto frag_read = [&](int kind, int j, bf16x8& f) __attribute__((always_inline)) {
            if (kind == 0) read_k(j >> 1, j & 1, f);
            else if (kind == 1) read_v(j >> 2, j & 3, f);
            else if ((j & 7) < 4) read_v(j >> 3, j & 3, f);
            else read_k(2 * (j >> 3) + (((j & 7) - 4) >> 1), j & 1, f);
        };
        auto frag_mfma = [&](int kind, int j, const bf16x8& f, f32x16 (&s)[2], const bf16x8 (&pf)[4]) __attribute__((always_inline)) {
            const bool is_v = kind == 1 || (kind == 2 && (j & 7) < 4);
            if (is_v) {
                const int t4 = kind == 1 ? (j >> 2) : (j >> 3), dt = j & 3;
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, pf[t4], o[dt], 0, 0, 0);
            } else {
                const int ks = kind == 0 ? (j >> 1) : 2 * (j >> 3) + (((j & 7) - 4) >> 1), kt = j & 1;
                s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[ks], s[kt], 0, 0, 0);
            }
        };
        auto read_kg = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < kLook; ++j) frag_read(0, j, ring[j]);
        };
        auto read_vg = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < kLook; ++j) frag_read(1, j, ring[j]);
        };
        auto zero_s = [&](f32x16 (&s)[2]) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = 0.f;
        };
        auto run_frags = [&](int kind, f32x16 (&s)[2], const bf16x8 (&pf)[4]) __attribute__((always_inline)) {
            const int n = kind == 2 ? 32 : 16;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                if (j < n) {
                    if (j + kLook < n) frag_read(kind, j + kLook, ring[(j + kLook) % (kLook + 1)]);
                    frag_mfma(kind, j, ring[j % (kLook + 1)], s, pf);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        bf16x8 no_p[4];
        auto qk = [&](f32x16 (&s)[2]) __attribute__((always_inline)) { zero_s(s); run_frags(0, s, no_p); };
        auto pv = [&](const bf16x8 (&pf)[4]) __attribute__((always_inline)) { f32x16 no_s[2]; run_frags(1, no_s, pf); };
        auto mm_both = [&](f32x16 (&s)[2], const bf16x8 (&pf)[4]) __attribute__((always_inline)) { zero_s(s); run_frags(2, s, pf); };
        auto mask_if_needed = [&](f32x16 (&s)[2], int x, int bits) {
            if (base(x) + TK - 1 <= wq_lo && in_vector(bits) == 15) return;
            int lim = qpos - base(x) - 4 * hh;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int gg = 0; gg < 4; ++gg) {
                    int top = (bits >> (2 * kt + (gg >> 1))) & 1 ? lim : -1;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (32 * kt + 8 * gg + i > top) s[kt][4 * gg + i] = -INFINITY;
                        asm("" : "+v"(top));                         // or each comparison is built on the others
                    }
                }
        };
        auto sm = [&](f32x16 (&s)[2], bf16x8 (&pf)[4]) {
            float mx = fmaxf(s[0][0], s[0][1]), my = fmaxf(s[1][0], s[1][1]);
#pragma unroll
            for (int r = 2; r < 16; r += 2) {
                mx = fmaxf(fmaxf(s[0][r], s[0][r + 1]), mx);
                my = fmaxf(fmaxf(s[1][r], s[1][r + 1]), my);
            }
            mx = half_max(fmaxf(mx, my));
            const float m_new = (mx > m_run + lazy_raw) ? mx : m_run;
            const float m_safe = (m_new == -INFINITY) ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f((m_run - m_safe) * c);
            const float ms = m_safe * c;
            m_run = m_new;
            float rs0 = 0.f, rs1 = 0.f;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[kt][r], c, -ms));
                    if (r & 1) rs1 += p; else rs0 += p;
                    pf[2 * kt + (r >> 3)][r & 7] = (__bf16)p;         // off by 2^-8 of a term or less; in two pieces PV would take twice the matrix time
                }
            l_run = l_run * alpha + (rs0 + rs1);
            if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
                for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
            }
        };
        // end of step t: K of tile t + 2 and V of tile t + 1 have landed, then everybody is past its reads of tile t
        auto step_end = [&](int t, int issued) {
            const int bits = ok[1];                                  // of tile t + 1
            describe(t + 4);
            if (!MX) {
                if (issued == 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
                else if (issued == 2) asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
                else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                if (t + 1 < ntiles && partly(t + 1, bits)) clean_v(t + 1, bits, (t + 1) & 3);
            }
            __syncthreads();
        };
        // after the matrix phase of step t
        auto feed = [&](int t) __attribute__((always_inline)) -> int {
            if (MX) {
                if (t + 2 < ntiles) store_raw(t + 2, ok[2], (t + 2) & 3);
                if (t + 3 < ntiles) load_raw();
                return 0;
            }
            const int issued = t + 3 < ntiles ? 4 : (t + 2 < ntiles ? 2 : 0);
            if (issued >= 2) issue_v((t + 2) & 3, false);
            if (issued == 4) issue_k((t + 3) & 3);
            return issued;
        };

        // ---- prologue: the pages of tiles 0 to 3 are looked up at once; K and V of tiles 0 and 1 are asked for, then, when Q has left its place, K of tile 2
        // (8-bit: 0 and 1 are stored, 2 asked for)
        at[0] = at[1] = 0;
        int ahead[4][RUNS];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            look_up(x);
#pragma unroll
            for (int g = 0; g < RUNS; ++g) ahead[x][g] = entry[g];
        }
        auto describe_first = [&](int x) __attribute__((always_inline)) {
#pragma unroll
            for (int g = 0; g < RUNS; ++g) entry[g] = ahead[x][g];
            describe(x);
        };
        describe_first(0);
        const int bits0 = ok[3];
        if (MX) {
            load_raw();
            const u32x4 k0 = raw_k, v0 = raw_v;
            const unsigned sk0 = scale_k, sv0 = scale_v;
            describe_first(1);
            load_raw();
            const u32x4 k1 = raw_k, v1 = raw_v;
            const unsigned sk1 = scale_k, sv1 = scale_v;
            raw_k = k0; raw_v = v0; scale_k = sk0; scale_v = sv0;
            store_raw(0, bits0, 0);
            raw_k = k1; raw_v = v1; scale_k = sk1; scale_v = sv1;
            store_raw(1, ok[3], 1);
        } else {
            issue_k(0); issue_v(0, true);
            describe_first(1);
            issue_k(1); issue_v(1, true);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (!MX && partly(0, bits0)) clean_v(0, bits0, 0);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) qf[ks] = as_bf16x8(*LDS_PTR(const u32x4, q_lds + l32 * 256 + (((2 * ks + hh) ^ (l32 & 15)) << 4)));
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) pin(qf[ks]);
        __syncthreads();                                             // nobody reads Q in LDS any more
        describe_first(2);
        if (MX) { if (ntiles > 2) load_raw(); }
        else issue_k(2);
        describe_first(3);
        // now ok[0 .. 3] are of tiles 0 .. 3, at of tile 3, v_at of tile 2

        f32x16 s[2]; bf16x8 pf[4];
        auto tile_active = [&](int x) { return x < ntiles && base(x) <= wq_last; };
        if constexpr (!ROTATED) {
            // step t: ka points into the slot of K(t), va into the slot of V(t-1)
            bool have_p = false, act = tile_active(0);
            va_slot = NBUF - 1;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) va[dt] += (NBUF - 1) * kTileBytes;
            if (act) read_kg();
            for (int t = 0; t < ntiles; ++t) {
                look_up(t + 4);
                __builtin_amdgcn_s_setprio(3);
                if (have_p && act) mm_both(s, pf);
                else if (act) qk(s);
                else if (have_p) pv(pf);
                __builtin_amdgcn_s_setprio(0);
                const int issued = feed(t);
                next_k_slot(); next_v_slot();
                const bool act_next = act && tile_active(t + 1);
                if (act) {
                    read_vg();
                    mask_if_needed(s, t, ok[0]);
                    sm(s, pf);
                }
                have_p = act; act = act_next;
                step_end(t, issued);
            }
            if (have_p) pv(pf);
        } else {
            // step t: va points into the slot of V(t), ka into the slot of K(t+1)
            bool have_s = tile_active(0);
            if (have_s) { read_kg(); qk(s); }
            next_k_slot();
            for (int t = 0; t < ntiles; ++t) {
                look_up(t + 4);
                const bool act_next = have_s && tile_active(t + 1);
                if (have_s) {
                    read_vg();
                    mask_if_needed(s, t, ok[0]);
                    sm(s, pf);
                    __builtin_amdgcn_s_setprio(3);
                    if (act_next) mm_both(s, pf);
                    else pv(pf);
                    __builtin_amdgcn_s_setprio(0);
                }
                const int issued = feed(t);
                next_k_slot(); next_v_slot();
                have_s = act_next;
                step_end(t, issued);
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // no copy is in flight when the rings are written below

        // ---- epilogue
        const float l_tot = half_sum(l_run);
        const bool began = first == 0, ended = first + count == unit;
        __syncthreads();                                             // every wave is past its last tile reads
        if (__builtin_amdgcn_readfirstlane(*LDS_PTR(const int, lds0 + kOddOff))) {
            const int from = max(base0, __builtin_amdgcn_readfirstlane(low_v) + 1), to = min(high, base0 + ntiles * TK - 1);
            for (int u = from; u <= to; ++u) {                       // once in a blue moon: a key after another, from memory
                const int page = table[u >> a.page_shift];
                if ((unsigned)page >= (unsigned)a.n_pages) continue;
                const int64_t row = (((int64_t)page * a.hkv + head) << a.page_shift) + (u & mask);
#pragma unroll
                for (int j = 0; j < 16; ++j) {                       // channels 8 j + 4 hh ..
                    unsigned w[2];
                    if (MX4) w[0] = w[1] = a.cache.vs[row * 4 + (j >> 2)] >= kFarScale ? 0x7fc07fc0u : 0u;
                    else if (MX) {
                        const unsigned b = *(const unsigned*)((const char*)a.cache.v + row * 128 + 8 * j + 4 * hh);
                        const float scale = __uint_as_float((unsigned)a.cache.vs[row * 4 + (j >> 2)] << 23);
                        w[0] = packed(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false));
                        w[1] = packed(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true));
                    } else {
                        const uint2 b = *(const uint2*)((const char*)a.cache.v + row * 256 + 16 * j + 8 * hh);
                        w[0] = b.x; w[1] = b.y;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned b = e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16;
                        if (u <= qpos && (b & 0x7f800000u) == 0x7f800000u) o[j >> 2][4 * (j & 3) + e] += __uint_as_float(b);
                    }
                }
            }
            __syncthreads();                                         // all have seen the flag
            if (thread_id() == 0) *LDS_PTR(unsigned, lds0 + kOddOff) = 0;
        }
        if (began && ended) {                                        // O^T / l through LDS, so that stores are whole rows
            const float inv = l_tot == 0.f ? 0.f : 1.0f / l_tot;
            const unsigned stage = lds0 + wave * (WQ * kOutPitch);
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int gg = 0; gg < 4; ++gg) {
                    bf16x4 w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = (__bf16)(o[dt][4 * gg + i] * inv);
                    *LDS_PTR(bf16x4, stage + l32 * kOutPitch + (32 * dt + 8 * gg + 4 * hh) * 2) = w;
                }
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const unsigned r = WQ * wave + 4 * x + r4, t = a.by_group.div(r);
                const u32x4 val = *LDS_PTR(const u32x4, stage + (4 * x + r4) * kOutPitch + pch * 16);
                if ((int)r < rows_live)
                    *(u32x4*)((uint16_t*)a.out + (int64_t)(seq.start + t0 + (int)t) * a.os0 + (int64_t)(head * a.group + (int)(r - t * a.group)) * a.os1 + pch * 8) = val;
            }
            const unsigned r = WQ * wave + l32, t = a.by_group.div(r);
            if (a.lse && hh == 0 && (int)r < rows_live)
                a.lse[(int64_t)(seq.start + t0 + (int)t) * a.hq + head * a.group + (int)(r - t * a.group)] = l_tot == 0.f ? -INFINITY : m_run * a.scale + logf(l_tot);
        } else {                                                     // [wave][dt][gg][lane] of 16 bytes: whole kilobytes
            const int64_t slot = 2 * (int64_t)home + (began ? 1 : 0);
            float* to = a.parts + slot * kChunkRows * kHeadDim + wave * (WQ * kHeadDim) + lane * 4;
            if (WQ * wave < rows_live) {
#pragma unroll
                for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                    for (int gg = 0; gg < 4; ++gg) {
                        u32x4 w;
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(o[dt][4 * gg + i]);
                        *(u32x4*)(to + (4 * dt + gg) * 256) = w;
                    }
            }
            if (hh == 0) {
                float* ml = a.stats + 2 * (slot * kChunkRows + WQ * wave + l32);
                ml[0] = m_run; ml[1] = l_tot;
            }
            if (began && tid == 0) {
                const unsigned rest = unit - first - count;
                int32_t* rec = a.record + 4 + 4 * home;
                rec[0] = seq.start + t0; rec[1] = live; rec[2] = head; rec[3] = 1 + (int)((rest + run.share - 1) / run.share);
            }
        }
        if (!run.next_steps(a)) break;
        __syncthreads();                                             // the staging has been read
    }
}

template <int HELD, int RUNS>
__global__ __launch_bounds__(512, 1) void paged_chunk_kernel(PagedArgs a) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    Run<true, HELD == HELD_MXFP4> run;
    const bool any = run.find(a, workgroup_id(), thread_id() & 63);
    if (workgroup_id() == 0 && thread_id() == 0) a.record[0] = run.whole ? 0 : (int)run.used;   // whole: nothing to join
    if (run.logical < run.used && thread_id() == 0) a.record[4 + 4 * run.logical + 3] = 0;
    if (!any) return;
    const unsigned home = run.logical;
    if (__builtin_amdgcn_readfirstlane(thread_id() >> 6) < 4) work<HELD, RUNS, false>(a, run, home, lds0);
    else work<HELD, RUNS, true>(a, run, home, lds0);
}

template <int HELD, int RUNS>
hipError_t launch(const PagedArgs& a, int rows, hipStream_t st) {
    const hipError_t e = hipFuncSetAttribute((const void*)paged_chunk_kernel<HELD, RUNS>, hipFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((paged_chunk_kernel<HELD, RUNS>), dim3(a.workgroups), dim3(512), kSmem, st, a);
    if (a.whole) return hipGetLastError();
    // A workgroup of the join takes half of the channels of 32 rows, or where these are fewer workgroups than the chip has compute units a sixteenth, its waves every fourth part;
    // more rows than were said come in turn.  us of the whole call, half / sixteenth (bf16, pages of 64): 32 workgroups of the first kind (4/1 heads, 1 x 64 tokens of 20000) 47.5 / 26.6,
    // 48 (32/8, 1 x 20 of 100000) 89.6 / 86.9, 64 (8/2, 1 x 64 of 16000) 44.4 / 29.2, 128 (32/8, 30 of 40000 and 20 of 9000) 53.5 / 52.3, 160 (8/2, 1 x 256 of 9000) 31.7 / 31.3,
    // (8/1, 1 x 300 of 20000) 45.5 / 45.8, 192 (32/4, 1 x 64 of 30000) 51.0 / 50.3, 256 (32/8, 1 x 64 of 16000) 37.9 / 39.0, 640 (32/8, 1 x 256 of 16000) 80.9 / 86.8.
    const unsigned pieces = ((unsigned)rows + 31) / 32;
    if (2 * pieces * a.cut_units < 256) hipLaunchKernelGGL((join_kernel<__bf16, true, 4>), dim3(a.cut_units, 16 * pieces), dim3(256), 0, st, a, kChunkRows, 16 * pieces);
    else hipLaunchKernelGGL((join_kernel<__bf16, true, 1>), dim3(a.cut_units, 2 * pieces), dim3(256), 0, st, a, kChunkRows, 2 * pieces);
    return hipGetLastError();
}

template <int HELD>
hipError_t launch_runs(int runs, const PagedArgs& a, int rows, hipStream_t st) {
    return runs == 1 ? launch<HELD, 1>(a, rows, st) : runs == 2 ? launch<HELD, 2>(a, rows, st) : launch<HELD, 4>(a, rows, st);
}

}  // namespace

hipError_t launch_paged_chunk(const CacheShape& sh, const PagedArgs& a, hipStream_t st) {
    const int rows = std::min(sh.max_q, 1 << a.tile_shift) * sh.group;       // of a tile, as far as is known
    const int runs = sh.page_shift >= 6 ? 1 : sh.page_shift == 5 ? 2 : 4;
    return sh.held == HELD_MXFP4 ? launch_runs<HELD_MXFP4>(runs, a, rows, st) : sh.held == HELD_MXFP8 ? launch_runs<HELD_MXFP8>(runs, a, rows, st) : launch_runs<HELD_PLAIN>(runs, a, rows, st);
}

}  // namespace cp
