// Attention of the new tokens of each sequence over pages of 4 bits, for few rows a KV head and for fp32: the formulas, tiles and operand layouts of attn_paged.hip (S^T = K . Q^T and
// O^T += V^T . P^T in 16x16 MFMAs, waves split the keys, nothing but fp32 queries by way of LDS before the merge), with a key loop for half of the 8-bit bytes.
//
//   K   a lane takes one key's 32 channels of one scale, 16 bytes, and makes them bf16 (exact) by 16 conversions that apply the scale
//   V   a lane takes 8 channels of 8 tokens, 4 bytes each; 32 conversions, and 32 v_perm that bring two tokens' together
//   e2m1 has no infinity or NaN: what may become one is seen in the scales alone, and a key that no row sees needs no zeros in place of its V
//   fp32: Q and P as three bf16 pieces of 8 bits, exactly from 2^-110 on (split8), so that a product is three bf16 MFMAs where one in fp32 takes the time of 16, with sums in fp32 as there
//
// A step's loads are half as many bytes as over 8-bit pages for as much work, so what a wave waits for counts: K of the next step is asked for when QK has read this one's, V when
// PV has, and neither by a branch.  Where the loads stand behind a branch the compiler has to wait for all of them at the first use of any (one token of 10^6 keys 203 us, 64 of 8000 108; without
// 195 and 103, past the caches 170 and 91, and with whole lines of V in an instruction 165 and 88).  Not kept: two steps at a time (64 single tokens of all lengths up to 32769: 90 us for 72, units are short), three workgroups to a
// compute unit (64 of 8000: 101 us for 91), K and V two steps ahead in registers of their own (fp32: 20 x 200 after 8000 249 us for 232, 8 x 1 of 20000 21.1 for 18.8),
// the merge's rows that are not there left out (no difference), waves that go on to the next unit without a barrier while the last of the four adds up (64 of up to 32769 67.6 us for 59.7), K as 4-bit operand of a scaled MFMA with Q in two e4m3 pieces (its sums are good to 2^-17 of their terms only).
// Scalars do not fit: every form keeps 22 to 82 of them in lanes of vector registers.  In bf16 with 16 rows a step that asks for another of its unit reads none of them, the last of a unit, which asks for the next unit's, 43
// for pages of 16 and 2 for larger ones.  No vector register is spilled.
// fp32 with its own MFMAs, 4/2 heads: 3 x up to 200 tokens after 3000 34.5 us, with pieces 20.9; 20 x 200 after 8000 682 and 256; 8/2 heads: 8 x 1 of 20000 37.0 and 19.5.
#include "paged.h"

#include <type_traits>

namespace cp {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
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
// of the four neighbouring lanes that share c16 >> 2 the I-th's
template <int I> __device__ __forceinline__ unsigned quad_lane(unsigned x) { return (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x55 * I, 0xf, 0xf, true); }
// eight neighbouring e2m1 to bf16
__device__ __forceinline__ u32x4 widen8(unsigned w, float scale) {
    return u32x4{as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)), as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                 as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)), as_u32(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}
// Eight fp32 as sums of three bf16 each: 8 of the 24 bits to a piece, cut off and not rounded, so that the largest stay finite.  Exact from 2^-110 on; of a smaller number what lies below
// bf16's last bit, 2^-133, is lost.  A logit is then off by 2^-133 sum_c |k_c| scale at most, which keys above 2^100
// alone make felt, and an output, whose largest weight is 1 or more, by 2^-133 sum_u |v_u|: values above 2^100 whose weights are next to nothing.
__device__ __forceinline__ void split8(f32x4 lo, f32x4 hi, bf16x8* piece) {
    u32x4 w[3];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float x = e < 2 ? lo[2 * e] : hi[2 * e - 4], y = e < 2 ? lo[2 * e + 1] : hi[2 * e - 3];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const unsigned p = __float_as_uint(x), q = __float_as_uint(y);
            w[i][e] = __builtin_amdgcn_perm(q, p, 0x07060302u);
            x -= __uint_as_float(p & 0xffff0000u); y -= __uint_as_float(q & 0xffff0000u);
        }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) piece[i] = as_bf16x8(w[i]);
}
// Elements go past the caches: where a sequence's new tokens fit a tile a call reads them once.  us, ordinary loads / past the caches (32/8 heads, pages of 64, caches that no other call has left in the
// chip): one token of 8000 keys 12.5 / 11.4, of 131072 34.6 / 31.2, of 10^6 194.9 / 170.0; 8 of 2000 15.1 / 14.1, 64 of 8000 102.6 / 91.5.  Sequences of several tiles, which read them again for each, take these loads too
// though ordinary ones are faster there: 8 x 16 tokens of 16000 60.7 / 64.0, 1 x 64 of 16000 37.4 / 39.1, 1 x 32 of 60000 56.7 / 61.8, 32 x 16 of 4000 59.8 / 60.4; fp32, 4/2 heads 3 x 200 of 3200 27.2 / 27.4, 20 x 200 of
// 8200 228 / 249, 32/8 heads 10 x 100 of 20000 1012 / 1156.  Scales, 16 tokens' to 64 bytes, by ordinary loads.
template <typename V>
__device__ __forceinline__ V get(const char* p) { return __builtin_nontemporal_load((const V*)p); }

constexpr int kWaveKeys = 32;                 // of a step, to each wave

typedef Run<false, true> Share;

// One unit, or the piece of it that lies in a workgroup's run.  All the same for a workgroup.
struct Unit {
    int seq, head, row, live;                 // row: its first token's, live: its tokens
    int keys, past, low, high;                // of the sequence; position of the unit's first token; last keys that its first and its last row see
    unsigned first, count, steps;             // steps first .. first + count - 1 of `steps`
    // the first key of a wave's r-th 16 (of pages of 16), in step x of the piece
    __device__ __forceinline__ int key(const PagedArgs& a, unsigned x, int wave, int r) const { return (int)((first + x) << a.step_shift) + wave * kWaveKeys + 16 * r; }
};
__device__ __forceinline__ Unit unit_of(const PagedArgs& a, const Share& run) {
    Unit n;
    const int t0 = run.tile << a.tile_shift;
    n.seq = run.seq; n.head = run.head; n.row = run.now.start + t0; n.live = min(1 << a.tile_shift, run.now.tokens - t0);
    n.keys = run.now.keys; n.past = run.now.keys - run.now.tokens + t0;
    n.low = min(n.past, n.keys - 1); n.high = min(n.past + n.live, n.keys) - 1;
    run.piece(a, n.first, n.count, n.steps);
    return n;
}
// Head and tile of step `rest` of a sequence.
__device__ __forceinline__ bool place_in(const PagedArgs& a, Share& run, unsigned rest) {
    run.head = first_lane((int)(rest / run.now.length));
    rest -= (unsigned)run.head * run.now.length;
    int lo = 0, hi = run.now.tiles - 1;                                        // the last tile that begins at or before it
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (run.now.before(a, mid, run.whole) <= rest) lo = mid; else hi = mid - 1;
    }
    run.tile = lo;
    run.at = rest - run.now.before(a, lo, run.whole);
    return run.has_steps(a);
}
// Run::find for a single sequence, whose arrays all lanes share: without the sums over lanes, and by scalar loads (one token of 300 keys, in a graph, 6.4 us, now 5.6; of 2000 8.8 and 8.1).
__device__ __forceinline__ bool find_one(const PagedArgs& a, Share& run, unsigned workgroup) {
    run.whole = a.whole; run.logical = ~0u; run.used = run.left = 0; run.seq = run.head = run.tile = 0; run.at = 0;
    const bool ascends = run.now.load_uniform<true>(a, 0, run.whole);
    const unsigned total = run.now.length * (unsigned)a.hkv;
    if (!ascends || total == 0) return false;
    run.share = max(run.whole ? 1u : a.least, (total + a.workgroups - 1) / a.workgroups);
    run.used = (total + run.share - 1) / run.share;
    const unsigned logical = (workgroup & 7) * ((run.used + 7) / 8) + (workgroup >> 3);
    if ((workgroup >> 3) >= (run.used + 7) / 8 || logical >= run.used) return false;
    run.logical = logical;
    run.left = min(run.share, total - logical * run.share);
    return place_in(a, run, logical * run.share);
}
// Run::find for 65 to 4096 sequences: the waves sum up 64 of them in turn, and look into those alone where the run begins.  us, with Run::find and so, 32/8 heads in a graph: 128 x 1 of 8000 keys 176.2 /
// 175.4, 256 of 4000 182.3 / 180.2, 512 of 2100 202.1 / 198.7, of up to 4000 82.7 / 77.3.
constexpr int kMany = 64 * 64;
__device__ __forceinline__ unsigned up_to(unsigned x, int lane) {              // of all lanes before and its own
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const unsigned o = __shfl_up(x, d); if (lane >= d) x += o; }
    return x;
}
__device__ __forceinline__ bool find_many(const PagedArgs& a, Share& run, unsigned workgroup, int lane, int wave, unsigned* shared) {
    run.whole = a.whole; run.logical = ~0u; run.used = run.left = 0; run.seq = run.head = run.tile = 0; run.at = 0; run.now = Sequence{};
    const int groups = (a.n_seqs + 63) >> 6;
    unsigned long long wrong = 0;
    Sequence s;
    auto load = [&](int g) __attribute__((always_inline)) {
        wrong |= __builtin_amdgcn_ballot_w64(!s.load<true>(a, min(64 * g + lane, a.n_seqs - 1), run.whole));
        return 64 * g + lane < a.n_seqs ? s.length * (unsigned)a.hkv : 0u;
    };
    for (int g = wave; g < groups; g += 4) {
        unsigned sum = load(g);
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        if (lane == 0) shared[g] = sum;
    }
    if (lane == 0) shared[64 + wave] = wrong != 0;
    __syncthreads();
    const unsigned of = lane < groups ? shared[lane] : 0u, upto = up_to(of, lane);
    const unsigned total = (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
    if (first_lane((int)(shared[64] | shared[65] | shared[66] | shared[67])) || total == 0) return false;
    run.share = max(run.whole ? 1u : a.least, (unsigned)first_lane((int)((total + a.workgroups - 1) / a.workgroups)));
    run.used = (unsigned)first_lane((int)((total + run.share - 1) / run.share));
    const unsigned logical = (workgroup & 7) * ((run.used + 7) / 8) + (workgroup >> 3);
    if ((workgroup >> 3) >= (run.used + 7) / 8 || logical >= run.used) return false;
    run.logical = logical;
    const unsigned begin = logical * run.share;
    run.left = min(run.share, total - begin);
    const int g = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > begin));
    const unsigned past = (unsigned)__builtin_amdgcn_readlane((int)(upto - of), g), mine = load(g), within = up_to(mine, lane);
    const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(past + within > begin));
    unsigned rest = begin - past - (unsigned)__builtin_amdgcn_readlane((int)(within - mine), l);
    run.seq = 64 * g + l;
    run.now = s.of_lane(l);
    return place_in(a, run, rest);
}
// Run::next_steps with scalar loads: a vector load's wait would be one for all keys and values that are under way.
__device__ __forceinline__ bool next_unit(const PagedArgs& a, Share& run) {
    const unsigned rest = run.whole ? 1u : a.setup + run.now.steps_of(a, run.tile) - run.at;
    if (run.left <= rest) return false;
    run.left -= rest;
    run.at = 0;
    if (++run.tile == run.now.tiles) {
        run.tile = 0;
        if (++run.head == a.hkv) {
            run.head = 0;
            do {
                if (++run.seq >= a.n_seqs) return false;
                run.now.load_uniform<true>(a, run.seq, run.whole);
            } while (run.now.tiles == 0);
        }
    }
    return run.has_steps(a);
}

enum { NOTHING = 0, SAME_UNIT = 1, NEXT_UNIT = 2 };

// SMALL: pages of 16 tokens, of which a wave's keys of a step lie in two.
template <typename T, int NQ, bool SMALL>
__global__ __launch_bounds__(kThreads, NQ == 1 || sizeof(T) == 2 ? 2 : 1) void paged_fp4_kernel(PagedArgs a) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int kPieces = F32 ? 3 : 1;
    constexpr int kRows = 16 * NQ, kGroups = kWaveKeys / 16, RUNS = SMALL ? 2 : 1, kRunGroups = kGroups / RUNS;
    extern __shared__ __attribute__((aligned(16))) float merge[];              // [wave][row][128], then (max, sum) [wave][row]
    float* const wave_stats = merge + 4 * kRows * kHeadDim;

    const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, kg = lane >> 4;
    const int wave = first_lane(tid >> 6);
    Share run;
    const bool any = a.n_seqs == 1 ? find_one(a, run, blockIdx.x)
                   : a.n_seqs > 64 && a.n_seqs <= kMany ? find_many(a, run, blockIdx.x, lane, wave, (unsigned*)merge) : run.find(a, blockIdx.x, lane);
    if (blockIdx.x == 0 && tid == 0) a.record[0] = (int)run.used;
    if (run.logical < run.used && tid == 0) a.record[4 + 4 * run.logical + 3] = 0;
    if (!any) return;
    const unsigned home = run.logical;
    const float c = a.scale_log2e, lazy_raw = fminf(kLazyLog2 / c, 3e38f);      // not infinite, whatever the scale: no maximum would be taken over then
    const int page_mask = (1 << a.page_shift) - 1;
    // An operand's row 4 a + b is key a + 4 b of its 16, so that the accumulators of S^T, four rows to a lane, hold keys kg + 4 i, and a load instruction of V has four neighbouring tokens, two
    // whole lines, where keys 4 kg + i make it half of four.  Scales of V: a lane asks for the word of one of its four tokens and has the others from its neighbours.  us, keys 4 kg + i with a
    // lane's four words in one load / so, 32/8 heads in a graph: one token of 10^6 170.8 / 165.2, 64 of up to 32769 60.9 / 58.9, 16 of 20000 (pages of 16) 63.8 / 60.8, 8 x 4 of 16000 31.7 / 30.9.
    const unsigned of_row = (unsigned)(c16 >> 2 | (c16 & 3) << 2);
    const unsigned in_k = of_row * 64 + (unsigned)kg * 16, in_v = (unsigned)kg * 64 + (unsigned)c16 * 4, in_ks = of_row * 4, in_vs = (unsigned)(kg + 4 * (c16 & 3)) * 4;
    // rotations to the right that bring a block's byte to the exponent's bits: the lane's 32 channels of K, its 8 of V.  What else is in the word is not looked at.
    const unsigned turn_k = 8u * (unsigned)kg + 9, turn_v = 8u * ((unsigned)c16 >> 2) + 9;

    // ---- the step that is looked up, the one that is asked for, and the one that is worked on, each ahead of the other, across the ends of units
    int entry[RUNS];
    auto look_up = [&](const Unit& n, unsigned x) __attribute__((always_inline)) {
        const scalar_list table = (scalar_list)(unsigned long long)(a.table + (int64_t)n.seq * a.max_pages);
#pragma unroll
        for (int r = 0; r < RUNS; ++r) entry[r] = table[max(min(n.key(a, x, wave, r), n.high), 0) >> a.page_shift];    // no branch; whether the keys are there is asked in load_k
    };
    int seen[RUNS], seen_next[RUNS];                                           // keys of a run that exist, of this step and the next
    int64_t at[RUNS];                                                          // first row of the runs asked for last
    u32x4 rk[kGroups]; unsigned rks[kGroups], rv[4 * kGroups], rvs[kGroups];
    auto load_k = [&](const Unit& n, unsigned x) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < RUNS; ++r) {                                       // a page that is not in the pool holds nothing: its keys are hidden, and read from page 0
            const int u = n.key(a, x, wave, r);
            const bool there = (unsigned)entry[r] < (unsigned)a.n_pages && u <= n.high;
            seen_next[r] = there ? n.keys - u : 0;
            at[r] = (((int64_t)(there ? entry[r] : 0) * a.hkv + n.head) << a.page_shift) + (u & page_mask);
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int r = g / kRunGroups, more = g % kRunGroups;
            rk[g] = get<u32x4>((const char*)a.cache.k + at[r] * 64 + 1024 * more + in_k);
            rks[g] = *(const unsigned*)((const char*)a.cache.ks + at[r] * 4 + 64 * more + in_ks);             // of a token
        }
    };
    auto load_v = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int r = g / kRunGroups, more = g % kRunGroups;
#pragma unroll
            for (int i = 0; i < 4; ++i) rv[4 * g + i] = get<unsigned>((const char*)a.cache.v + at[r] * 64 + 1024 * more + 256 * i + in_v);
            rvs[g] = *(const unsigned*)(a.cache.vs + at[r] * 4 + 64 * more + in_vs);
        }
    };
    // Lane's column is a row, 8 channels at 32 kg + 8 ks: of bf16 in registers; the pieces of fp32, three times as many, in LDS, once for the four waves, where the merge comes later.
    bf16x8 qf[NQ][F32 ? 1 : 4];
    bf16x8* const q_pieces = (bf16x8*)merge + lane;                            // [nq][ks][piece][lane]
    auto q_part = [&](const Unit& n, int nq, int ks) __attribute__((always_inline)) {
        const int r = 16 * nq + c16, of = (int)a.by_group.div((unsigned)r), t = min(of, n.live - 1), g = r - of * a.group;
        return (const T*)a.q + (int64_t)(n.row + t) * a.qs0 + (int64_t)(n.head * a.group + g) * a.qs1 + 32 * kg + 8 * ks;
    };
    f32x4 q_raw[F32 ? NQ : 1][2];
    auto load_q = [&](const Unit& n) __attribute__((always_inline)) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            if constexpr (F32) {                                               // a quarter of the channels to a wave
                const T* from = q_part(n, nq, wave);
                q_raw[nq][0] = *(const f32x4*)from; q_raw[nq][1] = *(const f32x4*)(from + 4);
            } else {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) qf[nq][ks] = *(const bf16x8*)q_part(n, nq, ks);
            }
        }
    };
    auto place_q = [&]() __attribute__((always_inline)) {
        if constexpr (F32) {
            __syncthreads();                                                   // the unit before has been read
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) {
                bf16x8 piece[3];
                split8(q_raw[nq][0], q_raw[nq][1], piece);
#pragma unroll
                for (int i = 0; i < 3; ++i) q_pieces[((nq * 4 + wave) * 3 + i) * 64] = piece[i];
            }
            __syncthreads();
        }
    };
    auto begin = [&](const Unit& n) __attribute__((always_inline)) {
        look_up(n, 0);
        load_q(n);
        __builtin_amdgcn_sched_barrier(0);                                     // in the loop's order, or its waits are for what is older in either
        load_k(n, 0);
        __builtin_amdgcn_sched_barrier(0);
        load_v();
        __builtin_amdgcn_sched_barrier(0);
        place_q();
        look_up(n, 1);
    };
    // The first step of the next unit is asked for in this one's last: what a unit begins and ends with, some 3 us, passes meanwhile (64 single tokens of up to 32769 keys 73.7 us without and 66.9 with it, before other steps that brought them to 59).
    // With 32 rows there are no registers for it, and with fp32 the queries' place is the merge's (with a place of their own: 20 x 200 after 8000 1 % faster, 3 x 200 after 3000 2 % slower).
    constexpr bool kAcross = NQ == 1 && !F32;
    Unit now = unit_of(a, run);
    begin(now);

    while (true) {
        const bool another = kAcross && next_unit(a, run);
        const Unit then = another ? unit_of(a, run) : now;
        if (another && now.count == 1) look_up(then, 0);
        const int high = now.high, low = now.low;
        int last[NQ];                                                          // the last key that the row sees
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) last[nq] = min(now.past + min((int)a.by_group.div((unsigned)(16 * nq + c16)), now.live - 1), now.keys - 1);

        f32x4 o[NQ][8];
        float m_run[NQ], l_run[NQ];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            m_run[nq] = -INFINITY; l_run[nq] = 0.f;
#pragma unroll
            for (int n = 0; n < 8; ++n) o[nq][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        bool odd = false;

        // What is asked for: the next step, that of another unit with its queries, or nothing.  Each has code of its own: where a wave asks by a branch it can only wait for all.
        auto work = [&](unsigned x, auto asks) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < RUNS; ++r) seen[r] = seen_next[r];
            f32x4 s[NQ][kGroups];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const float scale = __uint_as_float(__builtin_amdgcn_alignbit(rks[g], rks[g], turn_k));
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq) s[nq][g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) {
                    const bf16x8 kw = as_bf16x8(widen8(rk[g][ks], scale));
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                        for (int i = kPieces - 1; i >= 0; --i) {
                            const bf16x8 q = F32 ? q_pieces[((nq * 4 + ks) * 3 + i) * 64] : qf[nq][F32 ? 0 : ks];
                            s[nq][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kw, q, s[nq][g], 0, 0, 0);
                        }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (asks.value == SAME_UNIT) load_k(now, x + 1);
            if constexpr (asks.value == NEXT_UNIT) { load_q(then); load_k(then, 0); }
            __builtin_amdgcn_sched_barrier(0);
            // Hidden keys: behind the row's own, or without a page.
            bool whole = now.key(a, x, wave, RUNS - 1) + 16 * kRunGroups - 1 <= low;
#pragma unroll
            for (int r = 0; r < RUNS; ++r) whole = whole && seen[r] > 0;
            if (!whole) {
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    const int r = g / kRunGroups, u = now.key(a, x, wave, r) + 16 * (g % kRunGroups) + kg;
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq) {
                        const int lim = seen[r] > 0 ? last[nq] - u : -1;
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[nq][g][i] = 4 * i > lim ? -INFINITY : s[nq][g][i];
                    }
                }
            }
            bf16x8 pf[NQ][kPieces];
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) {
                float mx = -INFINITY;
#pragma unroll
                for (int g = 0; g < kGroups; ++g) mx = fmaxf(fmaxf(fmaxf(s[nq][g][0], s[nq][g][1]), fmaxf(s[nq][g][2], s[nq][g][3])), mx);
                mx = column_max(mx);
                // the reference point moves only when the maximum has outgrown it by 2^kLazyLog2: P <= 2^8 meanwhile, the same factor in O and l
                const float m_new = mx > m_run[nq] + lazy_raw ? mx : m_run[nq];
                const float m_safe = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = __builtin_amdgcn_exp2f((m_run[nq] - m_safe) * c);
                const float ms = m_safe * c;
                m_run[nq] = m_new;
                float sum = 0.f;
                f32x4 p4[kGroups];
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(s[nq][g][i], c, -ms));
                        sum += p;                                              // before P is rounded for the product: lse is as exact as fp32 allows
                        if constexpr (F32) p4[g][i] = p;
                        else pf[nq][0][4 * g + i] = (__bf16)p;                 // off by 2^-8 of a term or less; out's error against 64 bits stays that of its own rounding, 0.0015 to 0.0017 of its size
                    }
                if constexpr (F32) split8(p4[0], p4[1], pf[nq]);
                l_run[nq] = l_run[nq] * alpha + sum;
                if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
                    for (int n = 0; n < 8; ++n) o[nq][n] *= alpha;
                }
            }
            // A weight of 0 keeps everything of a hidden key out of a sum but what is not finite, which only scales from 253 on can bring (4 * 2^126 is infinite): they become others there.
            // `odd` says that some rows see such a key and others do not; the unit's end makes it NaN for those that do.
            unsigned scales[kGroups][4];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const unsigned turned = __builtin_amdgcn_alignbit(rvs[g], rvs[g], turn_v);
                scales[g][0] = quad_lane<0>(turned); scales[g][1] = quad_lane<1>(turned); scales[g][2] = quad_lane<2>(turned); scales[g][3] = quad_lane<3>(turned);
            }
            if (!whole) {
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    const int r = g / kRunGroups, u = now.key(a, x, wave, r) + 16 * (g % kRunGroups) + kg;
                    const int lim = seen[r] > 0 ? high - u : -1, sure = seen[r] > 0 ? low - u : -1;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool far = (scales[g][i] & 0x7f800000u) >= kFarScale << 23;
                        if (4 * i > sure && far) { scales[g][i] = 0x3f800000u; if (4 * i <= lim) odd = true; }
                    }
                }
            }
            u32x4 v[8];                                                        // [token][two channels a word]
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = widen8(rv[j], __uint_as_float(scales[j >> 2][j & 3]));
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                u32x4 w;                                                       // channel n of the lane's 8 tokens
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_perm(v[2 * e + 1][n >> 1], v[2 * e][n >> 1], n & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                    for (int x = kPieces - 1; x >= 0; --x) o[nq][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), pf[nq][x], o[nq][n], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (asks.value != NOTHING) load_v();
            if constexpr (asks.value == SAME_UNIT) { if (kAcross && x + 2 >= now.count) look_up(then, 0); else look_up(now, x + 2); }
            if constexpr (asks.value == NEXT_UNIT) look_up(then, 1);
        };
        for (unsigned x = 0; x + 1 < now.count; ++x) work(x, std::integral_constant<int, SAME_UNIT>());
        if constexpr (kAcross) {
            if (another) work(now.count - 1, std::integral_constant<int, NEXT_UNIT>());
            else work(now.count - 1, std::integral_constant<int, NOTHING>());
        } else work(now.count - 1, std::integral_constant<int, NOTHING>());

        if (__builtin_amdgcn_ballot_w64(odd) != 0) {
            const scalar_list table = (scalar_list)(unsigned long long)(a.table + (int64_t)now.seq * a.max_pages);
            for (unsigned x = 0; x < now.count; ++x)
                for (int i = 0; i < kWaveKeys; ++i) {                          // once in a blue moon: a key after another, from memory
                    const int u = now.key(a, x, wave, 0) + i;
                    if (u <= low || u > high) continue;
                    const int page = table[u >> a.page_shift];
                    if ((unsigned)page >= (unsigned)a.n_pages) continue;
                    const int64_t row = (((int64_t)page * a.hkv + now.head) << a.page_shift) + (u & page_mask);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {                              // channels 32 kg + 8 e ..
                        if (a.cache.vs[row * 4 + kg] < kFarScale) continue;
#pragma unroll
                        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                            for (int n = 0; n < 8; ++n)
                                if (u <= last[nq]) o[nq][n][e] = NAN;
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
                for (int half = 0; half < 2; ++half) {                         // channels 8 (4 kg + i) + 4 half ..
                    const int piece = 2 * (4 * kg + i) + half;
                    f32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = o[nq][4 * half + e][i];
                    *(f32x4*)(merge + (wave * kRows + r) * kHeadDim + 4 * (piece ^ c16)) = w;
                }
        }
        __syncthreads();
        const bool began = now.first == 0, ended = now.first + now.count == now.steps;
        const int64_t slot = 2 * (int64_t)home + (began ? 1 : 0);
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            const int r = 16 * nq + (tid >> 4), piece = tid & 15;              // 8 channels
            const int t = (int)a.by_group.div((unsigned)r), g = r - t * a.group;
            if (t >= now.live) continue;
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
                const int64_t row = now.row + t;
                const int h = now.head * a.group + g;
                const int64_t to = row * a.os0 + h * a.os1 + 8 * piece;
                if constexpr (F32) {
                    *(f32x4*)((float*)a.out + to) = f32x4{sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv};
                    *(f32x4*)((float*)a.out + to + 4) = f32x4{sum[4] * inv, sum[5] * inv, sum[6] * inv, sum[7] * inv};
                } else {
                    bf16x8 w;
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = (__bf16)(sum[e] * inv);
                    *(bf16x8*)((__bf16*)a.out + to) = w;
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
            const unsigned rest = now.steps - now.first - now.count;                        // of whole runs, the last perhaps not whole
            int32_t* rec = a.record + 4 + 4 * home;
            rec[0] = now.row; rec[1] = now.live; rec[2] = now.head; rec[3] = 1 + (int)((rest + run.share - 1) / run.share);
        }
        if constexpr (kAcross) {
            if (!another) break;
            now = then;
        } else {
            if (!next_unit(a, run)) break;
            now = unit_of(a, run);
            begin(now);
        }
    }
}

template <typename T, int NQ, bool SMALL>
hipError_t launch(const PagedArgs& a, hipStream_t st) {
    constexpr int smem = 4 * 16 * NQ * (kHeadDim + 2) * 4;
    if (smem > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)paged_fp4_kernel<T, NQ, SMALL>, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((paged_fp4_kernel<T, NQ, SMALL>), dim3(a.workgroups), dim3(kThreads), smem, st, a);
    return hipGetLastError();
}
template <typename T, int NQ>
hipError_t launch_pages(const CacheShape& sh, const PagedArgs& a, hipStream_t st) { return sh.page_shift < 5 ? launch<T, NQ, true>(a, st) : launch<T, NQ, false>(a, st); }

}  // namespace

hipError_t launch_paged_fp4(const CacheShape& sh, const PagedRoute& route, const PagedArgs& a, hipStream_t st) {
    if (sh.dtype == 1) return route.rows == 16 ? launch_pages<__bf16, 1>(sh, a, st) : launch_pages<__bf16, 2>(sh, a, st);
    return route.rows == 16 ? launch_pages<float, 1>(sh, a, st) : route.rows == 32 ? launch_pages<float, 2>(sh, a, st) : launch_pages<float, 4>(sh, a, st);
}

}  // namespace cp
