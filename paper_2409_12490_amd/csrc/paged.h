// What the two kernels of attention over pages share: how the work is cut, and what is left for the join.
//
// A unit is (sequence, KV head, tile of the sequence's new tokens); its rows are the tile's tokens times the KV head's query heads.  A unit takes as many
// steps over its keys as its last token sees, and `setup` more for what a workgroup does around them (with none, workgroups whose run held twenty units of two steps each
// took four times as long as the others).  All steps of all units laid end to end, units in order of sequence, KV head, tile, are dealt to the
// workgroups in equal runs: no workgroup has more than its share, whatever the lengths, and the device alone reads the lengths.  A workgroup
// finishes units that lie in its run; of one that began before it or goes on behind it, it leaves (sum, maximum, weighted V) in the workspace, and
// a second kernel adds these up in order.  (The last workgroup of a unit to arrive adding them up instead, with a ticket and fences that write the XCDs' L2 back: 39 us where the two
// kernels take 11, 350 for 101.  Parts that go past L2, without such fences: not tried.)
//
// Where all sequences are alike and there are units for every workgroup, workgroups first take whole units, round by round to and fro, and share what
// the rounds leave over as above: the 32 workgroups of an XCD then read the keys of one head at the same time, from its L2 (runs of equal length begin anywhere in
// a unit: 34 % of the reads come from L2 for 8192 new tokens of 32768, 32/8 heads, 3346 us; now 3145).  In the kernel of 256-row tiles units are not cut at all, or not those
// that the rounds leave over, where that takes no longer: see find.
#pragma once
#include "cache.h"
#include "paged_steps.h"

namespace cp {

struct PagedArgs {
    const void* q; CachePtr cache;
    const int32_t *table, *q_start, *kv_len;
    void* out; float* lse;
    float* parts;                             // [workgroup][2][rows][128], then (max, sum) [workgroup][2][rows][2]
    float* stats;
    int32_t* record;                          // [0]: workgroups with work; [4 + 4 w ..]: what the last unit of workgroup w needs, see Record
    int tokens, n_seqs, max_pages, n_pages, hq, hkv, group;
    int page_shift, tile_shift, step_shift;
    unsigned workgroups, least, setup;
    unsigned cut_units;                       // that there can be: a workgroup leaves one at most
    int whole;                                // units are not cut: a unit counts as one, whatever its steps
    int mxfp8;
    FastDiv by_group;
    float scale, scale_log2e;
    int64_t qs0, qs1, os0, os1;
};

// A unit that begins in a workgroup's run and ends in a later one's: parts of it are in slot 1 of this workgroup and slot 0 of `parts - 1` that follow.
struct Record { int32_t row, rows_of, head, parts; };             // first token, its tokens, KV head, number of parts (0: no such unit)

namespace {

// wave-uniform values from vector registers
__device__ __forceinline__ int first_lane(int x) { return __builtin_amdgcn_readfirstlane(x); }

struct Sequence {                             // one sequence, checked: whatever the arrays hold, rows and pages stay inside the tensors
    int start, tokens, keys, tiles;
    unsigned length;                          // of one KV head: the steps of its units, setup included

    // the same of tiles 0 .. j - 1
    __device__ __forceinline__ unsigned before(const PagedArgs& a, int j, int whole) const {
        return whole ? (unsigned)j : (unsigned)j * a.setup + TileSteps(tokens, keys, a.step_shift).before((unsigned)j, a.tile_shift, a.step_shift);
    }
    __device__ __forceinline__ unsigned steps_of(const PagedArgs& a, int j) const {    // without setup
        return TileSteps(tokens, keys, a.step_shift).of((unsigned)j, a.tile_shift, a.step_shift);
    }
    __device__ __forceinline__ bool load(const PagedArgs& a, int s, int whole) {       // whether its rows ascend
        const int from = a.q_start[s], to = a.q_start[s + 1], held = a.kv_len[s];
        start = min(max(from, 0), a.tokens);
        tokens = min(max(to, start), a.tokens) - start;
        keys = (int)min((long long)max(held, 0), (long long)a.max_pages << a.page_shift);
        tiles = (int)(((unsigned)tokens + (1u << a.tile_shift) - 1) >> a.tile_shift);
        length = before(a, tiles, whole);
        return from <= to;
    }
    __device__ __forceinline__ Sequence of_lane(int l) const {
        Sequence s;
        s.start = __builtin_amdgcn_readlane(start, l); s.tokens = __builtin_amdgcn_readlane(tokens, l); s.keys = __builtin_amdgcn_readlane(keys, l);
        s.tiles = __builtin_amdgcn_readlane(tiles, l); s.length = (unsigned)__builtin_amdgcn_readlane((int)length, l);
        return s;
    }
};

// What a workgroup works on: whole units first (rounds), then its run.  Every wave works it out by itself.
template <bool ROUNDS>
struct Run {
    unsigned logical, used, share, left;      // its number among those that share, these, steps of each, steps left to it
    int seq, head, tile; unsigned at;         // at: inside the unit, setup first
    Sequence now;
    int whole;                                // units are not cut
    unsigned place; int round, rounds;        // rounds: its number among all; the present round, and how many there are
    unsigned run_left, run_at; int run_seq, run_head, run_tile;     // where the run begins, kept for after the rounds

    __device__ __forceinline__ bool find(const PagedArgs& a, unsigned workgroup, int lane) {
        unsigned total = 0, mine = 0, upto = 0, units = 0, longest = 0;        // units, and the longest with its setup: for ROUNDS
        bool again = a.n_seqs > 64;
        whole = a.whole;
        Sequence s;
        unsigned long long wrong = 0;
        for (int base = 0; base < a.n_seqs; base += 64) {
            wrong |= __builtin_amdgcn_ballot_w64(!s.load(a, min(base + lane, a.n_seqs - 1), whole));
            mine = base + lane < a.n_seqs ? s.length * (unsigned)a.hkv : 0u;
            upto = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) { const unsigned o = __shfl_up(upto, d); if (lane >= d) upto += o; }
            total += (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
            if (ROUNDS) {
                const bool there = base + lane < a.n_seqs && s.tiles;
                units += there ? (unsigned)s.tiles : 0u;
                longest = max(longest, there ? a.setup + s.steps_of(a, s.tiles - 1) : 0u);
            }
        }
        used = 0; logical = 0; left = 0; round = rounds = 0;
        seq = head = tile = 0; at = 0; place = 0; now = Sequence{};
        // Rows that do not ascend are nobody's: sequences could share rows, and be more work than the host has bounded.  Nobody does anything then.
        if (wrong || total == 0) return false;
        unsigned skip = 0;                                         // what the rounds take
        if (ROUNDS && !whole) {
#pragma unroll
            for (int d = 32; d; d >>= 1) { units += __shfl_xor(units, d); longest = max(longest, (unsigned)__shfl_xor(longest, d)); }
            units = (unsigned)first_lane((int)units) * (unsigned)a.hkv;
            longest = (unsigned)first_lane((int)longest);
        }
        if (ROUNDS && !whole && a.n_seqs <= 64) {
            const Sequence one = s.of_lane(0);
            if (__builtin_amdgcn_ballot_w64(s.tokens != one.tokens || s.keys != one.keys) == 0 && units >= a.workgroups) {
                const unsigned last = one.steps_of(a, one.tiles - 1);
                rounds = first_lane((int)whole_rounds(units, a.workgroups, one.steps_of(a, 0), last));
            }
            if (rounds) {
                const unsigned cut = (unsigned)rounds * a.workgroups, heads = (unsigned)first_lane((int)(cut / (unsigned)one.tiles));
                const unsigned rest = cut - heads * (unsigned)one.tiles;
                skip = heads * one.length + one.before(a, (int)rest, whole);
                place = (workgroup & 7) * (a.workgroups / 8) + (workgroup >> 3);
            }
        }
        total -= skip;
        auto deal = [&]() {
            share = max(whole ? 1u : a.least, (unsigned)first_lane((int)((total + a.workgroups - 1) / a.workgroups)));
            used = (unsigned)first_lane((int)((total + share - 1) / share));
        };
        deal();
        if (ROUNDS && !whole && total) {
            const unsigned rest = units - (unsigned)rounds * a.workgroups, turns = (unsigned)first_lane((int)((rest + a.workgroups - 1) / a.workgroups));
            if (first_lane(uncut_pays(turns, longest, used, share, a.mxfp8))) {
                if (rounds) { rounds += (int)turns; total = used = 0; }        // the last round not full
                else {
                    whole = 1; again = true; total = units;
                    deal();
                }
            }
        }
        // neighbouring runs share keys (tiles of one head) and go to one XCD (workgroup id mod 8)
        logical = (workgroup & 7) * ((used + 7) / 8) + (workgroup >> 3);
        if ((workgroup >> 3) < (used + 7) / 8 && logical < used) {              // not where used is 0
            left = min(share, total - logical * share);
            const unsigned begin = skip + logical * share;
            unsigned past = 0;
            for (int base = 0; base < a.n_seqs; base += 64) {
                if (again) {
                    s.load(a, min(base + lane, a.n_seqs - 1), whole);
                    mine = base + lane < a.n_seqs ? s.length * (unsigned)a.hkv : 0u;
                    upto = mine;
#pragma unroll
                    for (int d = 1; d < 64; d <<= 1) { const unsigned o = __shfl_up(upto, d); if (lane >= d) upto += o; }
                }
                const unsigned long long behind = __builtin_amdgcn_ballot_w64(past + upto > begin);
                if (behind) {
                    const int l = __builtin_ctzll(behind);
                    unsigned rest = begin - past - (unsigned)__builtin_amdgcn_readlane((int)(upto - mine), l);
                    seq = base + l;
                    now = s.of_lane(l);
                    head = first_lane((int)(rest / now.length));
                    rest -= (unsigned)head * now.length;
                    int lo = 0, hi = now.tiles - 1;                // the last tile that begins at or before it
                    while (lo < hi) {
                        const int mid = (lo + hi + 1) >> 1;
                        if (now.before(a, mid, whole) <= rest) lo = mid; else hi = mid - 1;
                    }
                    tile = lo;
                    at = rest - now.before(a, lo, whole);
                    break;
                }
                past += (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
            }
        }
        else logical = ~0u;
        if (ROUNDS) {                                              // all of it is the same for the wave: back into scalar registers
            auto fix = [](auto& x) { x = first_lane((int)x); };
            fix(logical); fix(used); fix(share); fix(left); fix(at); fix(seq); fix(head); fix(tile); fix(rounds); fix(whole); fix(place);
            fix(now.start); fix(now.tokens); fix(now.keys); fix(now.tiles); fix(now.length);
        }
        if (ROUNDS && rounds) {
            run_left = left; run_at = at; run_seq = seq; run_head = head; run_tile = tile;
            return whole_unit(a);
        }
        return left > 0 && has_steps(a);
    }
    // the unit of the present round; false where a round that is not full has none for this workgroup
    __device__ __forceinline__ bool whole_unit(const PagedArgs& a) {
        const unsigned unit = (unsigned)round * a.workgroups + (round & 1 ? a.workgroups - 1 - place : place);
        now.load(a, 0, whole);                                            // all are alike but for their start
        const unsigned tiles = (unsigned)first_lane(now.tiles), heads = (unsigned)first_lane((int)(unit / tiles));
        tile = (int)(unit - heads * tiles);
        seq = first_lane((int)(heads / (unsigned)a.hkv));
        if (seq >= a.n_seqs) return false;
        head = (int)(heads - (unsigned)seq * (unsigned)a.hkv);
        now.load(a, seq, whole);
        now = now.of_lane(0);
        at = 0;
        left = a.setup + now.steps_of(a, tile);
        return true;
    }
    // What there is of the present unit: steps first .. first + count - 1 of `unit`.
    __device__ __forceinline__ void piece(const PagedArgs& a, unsigned& first, unsigned& count, unsigned& unit) const {
        unit = now.steps_of(a, tile);
        if (whole) { first = 0; count = unit; return; }
        first = at > a.setup ? at - a.setup : 0u;
        count = min(at + left - a.setup, unit) - first;
    }
    // Where the run has nothing but setup of its present unit, this is its last, and its steps are the next workgroup's.
    __device__ __forceinline__ bool has_steps(const PagedArgs& a) const { return whole || at + left > a.setup; }
    // on to the unit behind this one; false where the run or the work ends
    __device__ __forceinline__ bool next(const PagedArgs& a) {
        const unsigned rest = whole ? 1u : a.setup + now.steps_of(a, tile) - at;
        if (left <= rest) return false;
        left -= rest;
        at = 0;
        if (++tile < now.tiles) return true;
        tile = 0;
        if (++head < a.hkv) return true;
        head = 0;
        do {
            if (++seq >= a.n_seqs) return false;
            now.load(a, seq, whole);
            now = now.of_lane(0);
        } while (now.tiles == 0);
        return true;
    }
    __device__ __forceinline__ bool next_steps(const PagedArgs& a) {
        if (ROUNDS && round < rounds) {
            if (++round < rounds && whole_unit(a)) return true;
            round = rounds;
            left = run_left; at = run_at; seq = run_seq; head = run_head; tile = run_tile;
            if (left == 0) return false;
            now.load(a, seq, whole);
            now = now.of_lane(0);
            return has_steps(a);
        }
        return next(a) && has_steps(a);
    }
};

// Adds up the parts of a unit that more than one workgroup worked on: sum_x 2^(c (m_x - M)) O_x / sum_x 2^(c (m_x - M)) l_x.  All that a thread reads of
// several parts is asked for at once: a part's latency, not its bytes, is what the kernel takes.
// Few rows: 32 threads of 4 channels take a row, and GROUPS of them every GROUPS-th part, whose sums meet in LDS (8 units of 64 parts by four groups of 16
// threads, four parts at a time: 31 us, now 5).  WIDE, the layout of the kernel of 256-row tiles: a thread takes 8 channels of a row (4 with GROUPS), neighbouring threads
// neighbouring rows, and asks for no part that is not there (six at once, the last again where there are fewer, 12 follow-ups of 1 to 300 tokens over 8-bit pages: 13.4 us, now 11).
// The grid has a place for each unit that can be cut, and a workgroup finds the record of its own among all: with a place for each workgroup of the first kernel the
// units of 32 parts, all their pieces, were all on one XCD (1 x 64 tokens after 16000, 32/8 heads: 42 us, now 10; 1 x 256 17 and 9.6, 1 x 512 12.3 and 9.6).
template <typename T, bool WIDE, int GROUPS>
__global__ __launch_bounds__(256) void join_kernel(PagedArgs a, int rows, unsigned grid_y) {
    // threadIdx and its like are calls where this is compiled without IEEE mode: attn_bf16.h.  at once: rows, fours of channels, and of each thread
    constexpr int kRowsAtOnce = WIDE ? 32 : 8 / GROUPS, kAcross = WIDE ? 8 / GROUPS : 32, kPieces = WIDE && GROUPS == 1 ? 2 : 1, kAhead = kPieces == 2 ? 4 : 8;
    constexpr int kParts = 32 / (kAcross * kPieces);               // of a row's channels, a workgroup each
    __shared__ __attribute__((aligned(16))) float rest[GROUPS > 1 ? 8 * 128 : 4];
    __shared__ float rest_m[GROUPS * kRowsAtOnce], rest_l[GROUPS * kRowsAtOnce];
    const int tid = (int)__builtin_amdgcn_workitem_id_x(), lane = tid & 63;
    // the blockIdx.x-th unit that was cut: there are no more of them than units, where workgroups are up to 512
    constexpr int kRecords = WIDE ? 4 : 8;                         // of a lane
    const unsigned used = (unsigned)a.record[0];
    int4 all[kRecords];
#pragma unroll
    for (int i = 0; i < kRecords; ++i) all[i] = *(const int4*)(a.record + 4 + 4 * min(64u * i + lane, a.workgroups - 1));
    unsigned rank = __builtin_amdgcn_workgroup_id_x(), w = ~0u;
    int4 rec{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kRecords; ++i) {
        const bool cut = 64u * i + lane < used && all[i].w >= 2;
        const unsigned long long which = __builtin_amdgcn_ballot_w64(cut);
        const unsigned n = (unsigned)__builtin_popcountll(which);
        if (w == ~0u && rank < n) {
            const unsigned before = __builtin_amdgcn_mbcnt_hi((unsigned)(which >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)which, 0u));
            const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(cut && before == rank));
            w = 64u * i + (unsigned)l;
            rec.x = __builtin_amdgcn_readlane(all[i].x, l); rec.y = __builtin_amdgcn_readlane(all[i].y, l);
            rec.z = __builtin_amdgcn_readlane(all[i].z, l); rec.w = __builtin_amdgcn_readlane(all[i].w, l);
        }
        rank -= n;                                                 // of no meaning behind the unit
    }
    if (w == ~0u) return;
    const int parts = rec.w, live = rec.y * a.group;
    const int local = WIDE ? tid & 31 : (tid >> 5) % kRowsAtOnce, group = tid / (256 / GROUPS), across = WIDE ? (tid >> 5) % kAcross : tid & 31;
    const float c = a.scale_log2e;
    auto slot = [&](int x) { return 2 * (int64_t)(w + x) + (x == 0 ? 1 : 0); };
    const int half = (int)(__builtin_amdgcn_workgroup_id_y() % kParts), turn = (int)(__builtin_amdgcn_workgroup_id_y() / kParts), turns = (int)(grid_y / kParts);
    for (int first = turn * kRowsAtOnce; first < live; first += turns * kRowsAtOnce) {     // uniform
        const int r = min(first + local, live - 1);
        auto channel = [&](int j) { return 4 * (kAcross * (kPieces * half + j) + across); };
        auto place = [&](int j) {
            const int cg = channel(j) >> 2;
            return WIDE ? (r >> 5) * 4096 + (cg >> 1) * 256 + ((cg & 1) * 32 + (r & 31)) * 4 : r * kHeadDim + 4 * cg;
        };
        float M = -INFINITY, L = 0.f;
        float4 sum[kPieces];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) sum[j] = float4{0.f, 0.f, 0.f, 0.f};
        auto add = [&](float m, float l, const float4 (&v)[kPieces], float safe) {
            const float f = __builtin_amdgcn_exp2f((m - safe) * c);
            L = fmaf(f, l, L);
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                sum[j].x = fmaf(f, v[j].x, sum[j].x); sum[j].y = fmaf(f, v[j].y, sum[j].y);
                sum[j].z = fmaf(f, v[j].z, sum[j].z); sum[j].w = fmaf(f, v[j].w, sum[j].w);
            }
        };
        auto move_to = [&](float top) -> float {                   // the reference point; returns what exponents are taken from
            const float safe = top == -INFINITY ? 0.f : top, f = __builtin_amdgcn_exp2f((M - safe) * c);
            L *= f;
#pragma unroll
            for (int j = 0; j < kPieces; ++j) { sum[j].x *= f; sum[j].y *= f; sum[j].z *= f; sum[j].w *= f; }
            M = top;
            return safe;
        };
        for (int x0 = group; x0 < parts; x0 += GROUPS * kAhead) {
            float2 ml[kAhead]; float4 v[kAhead][kPieces];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (WIDE && x0 + i * GROUPS >= parts) continue;    // the same for a wave
                const int64_t from = slot(min(x0 + i * GROUPS, parts - 1)) * rows;
                ml[i] = *(const float2*)(a.stats + 2 * (from + r));
#pragma unroll
                for (int j = 0; j < kPieces; ++j) v[i][j] = *(const float4*)(a.parts + from * kHeadDim + place(j));
            }
            float top = M;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) top = x0 + i * GROUPS < parts ? fmaxf(top, ml[i].x) : top;
            const float safe = move_to(top);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (x0 + i * GROUPS < parts) add(ml[i].x, ml[i].y, v[i], safe);
        }
        if constexpr (GROUPS > 1) {
            __syncthreads();                                       // the row before has been read
            *(float4*)(rest + 4 * tid) = sum[0];
            if (across == 0) { rest_m[group * kRowsAtOnce + local] = M; rest_l[group * kRowsAtOnce + local] = L; }
            __syncthreads();
            if (group != 0) continue;
            float top = M;
#pragma unroll
            for (int x = 1; x < GROUPS; ++x) top = fmaxf(top, rest_m[local + x * kRowsAtOnce]);
            const float safe = move_to(top);
#pragma unroll
            for (int x = 1; x < GROUPS; ++x) {
                const float4 v[1] = {*(const float4*)(rest + 4 * (tid + 256 / GROUPS * x))};
                add(rest_m[local + x * kRowsAtOnce], rest_l[local + x * kRowsAtOnce], v, safe);
            }
        }
        if (first + local >= live) continue;
        const float inv = L == 0.f ? 0.f : 1.0f / L;
        const int t = (int)a.by_group.div((unsigned)r), h = rec.z * a.group + r - t * a.group;
        const int64_t row = rec.x + t;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int64_t to = row * a.os0 + h * a.os1 + channel(j);
            const float4 y = {sum[j].x * inv, sum[j].y * inv, sum[j].z * inv, sum[j].w * inv};
            if constexpr (sizeof(T) == 4) {
                *(float4*)((float*)a.out + to) = y;
            } else {
                typedef __attribute__((ext_vector_type(4))) __bf16 four;
                *(four*)((__bf16*)a.out + to) = four{(__bf16)y.x, (__bf16)y.y, (__bf16)y.z, (__bf16)y.w};
            }
        }
        if (a.lse && channel(0) == 0) a.lse[row * a.hq + h] = L == 0.f ? -INFINITY : M * a.scale + logf(L);
    }
}

}  // namespace

hipError_t launch_paged_rows(const CacheShape& sh, const PagedRoute& route, const PagedArgs& a, hipStream_t st);
hipError_t launch_paged_chunk(const CacheShape& sh, const PagedArgs& a, hipStream_t st);

}  // namespace cp
