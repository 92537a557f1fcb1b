// What the two kernels of attention over pages share: how the work is cut, and what is left for the join.
//
// A unit is (sequence, KV head, tile of the sequence's new tokens); its rows are the tile's tokens times the KV head's query heads.  A unit takes as many
// steps over its keys as its last token sees.  All steps of all units laid end to end, units in order of sequence, KV head, tile, are dealt to the
// workgroups in equal runs: no workgroup has more than its share, whatever the lengths, and the device alone reads the lengths.  A workgroup
// finishes units that lie in its run; of one that began before it or goes on behind it, it leaves (sum, maximum, weighted V) in the workspace, and
// join_kernel adds these up in order.
#pragma once
#include "cache.h"

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
    unsigned workgroups, least;
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
    int start, tokens, keys, tiles, ahead;    // ahead: steps of the keys that all its tokens see, rounded up
    unsigned steps;                           // of one KV head

    __device__ __forceinline__ unsigned before(int j, int tile_shift, int step_shift) const {   // steps of tiles 0 .. j-1, j < tiles
        // tile i: ahead + ceil((i + 1) tile / step)
        if (tile_shift >= step_shift) return (unsigned)j * ahead + (((unsigned)j * (j + 1) / 2) << (tile_shift - step_shift));
        const int m = step_shift - tile_shift;
        const unsigned a = (unsigned)j >> m, b = (unsigned)j & ((1u << m) - 1);
        return (unsigned)j * ahead + ((a * (a + 1) / 2) << m) + b * (a + 1);
    }
    __device__ __forceinline__ unsigned steps_of(int j, int tile_shift, int step_shift) const {
        if (j == tiles - 1) return max(1u, (unsigned)(keys + (1 << step_shift) - 1) >> step_shift);   // its last token sees all keys
        return ahead + ((unsigned)(((j + 1) << tile_shift) + (1 << step_shift) - 1) >> step_shift);
    }
    // uniform: s is the same in all lanes, and so is what follows
    __device__ __forceinline__ void load(const PagedArgs& a, int s, bool uniform) {
        int from = a.q_start[s], to = a.q_start[s + 1], held = a.kv_len[s];
        if (uniform) { from = first_lane(from); to = first_lane(to); held = first_lane(held); }
        start = min(max(from, 0), a.tokens);
        tokens = min(max(to, start), a.tokens) - start;
        keys = (int)min((long long)max(held, 0), (long long)a.max_pages << a.page_shift);
        tiles = (tokens + (1 << a.tile_shift) - 1) >> a.tile_shift;
        ahead = (max(keys - tokens, 0) + (1 << a.step_shift) - 1) >> a.step_shift;
        steps = tiles ? before(tiles - 1, a.tile_shift, a.step_shift) + steps_of(tiles - 1, a.tile_shift, a.step_shift) : 0u;
    }
};

// A workgroup's run: where it begins and how long it is.  Every wave works it out by itself.
struct Run {
    unsigned logical, used, share, left;      // its number among those with work, these, steps of each, steps of this one
    int seq, head, tile; unsigned step;
    Sequence now;

    __device__ __forceinline__ bool find(const PagedArgs& a, unsigned workgroup, int lane) {
        unsigned total = 0, mine = 0, upto = 0;
        Sequence s;
        for (int base = 0; base < a.n_seqs; base += 64) {
            mine = 0;
            if (base + lane < a.n_seqs) { s.load(a, base + lane, false); mine = s.steps * (unsigned)a.hkv; }
            upto = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) { const unsigned o = __shfl_up(upto, d); if (lane >= d) upto += o; }
            total += (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
        }
        if (total == 0) return false;
        share = max(a.least, (unsigned)first_lane((int)((total + a.workgroups - 1) / a.workgroups)));
        used = (unsigned)first_lane((int)((total + share - 1) / share));
        // neighbouring runs share keys (tiles of one head) and go to one XCD (workgroup id mod 8)
        logical = (workgroup & 7) * ((used + 7) / 8) + (workgroup >> 3);
        if ((workgroup >> 3) >= (used + 7) / 8 || logical >= used) return false;
        const unsigned begin = logical * share;
        left = min(share, total - begin);
        unsigned past = 0;
        for (int base = 0; base < a.n_seqs; base += 64) {
            if (a.n_seqs > 64) {
                mine = 0;
                if (base + lane < a.n_seqs) { s.load(a, base + lane, false); mine = s.steps * (unsigned)a.hkv; }
                upto = mine;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) { const unsigned o = __shfl_up(upto, d); if (lane >= d) upto += o; }
            }
            const unsigned long long behind = __builtin_amdgcn_ballot_w64(past + upto > begin);
            if (behind) {
                const int at = __builtin_ctzll(behind);
                unsigned rest = begin - past - (unsigned)__builtin_amdgcn_readlane((int)(upto - mine), at);
                seq = base + at;
                now.load(a, seq, true);
                head = first_lane((int)(rest / now.steps));
                rest -= (unsigned)head * now.steps;
                int lo = 0, hi = now.tiles - 1;                    // the last tile that begins at or before it
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (now.before(mid, a.tile_shift, a.step_shift) <= rest) lo = mid; else hi = mid - 1;
                }
                tile = lo;
                step = rest - now.before(lo, a.tile_shift, a.step_shift);
                return true;
            }
            past += (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
        }
        return false;
    }
    // the unit behind this one; false past the last
    __device__ __forceinline__ bool next(const PagedArgs& a) {
        step = 0;
        if (++tile < now.tiles) return true;
        tile = 0;
        if (++head < a.hkv) return true;
        head = 0;
        do {
            if (++seq >= a.n_seqs) return false;
            now.load(a, seq, true);
        } while (now.tiles == 0);
        return true;
    }
};

}  // namespace

hipError_t launch_paged_rows(const CacheShape& sh, const PagedRoute& route, const PagedArgs& a, hipStream_t st);
hipError_t launch_paged_chunk(const CacheShape& sh, const PagedArgs& a, hipStream_t st);

}  // namespace cp
