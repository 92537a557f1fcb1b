// How many steps over its keys each tile of a sequence's new tokens takes, as the kernels of attention over pages count them, and two rules by which they deal the tiles out.
//
// With n new tokens of `keys` in all, tile i (of 2^tile_shift tokens) sees keys up to its last token and takes
//   ahead + min(cap, ceil((i + 1) tile / step)),   ahead = ceil(max(keys - n, 0) / step),  cap = max(1, ceil(keys / step)) - ahead
// steps: never fewer than its last token needs, at most one more, and never more than the keys fill.  The latter holds too where there are more
// new tokens than keys (rows that see nothing), and keeps the sums below within what the host has bounded by the tensors' sizes.
#pragma once
#include "fast_div.h"

namespace cp {

struct TileSteps {
    unsigned ahead, cap;

    __host__ __device__ __forceinline__ TileSteps(int tokens, int keys, int step_shift) {
        const unsigned up = (1u << step_shift) - 1, all = ((unsigned)keys + up) >> step_shift;
        ahead = ((unsigned)(keys > tokens ? keys - tokens : 0) + up) >> step_shift;
        cap = (all > 1 ? all : 1) - ahead;
    }
    __host__ __device__ __forceinline__ unsigned of(unsigned i, int tile_shift, int step_shift) const {
        const unsigned mine = (((i + 1) << tile_shift) + (1u << step_shift) - 1) >> step_shift;
        return ahead + (mine < cap ? mine : cap);
    }
    // of tiles 0 .. j - 1 together
    __host__ __device__ __forceinline__ unsigned before(unsigned j, int tile_shift, int step_shift) const {
        const unsigned full = (cap << step_shift) >> tile_shift, i = j < full ? j : full;      // tiles from `full` on take cap
        unsigned n = j * ahead + (j - i) * cap;
        if (tile_shift >= step_shift) return n + ((i * (i + 1) / 2) << (tile_shift - step_shift));
        const int m = step_shift - tile_shift;
        const unsigned whole = i >> m, rest = i & ((1u << m) - 1);
        return n + ((whole * (whole + 1) / 2) << m) + rest * (whole + 1);
    }
};

// Where all sequences are alike, how often every workgroup takes a whole unit before they share what is left: none where there are not units for all.  To and fro (tiles that begin
// early see fewer keys), so an even number, unless the steps of a sequence's first and last tile are nearly the same.
__host__ __device__ __forceinline__ unsigned whole_rounds(unsigned units, unsigned workgroups, unsigned first, unsigned last) {
    const unsigned rounds = units / workgroups;
    return 16 * (last - (last < first ? last : first)) > last ? rounds & ~1u : rounds;
}

// Whether what the rounds leave takes no longer in `turns` of whole units, the longest `longest` steps with its setup, than in `used` runs of `share` steps.
// Cutting evens the work out but is not free: what is left for the join is written and read again, 9 steps' worth where every workgroup leaves some and 4 in
// any case, and in plain pages a step of a run takes a quarter longer than one of a whole unit.  us, cut / whole (32/8 heads, the only layout that this was measured at): 4 x 300 new
// tokens of 600 40.5 / 29.6, of 1000 47.8 / 38.9, of 4000 102 / 106; 16 x 64 of 600 43.2 / 30.9, of 2000 59.9 / 63.2; 1 x 2000 of 2400 78.3 / 74.6; 16 x 300 of 600 (two rounds and
// a half) 78.1 / 72.3; 8 bits 4 x 300 of 1000 50.7 / 42.7, of 2000 67.7 / 68.6.
__host__ __device__ __forceinline__ bool uncut_pays(unsigned turns, unsigned longest, unsigned used, unsigned share, bool mxfp8) {
    const unsigned cut = 4 + 9 * used / 256 + share + (turns == 1 && !mxfp8 ? share / 4 : 0);
    return turns * longest <= cut;
}

}  // namespace cp
