// How many steps over its keys each tile of a sequence's new tokens takes, as the kernels of attention over pages count them.
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

}  // namespace cp
