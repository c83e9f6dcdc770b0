// How the attentions over the paged cache walk over rows and keys: tiles of a
// sequence's rows, the blocks of BLK key positions that they see, the parts that
// the blocks are split into.  Args: the kernel's arguments with kv, T, H, grp (=
// H / G), window, sinks and splits.
#pragma once

#include "kvcache.h"

namespace mq {

// What one row sees: positions (lo, hi], and below the sinks.
struct Sees {
    int32_t lo, hi;
};

// A tile of rows of one sequence and the blocks that its rows see.  Positions
// are below 2^31 and above -2^26 (lengths are int32).
template <int BLK>
struct RowTile {
    int32_t b;
    int32_t s0, pos0;         // the sequence's first token row and its position
    uint32_t row0, rows;      // first row (token, head of the group), the sequence's rows
    int32_t n, skip0, skip1;  // blocks to walk: n, without those in [skip0, skip1)
    int32_t hi_min, hi_max;   // positions of the first and last token
    int32_t last;             // of the page list's entries, the last one that a row sees
    __device__ int32_t block(int32_t i) const { return i < skip0 ? i : i + (skip1 - skip0); }
    // Every row sees all positions of the block.
    template <class Args>
    __device__ bool full(const Args& p, int32_t blk) const
    {
        return blk * BLK + (BLK - 1) <= hi_min &&
               (p.window == 0 || blk * BLK > hi_max - p.window);
    }
};

// What a tile of R rows from t.row0 on sees; len: the sequence's length, s1: the end
// of its token rows.
template <int R, int BLK, class Args>
__device__ inline void set_seen(const Args& p, int32_t s1, int32_t len, RowTile<BLK>& t)
{
    const int32_t grp = p.grp;
    t.pos0 = len - (s1 - t.s0);
    t.hi_max = t.pos0 + (int32_t)((min(t.row0 + (R - 1), t.rows - 1)) / (uint32_t)grp);
    t.hi_min = t.pos0 + (int32_t)(t.row0 / (uint32_t)grp);
    // blocks with places, up to the last row's
    const int64_t list = ((p.kv.ld << p.kv.shift) + BLK - 1) / BLK;
    const int32_t end = t.hi_max < 0 ? 0 : (int32_t)min((int64_t)(t.hi_max / BLK + 1), list);
    t.last = (int32_t)min((int64_t)(t.hi_max >> p.kv.shift), p.kv.ld - 1);
    t.skip0 = t.skip1 = 0;
    if (p.window > 0) {
        t.skip1 = t.hi_min >= p.window ? min((t.hi_min - p.window + 1) / BLK, end) : 0;
        t.skip0 = min((int32_t)(((int64_t)p.sinks + BLK - 1) / BLK), t.skip1);
    }
    t.n = end - (t.skip1 - t.skip0);
}

// Tile of R rows from row0 on of sequence b with token rows [s0, s1).
template <int R, int BLK, class Args>
__device__ inline void set_tile(const Args& p, int32_t b, int32_t s0, int32_t s1, int32_t len,
                                uint32_t row0, RowTile<BLK>& t)
{
    t.b = b;
    t.s0 = s0;
    t.rows = (uint32_t)(s1 - s0) * (uint32_t)p.grp;
    t.row0 = row0;
    set_seen<R>(p, s1, len, t);
}

// The tile's index counts from floor(starts[b] grp / R) + b for sequence b: an
// upper bound of the tiles before it that needs no scan.
template <int R, int BLK, class Args>
__device__ inline bool find_tile(const Args& p, int64_t index, RowTile<BLK>& t)
{
    const int32_t* starts = p.kv.starts;
    const int32_t grp = p.grp;
    t.b = find_seq(p.kv.B, index, [=](int32_t i) { return (int64_t)starts[i] * grp / R + i; });
    const int32_t s0 = starts[t.b], s1 = starts[t.b + 1], len = max(p.kv.lens[t.b], 0);
    if (s0 < 0 || s1 > (int32_t)p.T || s0 >= s1) return false;
    const int64_t row0 = (index - ((int64_t)s0 * grp / R + t.b)) * R;
    t.s0 = s0;
    t.rows = (uint32_t)(s1 - s0) * (uint32_t)grp;  // below 2^32 (T H D is below 2^36)
    if (row0 < 0 || row0 >= (int64_t)t.rows) return false;
    t.row0 = (uint32_t)row0;
    set_seen<R>(p, s1, len, t);
    return true;
}

// A row, by default lane & 15 of the 16 from `first` on: token row, query head, what it
// sees.
struct RowAt {
    bool have;
    int64_t t;
    int32_t head;
    Sees sees;
    template <class Args, int BLK>
    __device__ RowAt(const Args& p, const RowTile<BLK>& tile, uint32_t first, int32_t g0)
        : RowAt(p, tile, first, g0, threadIdx.x & 15)
    {
    }
    // row r from `first` on
    template <class Args, int BLK>
    __device__ RowAt(const Args& p, const RowTile<BLK>& tile, uint32_t first, int32_t g0, uint32_t r)
    {
        const uint32_t x = first + r;  // no overflow: rows below 2^32 - 64
        have = x < tile.rows;
        const uint32_t row = have ? x : tile.rows - 1, tok = row / (uint32_t)p.grp;
        t = (int64_t)tile.s0 + tok;
        head = g0 * p.grp + (int32_t)(row - tok * (uint32_t)p.grp);
        sees.hi = max(tile.pos0 + (int32_t)tok, -1);
        sees.lo = p.window > 0 && sees.hi >= p.window ? sees.hi - p.window : -1;
    }
};

// The split's blocks [i0, i1) of the tile.
template <class Args, int BLK>
__device__ inline void split_range(const Args& p, const RowTile<BLK>& t, int split, int32_t& i0,
                                   int32_t& i1)
{
    const int32_t per = (t.n + p.splits - 1) / p.splits;
    i0 = per * split;
    i1 = min(i0 + per, t.n);
}

// Work-groups go to the eight XCDs in turn, each with an L2 of its own: those
// that read the same keys (a cache head's part) are given to one XCD, or to
// 8 / n of them in turn where there are n < 8 such parts.  The tiles of an
// XCD come heaviest first up to the middle (the last tokens of a prompt see
// the most keys), then lightest first, so that a CU's two work-groups add up
// to the same.
struct Place {
    int64_t tile;
    int32_t part;  // g + G * split
};
template <class Args>
__device__ inline Place place_of(const Args& p, int64_t id, int64_t tiles)
{
    const int64_t parts = (int64_t)p.kv.G * p.splits;
    Place w;
    int64_t n = tiles, at;
    if (parts % 8 == 0) {
        const int64_t slot = id >> 3;
        w.part = (int32_t)((slot / tiles) * 8 + (id & 7));
        at = slot % tiles;
    } else if (8 % parts == 0) {
        const int64_t r = 8 / parts;
        w.part = (int32_t)((id & 7) % parts);
        n = (tiles + r - 1) / r;
        at = id >> 3;
        w.tile = ((id & 7) / parts);  // of every r tiles
        at = at < n - n / 2 ? n - 1 - at : at - (n - n / 2);
        w.tile += at * r;
        return w;
    } else {
        w.part = (int32_t)(id / tiles);
        at = id % tiles;
    }
    w.tile = at < n - n / 2 ? n - 1 - at : at - (n - n / 2);
    return w;
}

// Row tiles of all sequences, at most.
inline int64_t row_tiles(int64_t T, int64_t B, int32_t grp, int R) { return T * grp / R + B; }

}  // namespace mq
