// Which keys a tile of rows reads in sliding-window attention, and in which order (host and device, no GPU needed).
#pragma once

namespace slim {

struct SlidingRows {
    int n_q, n_k, G, Hkv, window, sinks;                 // G: query heads per kv head; window, sinks: at most n_k
    float scale_log2e;
};

// The keys that rows r0 .. r0 + count - 1 of a kv head see: [0, first) and [start, end); the first and last row's positions.
struct SlidingSpan {
    int p0, p1, first, start, end;
    constexpr SlidingSpan(const SlidingRows& a, int r0, int count) : p0(0), p1(0), first(0), start(0), end(0) {
        const int off = a.n_k - a.n_q, last = a.n_q - 1, i0 = r0 / a.G, i1 = (r0 + count - 1) / a.G;
        p0 = off + (i0 < last ? i0 : last);
        p1 = off + (i1 < last ? i1 : last);
        start = p0 - a.window + 1 > 0 ? p0 - a.window + 1 : 0;
        first = a.sinks < start ? a.sinks : start;
        end = p1 + 1;
    }
};

// The tiles of 128 keys of a workgroup with many rows: `apart` tiles from key 0 on, which hold the first tokens, then tiles from key `start` on, `all` in all.  Where the two would
// meet inside a tile the stretch begins at key 0 and there is nothing apart.  Tiles `clean` .. `masked` - 1 need no mask, but for the first unit of 32 keys of tile `clean`; neither
// does the first unit of tile `masked`.  left: keys of the last tile.
constexpr int kSlideTile = 128;
struct SlidingTiles {
    int start, apart, all, clean, masked, left;
    constexpr SlidingTiles(const SlidingSpan& s, int window) : start(s.start), apart(0), all(0), clean(0), masked(0), left(0) {
        const int tiles = (s.first + kSlideTile - 1) / kSlideTile;
        if (s.first > 0 && tiles * kSlideTile <= s.start) apart = tiles;
        else if (s.first > 0) start = 0;
        all = apart + (s.end - start + kSlideTile - 1) / kSlideTile;
        const int edge = s.p1 - window + 1 - start;      // keys of the stretch that some row's window does not reach
        clean = apart + ((edge > 0 ? edge : 0) + kSlideTile - 1) / kSlideTile;
        if (clean > all) clean = all;
        const int whole = s.p0 - 31 - start;
        masked = apart + (whole > 0 ? whole : 0) / kSlideTile;
        if (masked < clean) masked = clean;
        left = s.end - start - (all - 1 - apart) * kSlideTile;
    }
};

}  // namespace slim
