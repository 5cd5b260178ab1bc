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

// The tiles of 128 keys of a workgroup with many rows: `apart` tiles from key k00 on, which hold the first tokens, then tiles from key `start` on, `all` in all.  Where the two would
// meet inside a tile the stretch begins at key 0 and there is nothing apart.  Tiles `clean` .. `masked` - 1 need no mask, but for the first unit of 32 keys of tile `clean`; neither
// does the first unit of tile `masked`.  The last tile is never among them.  left: keys of the last tile.
constexpr int kSlideTile = 128;
struct SlidingTiles {
    int k00, start, apart, all, clean, masked, left;
    constexpr SlidingTiles(const SlidingSpan& s, int window) : k00(0), start(s.start), apart(0), all(0), clean(0), masked(0), left(0) {
        const int tiles = (s.first + kSlideTile - 1) / kSlideTile;
        if (s.first > 0 && tiles * kSlideTile <= s.start) apart = tiles;
        else if (s.first > 0) start = 0;
        if (apart == 0) k00 = start;
        all = apart + (s.end - start + kSlideTile - 1) / kSlideTile;
        const int edge = s.p1 - window + 1 - start;      // keys of the stretch that some row's window does not reach
        clean = apart + ((edge > 0 ? edge : 0) + kSlideTile - 1) / kSlideTile;
        if (clean > all) clean = all;
        const int whole = s.p0 - 31 - start;
        masked = apart + (whole > 0 ? whole : 0) / kSlideTile;
        if (masked < clean) masked = clean;
        left = s.end - start - (all - 1 - apart) * kSlideTile;
    }
    // Tiles from .. to - 1 of them (from < to), as a plan of its own.
    constexpr SlidingTiles part(int from, int to) const {
        SlidingTiles r = *this;
        r.k00 = from < apart ? from * kSlideTile : start + (from - apart) * kSlideTile;
        r.apart = to <= apart || from >= apart ? 0 : apart - from;
        r.start = r.apart ? start : r.k00;
        r.all = to - from;
        r.clean = clean - from < r.apart ? r.apart : clean - from;
        if (to <= apart || r.clean > r.all) r.clean = r.all;
        r.masked = masked - from < r.all - 1 ? masked - from : r.all - 1;
        if (r.masked < r.clean) r.masked = r.clean;
        r.left = to == all ? left : kSlideTile;
        return r;
    }
};

// In how many parts the keys of a row tile of 256 rows are dealt to workgroups (host).  One CU holds one workgroup, 256 of them run at once; a workgroup takes 12 us and 2.8 us a tile;
// parts are written and read once more, 528 bytes a row, in a launch of 5 us.
inline double sliding_parts_us(long long row_tiles, long long tiles, long long rows, int parts) {
    const long long rounds = (row_tiles * parts + 255) / 256;
    return rounds * (12.0 + 2.8 * ((tiles + parts - 1) / parts)) + (parts > 1 ? 5.0 + rows * parts * 528.0 * 2 / 4.5e6 : 0.0);
}
inline int sliding_parts(int n_q, int n_k, int G, int Hkv, int window, int sinks) {
    const long long rows = (long long)n_q * G * Hkv, row_tiles = ((long long)n_q * G + 255) / 256 * Hkv;
    const int span = 256 / G + 1 < n_q ? 256 / G + 1 : n_q;                            // queries of a row tile, about
    const long long near = (long long)window + span < n_k ? (long long)window + span : n_k;
    const long long tiles = (near + kSlideTile - 1) / kSlideTile + (near < n_k ? (sinks + kSlideTile - 1) / kSlideTile : 0);
    int best = 1;
    for (int parts = 2; parts <= 64 && parts <= tiles; ++parts)
        if (sliding_parts_us(row_tiles, tiles, rows, parts) < sliding_parts_us(row_tiles, tiles, rows, best)) best = parts;
    return best;
}

}  // namespace slim
