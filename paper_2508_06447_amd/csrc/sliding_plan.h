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

// The tiles of 128 keys of a workgroup with many rows: `units` times 32 keys from key k00 on, which hold the first tokens, then keys from key `start` on; `apart` tiles have some of the
// former, `all` there are.  Fewer than four such units share the first tile with the beginning of the stretch; four or more fill whole tiles.  Where the two would meet inside a unit
// (inside a tile) the stretch begins at key 0 and there is nothing apart.  Tiles `clean` .. `masked` - 1 need no mask, but for the first unit of 32 keys of tile `clean`; neither does the
// first unit of tile `masked`.  The last tile is never among them.  left: keys of the last tile.
constexpr int kSlideTile = 128;
struct SlidingTiles {
    int k00, start, units, apart, all, clean, masked, left;
    constexpr SlidingTiles(const SlidingSpan& s, int window) : k00(0), start(s.start), units(0), apart(0), all(0), clean(0), masked(0), left(0) {
        units = (s.first + 31) / 32;
        if (units > 3) units = (units + 3) / 4 * 4;
        if (units * 32 > s.start) {
            start = 0;
            units = 0;
        }
        apart = (units + 3) / 4;
        if (units == 0) k00 = start;
        const int before = units * 32;
        all = (before + s.end - start + kSlideTile - 1) / kSlideTile;
        const int edge = s.p1 - window + 1 - start;      // keys of the stretch that some row's window does not reach
        clean = (before + (edge > 0 ? edge : 0) + kSlideTile - 1) / kSlideTile;
        if (clean > all) clean = all;
        const int whole = s.p0 - 31 - start;
        masked = (before + (whole > 0 ? whole : 0)) / kSlideTile;
        if (masked < clean) masked = clean;
        left = before + s.end - start - (all - 1) * kSlideTile;
    }
    // Key of the stretch's tiles: that of tile i is origin() + 128 i.
    constexpr int origin() const { return start - units * 32; }
    // Tiles from .. to - 1 of them (from < to), as a plan of its own.
    constexpr SlidingTiles part(int from, int to) const {
        SlidingTiles r = *this;
        r.k00 = (from < apart ? k00 : origin()) + from * kSlideTile;
        r.units = from >= apart || 4 * to <= units ? 0 : units - 4 * from;
        r.apart = (r.units + 3) / 4;
        r.start = r.units ? start : r.k00;
        r.all = to - from;
        r.clean = clean - from < r.apart ? r.apart : clean - from;
        if (4 * to <= units || r.clean > r.all) r.clean = r.all;
        r.masked = masked - from < r.all - 1 ? masked - from : r.all - 1;
        if (r.masked < r.clean) r.masked = r.clean;
        r.left = to == all ? left : kSlideTile;
        return r;
    }
};

// ---- which kernel, and over how many workgroups a tile's keys are dealt (host).  us, bfloat16, 32 / 8 heads of 128, window 4096, 64 first tokens, behind 8192 tokens.
// Keys that a tile of `rows` rows reads, the first tokens apart.
inline long long sliding_keys(int n_q, int n_k, int G, int window, int rows) {
    const long long span = rows / G + 1 < n_q ? rows / G + 1 : n_q;                    // its queries, about
    return window + span < n_k ? window + span : n_k;
}

// Tiles of 16 rows: 32-key units of a tile.  A wave's unit is 16 KB of keys and values, and what bounds these tiles is how fast the CUs take them: 1.8 ns a unit over the whole
// chip, whatever the number of rows in it (64 queries 38 us, 17024 units; 512 232 us, 136192; 16 queries over 32768 keys 65 to 73 us, 32768).
inline long long sliding_units_of_tile(int n_q, int n_k, int G, int window, int sinks) {
    const long long near = sliding_keys(n_q, n_k, G, window, 16);
    return (near + 31) / 32 + (near < n_k ? (sinks + 31) / 32 : 0);
}
// Workgroups of four waves that share a tile: 512 of them in all for up to 64 rows of the output (a token 9.0 us, with 256 10.0; 2 tokens 10.6 / 10.7), 256 where there are more, since
// every part of a row is written and read once more (4 tokens 12.4 / 11.9, 16 20.1 / 17.7, 32 26.9 / 24.6; float32, 1000 queries of 4 / 2 heads of 64, window 300, 12.7 / 11.1); every
// wave the same number of units where that can be.  A part that saves a wave one unit costs its launch (a token with a window of 100 7.2 / 6.9 us alone, 64 with 256 12.0 / 10.8; two
// units, a token with a window of 256 7.0 / 8.2).
inline int sliding_splits(int n_q, int n_k, int G, int Hkv, int window, int sinks, int most_parts) {
    const long long tiles = ((long long)n_q * G + 15) / 16 * Hkv, units = sliding_units_of_tile(n_q, n_k, G, window, sinks);
    long long most = ((long long)n_q * G * Hkv <= 64 ? 512 : 256) / tiles;
    most = most < 1 ? 1 : most > most_parts ? most_parts : most;
    const long long rounds = (units + 4 * most - 1) / (4 * most), want = (units + 4 * rounds - 1) / (4 * rounds);
    const long long parts = want < most ? want : most;
    return (units + 3) / 4 - (units + 4 * parts - 1) / (4 * parts) < 2 ? 1 : (int)parts;
}

// Tiles of 256 rows: one CU holds one workgroup, 256 of them run at once; a workgroup takes 12 us and 2.8 us a tile of 128 keys; parts are written and read once more, 528 bytes a
// row, in a launch of 5 us.  64 queries in 1 / 2 / 4 / 8 / 16 parts 91 / 58 / 40 / 35 / 39, 512 92 / 64 / 50 / 70 / 107, 2048 119 / 145; 1511 queries of 28 / 4 heads behind 9856 tokens,
// all in sight, in 1 / 2 / 3 / 4 / 6 237 / 256 / 209 / 230 / 241.  (The 12 us are those of an earlier state of the kernel, now about 10.)
inline double sliding_many_us(int n_q, int n_k, int G, int Hkv, int window, int sinks, int parts) {
    const long long rows = (long long)n_q * G * Hkv, row_tiles = ((long long)n_q * G + 255) / 256 * Hkv, near = sliding_keys(n_q, n_k, G, window, 256);
    const long long tiles = (near + (near < n_k ? (sinks + 31ll) / 32 * 32 : 0) + kSlideTile - 1) / kSlideTile, rounds = (row_tiles * parts + 255) / 256;
    return rounds * (12.0 + 2.8 * ((tiles + parts - 1) / parts)) + (parts > 1 ? 5.0 + rows * parts * 528.0 * 2 / 4.5e6 : 0.0);
}
// In how many parts a call's tiles of 256 rows run; 0: it runs in tiles of 16 rows (6 us, and over the whole chip 6 ns a tile and 1.8 ns a unit; 16 queries 17.8 us, in tiles of 256
// 30; 32 24.5 / 31.5; 48 38 / 34; 64 of 28 / 4 heads with a window of 500 13.4 / 21; 16 over 32768 keys 73 / 65; windows of 16, where a tile is one unit and its other waves have
// nothing: 1024 26 / 13, 4096 92 / 30, 32768 742 / 237).  Of 26 calls of 1 to 32768 queries, six head layouts and windows of 16 to 32768, each measured both ways and
// in several numbers of parts, the faster tiles are chosen in all; a number of parts that is more than 2 % slower than another in three (48 queries 37 us in 17 parts, 34 in eight; 200 behind
// 2000 tokens, window 1024, 64 / 8 heads 35 in three, 32 in one; 28 / 4 29.5 in five, 28 in four).
inline int sliding_parts(int n_q, int n_k, int G, int Hkv, int window, int sinks) {
    int best = 1;
    double us = sliding_many_us(n_q, n_k, G, Hkv, window, sinks, 1);
    for (int parts = 2; parts <= 64; ++parts) {
        const double t = sliding_many_us(n_q, n_k, G, Hkv, window, sinks, parts);
        if (t < us) { us = t; best = parts; }
    }
    const double few = 6.0 + (double)(((long long)n_q * G + 15) / 16 * Hkv) * (6.0 + 1.8 * (double)sliding_units_of_tile(n_q, n_k, G, window, sinks)) * 1e-3;
    return few < us ? 0 : best;
}

}  // namespace slim
