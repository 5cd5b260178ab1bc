// Causal attention with a sliding window and a few first tokens that stay visible, for the last n_q of n_k tokens: query i, at position p = n_k - n_q + i, sees key j if j <= p and
// (j > p - window or j < n_sinks).  A prompt (n_q = n_k), a follow-up prompt behind a cache, a decoded token (n_q = 1).
//
// A row is a (query, head) pair; the rows of a kv head are numbered query by query, head by head, so that consecutive rows share keys and any number of query heads per kv head
// fills the tiles.  What a tile of rows reads: the keys from the first one in its first query's window to its last query's position, and in front of them the first tokens that
// this stretch leaves behind.
#include "row_tile.h"
#include "sliding_plan.h"
#include <algorithm>
#include <mutex>

namespace slim {

// Workgroup -> (kv head, number within it): each XCD its own kv heads where they divide over the XCDs, so that a head's keys meet in one L2.
__device__ __forceinline__ int own_kv_head(int Hkv, int& number) {
    if (Hkv % 8 == 0) {
        const int j = blockIdx.x >> 3, per = Hkv >> 3;
        number = j / per;
        return (blockIdx.x & 7) * per + j % per;
    }
    number = blockIdx.x / Hkv;
    return blockIdx.x % Hkv;
}

// ---- few rows: 16 of them per workgroup, the units of 32 keys dealt to its waves and to `splits` workgroups
// Bound by latency (a token over 4160 keys of 32 / 8 heads 7 us and 2.2 for the merge: Query and keys in one trip to memory, the waves' merge, the workgroups'), and from some hundred
// tiles on by how fast the CUs take keys, 1.8 ns a unit of 16 KB over the whole chip (sliding_plan.h).  Keys one unit ahead in registers: slower, fewer waves share a CU then.
constexpr int kSlideWaves = 4;

// Values of keys of the unit that some row does not see may be infinite or undefined: their weight is 0, which a product would turn into an undefined sum.  The unit's values
// are added key by key then, each to the rows that see it.
template <typename T, int D, typename F>
__device__ __forceinline__ void add_values_singly(RowTile<T, D>& t, const float* w, const T* v_unit, size_t stride, int have, F sees) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, qr = lane >> 4;
#pragma unroll 1
    for (int at = 0; at < 4; ++at) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int key = (i >> 2) * 16 + at * 4 + (i & 3);
            const float wk = __shfl(w[i], at * 16 + l16, 64);
            if (key < have && sees(key)) {
                const T* row = v_unit + (size_t)key * stride + qr * 4;
#pragma unroll
                for (int dt = 0; dt < RowTile<T, D>::DT; ++dt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) t.o[dt][e] += wk * Elem<T>::ld(row + dt * 16 + e);
            }
        }
    }
}
__device__ __forceinline__ bool odd_bits(const uint4& c, float) {
    float f[4];
    Elem<float>::unpack(c, f);
    return !(fabsf(f[0]) < INFINITY) || !(fabsf(f[1]) < INFINITY) || !(fabsf(f[2]) < INFINITY) || !(fabsf(f[3]) < INFINITY);
}
__device__ __forceinline__ bool odd_bits(const uint4& c, bf16_t) {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i == 0 ? c.x : i == 1 ? c.y : i == 2 ? c.z : c.w;
        odd |= (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
    }
    return odd;
}

// Units u0, u0 + step, .. of the keys [f0, f1) and [s0, s1), which hold what the rows see of some stretch.  p: position of row l16.
template <typename T, int D>
__device__ __forceinline__ void sliding_units(RowTile<T, D>& t, const T* __restrict__ k, const T* __restrict__ v, const SlidingRows& a, const SlidingSpan& sp, int f0, int f1, int s0, int s1, int p,
                                              int u0, int step, unsigned tile) {
    typedef RowTile<T, D> Tile;
    constexpr int NT = Tile::NT, NP = Tile::NP, KS = Tile::KS, V = Elem<T>::kVec, PC = 8 / V;      // 16-byte pieces of eight channels
    const int lane = threadIdx.x & 63, l16 = lane & 15, qr = lane >> 4;
    const size_t stride = (size_t)a.Hkv * D;
    const int u_first = max(0, f1 - f0 + kTileKeys - 1) / kTileKeys, n_units = u_first + max(0, s1 - s0 + kTileKeys - 1) / kTileKeys;
    for (int u = u0; u < n_units; u += step) {
        const int j0 = u < u_first ? f0 + u * kTileKeys : s0 + (u - u_first) * kTileKeys, have = min(kTileKeys, (u < u_first ? f1 : s1) - j0);
        uint4 kx[2][KS][PC], vx[2][KS][PC];
        size_t at[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            at[h] = (size_t)(j0 + min(l16 + 16 * h, have - 1)) * stride + qr * (D / 4);      // rows behind the last key repeat it: not seen
#pragma unroll
            for (int j = 0; j < KS; ++j)
#pragma unroll
                for (int c = 0; c < PC; ++c) kx[h][j][c] = *reinterpret_cast<const uint4*>(k + at[h] + j * 8 + c * V);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < KS; ++j)
#pragma unroll
                for (int c = 0; c < PC; ++c) vx[h][j][c] = *reinterpret_cast<const uint4*>(v + at[h] + j * 8 + c * V);
        auto terms = [&](const uint4* c, bf16x8* x) {
            if constexpr (sizeof(T) == 2) {
                x[0] = __builtin_bit_cast(bf16x8, c[0]);
            } else {
                float f[8];
                Elem<float>::unpack(c[0], f);
                Elem<float>::unpack(c[1], f + 4);
                bf16_terms<NT>(f, x);
            }
        };
        f32x4 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            typename Tile::Scores sum;
#pragma unroll
            for (int j = 0; j < KS; ++j) {
                bf16x8 x[NT];
                terms(kx[h][j], x);
                t.template add_scores<NT>(x, j, sum);
            }
            s[h] = sum.sum();
        }
        const bool whole = have == kTileKeys && j0 + kTileKeys - 1 <= sp.p0 && (j0 > sp.p1 - a.window || j0 + kTileKeys <= a.sinks);      // every row sees every key
        // (without branches: nothing but comparisons and selections)
        auto sees = [&](int key) { const int j = j0 + key; return (key < have) & (j <= p) & ((j > p - a.window) | (j < a.sinks)); };
        if (!whole) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = s[h][e];
                    s[h][e] = sees(h * 16 + qr * 4 + e) ? x : -INFINITY;
                }
        }
        float w[8];
        t.weigh(s, a.scale_log2e, w);
        if (!whole) {
            bool odd = false;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < KS; ++j)
#pragma unroll
                    for (int c = 0; c < PC; ++c) odd |= odd_bits(vx[h][j][c], T());
            if (__any(odd)) {
                add_values_singly<T, D>(t, w, v + (size_t)j0 * stride, stride, have, sees);
                continue;
            }
        }
        bf16x8 pw[NP], x[2][KS][NT];
        bf16_terms<NP>(w, pw);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < KS; ++j) terms(vx[h][j], x[h][j]);
#pragma unroll
        for (int b = 0; b < NT; ++b) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < KS; ++j) *(LdsB128)(tile + Tile::v_piece(l16 + 16 * h, qr * KS + j)) = x[h][j][b];
            t.template add_values<NT>(pw, b, tile);
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(64 * kSlideWaves) sliding_rows_kernel(const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v, SlidingRows a, int n_rt, int splits,
                                                                        T* __restrict__ out, float* __restrict__ part) {
    typedef RowTile<T, D> Tile;
    __shared__ __align__(16) unsigned char lds[kSlideWaves * Tile::kLdsBytes];
    int rt;
    const int g = own_kv_head(a.Hkv, rt), split = rt / n_rt;         // (row tiles that read the same keys side by side)
    rt -= split * n_rt;
    const int lane = threadIdx.x & 63, l16 = lane & 15, Hq = a.G * a.Hkv, rows = a.n_q * a.G;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r0 = rt * kTileRows, count = min(kTileRows, rows - r0);
    const SlidingSpan sp(a, r0, count);
    const int r = min(r0 + l16, rows - 1), i = r / a.G;
    Tile t;
    t.begin(q + ((size_t)i * Hq + g * a.G + (r - i * a.G)) * D);
    sliding_units<T, D>(t, k + (size_t)g * D, v + (size_t)g * D, a, sp, 0, sp.first, sp.start, sp.end, a.n_k - a.n_q + i, split * kSlideWaves + wave, splits * kSlideWaves,
                        (unsigned)(uintptr_t)lds + wave * Tile::kLdsBytes);
    merge_waves<T, D, kSlideWaves>(t, lds, count, [&](int x, int dd, float acc, float l, float M) {
        const int i = (r0 + x) / a.G;
        const size_t row = (size_t)i * Hq + g * a.G + (r0 + x - i * a.G);
        if (splits == 1) {
            Elem<T>::st(out + row * D + dd, acc / l);
        } else {
            float* dst = part + ((size_t)split * a.n_q * Hq + row) * (D + 2);
            dst[dd] = acc;
            if (dd == 0) { dst[D] = M; dst[D + 1] = l; }
        }
    });
}

// ---- many rows: bfloat16, 256 rows per workgroup, 64 per wave
// The weights enter the product with the values as one bfloat16, rounded by up to 2^-8 as in the prompt attention, where the tiles of 16 rows take two: a second term is half as many
// matrix instructions again, which bound this kernel.  Against 64 bits the results are off by 2.3 10^-3 of their size instead of 1.7 10^-3, of which the output's own rounding is 1.65.
// Sums, the reference and the results are float.
// The loop of the prompt attention (gen_attn_asm.py, which says how it runs), over the tiles of 128 keys that the workgroup's rows see: those of the first tokens, if the stretch
// leaves any behind, then the stretch; up to 96 first tokens share a tile with its beginning (with a tile of their own 32768 tokens, window 1024 637 us instead of 596,
// window 4096 1775 instead of 1748).  Where the two would meet the stretch begins at key 0 instead.
// Bound by the matrix instructions and what stands between them in the loop, 2.8 us for a tile of 128 keys on every CU (1.5 PFLOP/s), and by what a workgroup does beside its tiles,
// about 10 us with its CU to itself (first loads 5, softmax reference and edges 2, results 3): 32768 tokens of 32 / 8 heads, window 4096, 1.65 to 1.77 ms (1.18 to 1.26 PFLOP/s, by inputs and cards), window 1024
// 0.59 ms (0.92), window 256 0.30 ms (0.46).
constexpr int LD = 128, LW = 4, LKV = kSlideTile, LTILE_BYTES = LKV * LD * 2, LSTAGE_BYTES = 2 * LTILE_BYTES, LSTAGES = 2, LROWS = 64 * LW;
constexpr int kPartRow = LD + 4;         // floats of a row's partial result (16-byte aligned)

__global__ void __launch_bounds__(64 * LW) __attribute__((amdgpu_waves_per_eu(1, 1)))
sliding_many_kernel(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ Kg, const bf16_t* __restrict__ Vg, bf16_t* __restrict__ O, SlidingRows a, int n_rt, int splits,
                    float* __restrict__ part) {
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, hh = lane >> 5;
    // Workgroup -> (kv head, row tile, part of its keys): each XCD its own kv heads, whose keys then meet in one L2.  Long tiles of a prompt start with the last row, which has the most
    // keys, so that short ones fill the end; tiles of fewer than 2048 keys with the first, so that the workgroups do not start and end together.  us from the last row on / from the first,
    // 32 / 8 heads: 32768 tokens, window 4096 1654 / 1682, 2048 962 / 975, 1024 586 / 598, 256 307 / 300; 8192 tokens, all in sight 434 / 489, window 4096 341 / 365, 2048 232 / 226,
    // 1024 143 / 139, 512 97 / 94; with 64 heads, 2048 430 / 441 and 1024 277 / 271; 28 / 4, 2048 199 / 204.  (Around the line it goes by the rounds of workgroups too: 1 to 3 % of the
    // slower side are taken where those are few or the windows long.)
    int rt;
    const int g = own_kv_head(a.Hkv, rt);
    const int split = rt % splits;
    rt /= splits;
    if (a.window + LROWS / a.G >= 2048) rt = n_rt - 1 - rt;
    const int Hq = a.G * a.Hkv, rows = a.n_q * a.G, off = a.n_k - a.n_q, r0 = rt * LROWS, rw = r0 + wave * 64;
    const unsigned rowbytes = (unsigned)a.Hkv * LD * 2, tile_bytes = rowbytes * LKV;
    const SlidingSpan all(a, r0, LROWS), mine(a, min(rw, rows - 1), 64);
    const SlidingTiles whole(all, a.window);
    const int from = (int)((long long)split * whole.all / splits), to = (int)((long long)(split + 1) * whole.all / splits);
    // a partial result: rows of kPartRow floats, the values, the reference and the sum
    float* part_rows = part + ((size_t)split * a.Hkv + g) * rows * kPartRow;
    if (from == to) {                                    // more parts than tiles: no keys
        const int r = r0 + threadIdx.x;
        if (r < rows) {
            part_rows[(size_t)r * kPartRow + LD] = -INFINITY;
            part_rows[(size_t)r * kPartRow + LD + 1] = 0.f;
        }
        return;
    }
    const SlidingTiles tl = whole.part(from, to);
    const int start = tl.start, k00 = tl.k00;
    const unsigned nst = tl.apart, first_units = tl.units, nkt = tl.all, nhead = tl.clean, nmain = tl.masked, last_tile = nkt - 1;
    const unsigned last_ragged = tl.left != LKV ? last_tile : 0xffffffffu, nl1 = tl.left - 1;   // rows of the last tile behind its keys repeat the last one
    const unsigned n_units = 4 * last_tile + (tl.left + 31) / 32;
    const uint64_t jump = (uint64_t)(start - k00 - (int)first_units * 32) * rowbytes;
    const unsigned jump_lo = nst ? (unsigned)jump : 0, jump_hi = nst ? (unsigned)(jump >> 32) : 0;
    const uint64_t kb = (uint64_t)(uintptr_t)(Kg + (size_t)g * LD) + (uint64_t)k00 * rowbytes;
    const uint64_t vb = (uint64_t)(uintptr_t)(Vg + (size_t)g * LD) + (uint64_t)k00 * rowbytes;
    const unsigned kbase_lo = (unsigned)kb, kbase_hi = (unsigned)(kb >> 32), vbase_lo = (unsigned)vb, vbase_hi = (unsigned)(vb >> 32);
    const int qw0 = mine.p0, lowq = mine.p1 - a.window, window = a.window, sinks = a.sinks;

    // the lane's two rows
    const int ra = min(rw + l32, rows - 1), rb = min(rw + 32 + l32, rows - 1), ia = ra / a.G, ib = rb / a.G;
    const size_t qa = ((size_t)ia * Hq + g * a.G + (ra - ia * a.G)) * LD, qb = ((size_t)ib * Hq + g * a.G + (rb - ib * a.G)) * LD;
    const bf16_t *qrow0 = Q + qa + hh * 8, *qrow1 = Q + qb + hh * 8;
    float *stat0 = part_rows + (size_t)ra * kPartRow + LD, *stat1 = part_rows + (size_t)rb * kPartRow + LD;              // used where there are parts
    const int hh4 = 4 * hh, limabs0 = off + ia - hh4, limabs1 = off + ib - hh4;
    const unsigned valid0 = hh == 0 && rw + l32 < rows, valid1 = hh == 0 && rw + 32 + l32 < rows;
    // Each row's product with its own token: a reference that is never minus infinity, whatever the first unit's mask leaves of the row.
    auto own_product = [&](const bf16_t* qr, int i) {
        const bf16_t* kr = Kg + ((size_t)(off + i) * a.Hkv + g) * LD + hh * 8;
        float sum = 0.f;
#pragma unroll
        for (int st = 0; st < 8; ++st) {
            float x[8], y[8];
            Elem<bf16_t>::unpack(*reinterpret_cast<const uint4*>(qr + st * 16), x);
            Elem<bf16_t>::unpack(*reinterpret_cast<const uint4*>(kr + st * 16), y);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += x[e] * y[e];
        }
        return sum + __shfl_xor(sum, 32, 64);
    };
    // (with a first token in sight the first unit holds a key that every row sees; 4.7 us of a workgroup's 110 where that is not so)
    float own0 = -INFINITY, own1 = -INFINITY;
    if (a.sinks == 0 || splits > 1) { own0 = own_product(qrow0, ia); own1 = own_product(qrow1, ib); }

    // LDS byte addresses of the lane's fragment reads and the operands of its tile loads, as the prompt attention's.
    auto k_at = [](int r, int c) { return (r * 16 + (c ^ (r & 15))) * 16; };
    auto v_at = [](int r, int c) { return (r * 16 + (c ^ ((r & 3) << 2))) * 16; };
    const unsigned lds_base = (unsigned)(uintptr_t)lds;
    const unsigned koff0 = lds_base + k_at(l32, hh);
    const int q4 = lane >> 4, sl = lane & 15, key_lane = 4 * (q4 >> 1) + (sl >> 2);
    const unsigned voff0 = lds_base + LTILE_BYTES + v_at(key_lane, 2 * (q4 & 1) + ((sl & 3) >> 1)) + (sl & 1) * 8;
    const unsigned row0 = wave * 4 + (lane >> 4), slot = lane & 15;
    const unsigned kchunk = (slot ^ (row0 & 15)) * 16, vchunk = (slot ^ ((row0 & 3) << 2)) * 16;
    const unsigned ldsw = lds_base + wave * 1024;
    // of the lane's first row of the result, which is there in bfloat16, or in float where there are parts
    const unsigned oaddr = splits == 1 ? lds_base + wave * (64 * LD * 2) + l32 * (LD * 2) + ((l32 & 15) << 4) + 8 * hh : lds_base + wave * (64 * LD * 4) + l32 * (LD * 4) + ((l32 ^ hh) << 4);
    float odd = 0.f;                                     // not 0: some result is not finite

    asm volatile(
#include "sliding_bf16_body.inc"
        : [odd] "+v"(odd)
        : [oaddr] "v"(oaddr), [koff0] "v"(koff0), [voff0] "v"(voff0), [r0] "v"(row0), [kchunk] "v"(kchunk), [vchunk] "v"(vchunk),
          [qrow0] "v"(qrow0), [qrow1] "v"(qrow1), [stat0] "v"(stat0), [stat1] "v"(stat1),
          [limabs0] "v"(limabs0), [limabs1] "v"(limabs1), [valid0] "v"(valid0), [valid1] "v"(valid1), [own0] "v"(own0), [own1] "v"(own1), [hh4] "v"(hh4),
          [kbase_lo] "s"(kbase_lo), [kbase_hi] "s"(kbase_hi), [vbase_lo] "s"(vbase_lo), [vbase_hi] "s"(vbase_hi),
          [nkt] "s"(nkt), [nhead] "s"(nhead), [nmain] "s"(nmain), [nst] "s"(nst), [first_units] "s"(first_units), [origin] "s"(tl.origin()), [start] "s"(start), [last_tile] "s"(last_tile), [last_ragged] "s"(last_ragged),
          [rowbytes] "s"(rowbytes), [tile_bytes] "s"(tile_bytes), [jump_lo] "s"(jump_lo), [jump_hi] "s"(jump_hi), [scale] "s"(a.scale_log2e), [nl1] "s"(nl1),
          [ldsw] "s"(ldsw), [qw0] "s"(qw0), [lowq] "s"(lowq), [window] "s"(window), [sinks] "s"(sinks), [k00] "s"(k00),
          [n_units] "s"(n_units), [split] "s"(splits - 1)
        :
#include "sliding_bf16_clobbers.inc"
    );
    // The wave's 64 rows lie in LDS: whole rows are written, past the caches, which hold keys (8192 tokens, window 256 76.7 us without, 71.0; 32768, window 4096 1720 / 1699).
    if (splits == 1) {
        const int c = lane & 15, step_i = 4 / a.G, step_h = 4 - step_i * a.G;
        int r = rw + (lane >> 4), i = r / a.G, h = r - i * a.G;
        const unsigned char* src = lds + wave * (64 * LD * 2);
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            const int x = t * 4 + (lane >> 4);
            const uint4 v = *reinterpret_cast<const uint4*>(src + x * (LD * 2) + ((c ^ (x & 15)) << 4));
            if (r < rows) store_stream16(O + ((size_t)i * Hq + g * a.G + h) * LD + c * 8, v);
            r += 4;
            i += step_i;
            h += step_h;
            if (h >= a.G) { h -= a.G; ++i; }
        }
    } else {
        const int c = lane & 31;
        const unsigned char* src = lds + wave * (64 * LD * 4);
#pragma unroll
        for (int t = 0; t < 32; ++t) {
            const int x = t * 2 + (lane >> 5);
            const uint4 v = *reinterpret_cast<const uint4*>(src + x * (LD * 4) + ((c ^ (x & 31)) << 4));
            if (rw + x < rows) *reinterpret_cast<uint4*>(part_rows + (size_t)(rw + x) * kPartRow + c * 4) = v;
        }
    }
    // Keys or values that are not finite: perhaps behind a mask, where a weight of 0 does not undo them.  The wave's rows are computed again, 16 at a time.
    __syncthreads();
    if (!__any(!(odd == 0.f))) return;
    const int l16 = lane & 15, qr = lane >> 4;
#pragma unroll 1
    for (int t = 0; t < 4; ++t) {
        const int first = rw + t * kTileRows;
        if (first >= rows) break;
        const SlidingSpan sp(a, first, kTileRows);
        const int r = min(first + l16, rows - 1), i = r / a.G;
        const size_t at = ((size_t)i * Hq + g * a.G + (r - i * a.G)) * LD;
        RowTile<bf16_t, LD> tile;
        tile.begin(Q + at);
        // the keys of the workgroup's tiles, up to the row tile's last position
        const int f0 = first_units ? k00 : 0, f1 = first_units ? min(sp.first, k00 + (int)first_units * 32) : 0;
        const int s1 = min(sp.end, tl.origin() + (int)last_tile * LKV + tl.left);
        sliding_units<bf16_t, LD>(tile, Kg + (size_t)g * LD, Vg + (size_t)g * LD, a, sp, f0, f1, start, s1, off + i, 0, 1, lds_base + wave * RowTile<bf16_t, LD>::kLdsBytes);
        tile.finish_sum();
        if (first + l16 >= rows) continue;
        if (splits > 1) {
            float* dst = part_rows + (size_t)r * kPartRow;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f32x4*>(dst + dt * 16 + qr * 4) = tile.o[dt];
            if (qr == 0) { dst[LD] = tile.reference(); dst[LD + 1] = tile.l; }
        } else {
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
                *reinterpret_cast<uint2*>(O + at + dt * 16 + qr * 4) = make_uint2(pack_bf16x2(tile.o[dt][0] / tile.l, tile.o[dt][1] / tile.l),
                                                                                  pack_bf16x2(tile.o[dt][2] / tile.l, tile.o[dt][3] / tile.l));
        }
    }
}

// part[split][kv head][row][kPartRow] -> out: 32 lanes a row, four channels each.
__global__ void __launch_bounds__(256) sliding_merge_kernel(const float* __restrict__ part, int splits, SlidingRows a, bf16_t* __restrict__ out) {
    const int rows = a.n_q * a.G, total = rows * a.Hkv, row = blockIdx.x * 8 + (threadIdx.x >> 5), c = (threadIdx.x & 31) * 4;
    if (row >= total) return;
    const float* p = part + (size_t)row * kPartRow;
    const size_t step = (size_t)total * kPartRow;
    float M = -INFINITY;
    for (int s = 0; s < splits; ++s) M = fmaxf(M, p[s * step + LD]);
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const float m = p[s * step + LD], sum = p[s * step + LD + 1];
        const f32x4 v = *reinterpret_cast<const f32x4*>(p + s * step + c);
        const float w = sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - M);
        l += w * sum;
        if (sum != 0.f) o += w * v;                      // (what a part without keys left is not looked at)
    }
    const int g = row / rows, r = row - g * rows, i = r / a.G;
    *reinterpret_cast<uint2*>(out + ((size_t)i * a.G * a.Hkv + g * a.G + (r - i * a.G)) * LD + c) = make_uint2(pack_bf16x2(o[0] / l, o[1] / l), pack_bf16x2(o[2] / l, o[3] / l));
}

static int launch_sliding_many(const void* q, const void* k, const void* v, const SlidingRows& a, int splits, void* out, float* part, hipStream_t st) {
    const int smem = LSTAGES * LSTAGE_BYTES;
    static std::once_flag once;
    static hipError_t err = hipSuccess;
    std::call_once(once, [&] { err = hipFuncSetAttribute((const void*)sliding_many_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, smem); });
    if (err != hipSuccess) return set_hip_error(err);
    const int n_rt = (int)(((long long)a.n_q * a.G + LROWS - 1) / LROWS);
    hipLaunchKernelGGL(sliding_many_kernel, dim3((unsigned)((long long)n_rt * a.Hkv * splits)), dim3(64 * LW), smem, st, (const bf16_t*)q, (const bf16_t*)k, (const bf16_t*)v,
                       (bf16_t*)out, a, n_rt, splits, part);
    const int rc = check_launch();
    if (rc || splits == 1) return rc;
    hipLaunchKernelGGL(sliding_merge_kernel, dim3((unsigned)(((long long)a.n_q * a.G * a.Hkv + 7) / 8)), dim3(256), 0, st, part, splits, a, (bf16_t*)out);
    return check_launch();
}

// In how many parts a call's tiles of 256 rows run, 0: in tiles of 16.  (rowbytes and the 24-bit multiplies of the tile loads' offsets bound the number of kv heads.)
static int sliding_many(const SlidingRows& a, int dtype) {
    return dtype == SLIM_BF16 && a.Hkv <= 4096 ? sliding_parts(a.n_q, a.n_k, a.G, a.Hkv, a.window, a.sinks) : 0;
}
// (a window or a number of first tokens beyond the keys is all of them)
static SlidingRows sliding_rows(int n_q, int n_k, int Hq, int Hkv, int window, int sinks, float scale) {
    return SlidingRows{n_q, n_k, Hq / Hkv, Hkv, std::min(window, n_k), std::min(sinks, n_k), scale * 1.4426950408889634f};
}

size_t sliding_workspace_floats(int n_q, int n_k, int Hq, int Hkv, int d, int window, int sinks, int dtype) {
    const SlidingRows a = sliding_rows(n_q, n_k, Hq, Hkv, window, sinks, 0.f);
    if (const int parts = sliding_many(a, dtype)) return parts > 1 ? (size_t)parts * n_q * Hq * kPartRow : 0;
    const int splits = sliding_splits(n_q, n_k, a.G, Hkv, a.window, a.sinks, kMergeParts);
    return splits > 1 ? (size_t)splits * n_q * Hq * (d + 2) : 0;
}

int launch_sliding_attn(const void* q, const void* k, const void* v, int n_q, int n_k, int Hq, int Hkv, int d, int window, int sinks, float scale, int dtype, void* out,
                        float* part, hipStream_t st) {
    const SlidingRows a = sliding_rows(n_q, n_k, Hq, Hkv, window, sinks, scale);
    if (const int parts = sliding_many(a, dtype)) return launch_sliding_many(q, k, v, a, parts, out, part, st);
    const int splits = sliding_splits(n_q, n_k, a.G, Hkv, a.window, a.sinks, kMergeParts);
    const long long tiles = ((long long)n_q * a.G + kTileRows - 1) / kTileRows;
    const dim3 grid((unsigned)(tiles * Hkv * splits));
#define SLIM_SLIDE(T, D) hipLaunchKernelGGL((sliding_rows_kernel<T, D>), grid, dim3(64 * kSlideWaves), 0, st, (const T*)q, (const T*)k, (const T*)v, a, (int)tiles, splits, (T*)out, part)
    if (dtype == SLIM_BF16) SLIM_SLIDE(bf16_t, 128);
    else if (d == 32) SLIM_SLIDE(float, 32);
    else if (d == 64) SLIM_SLIDE(float, 64);
    else SLIM_SLIDE(float, 128);
#undef SLIM_SLIDE
    const int rc = check_launch();
    return rc || splits == 1 ? rc : launch_merge_rows(part, splits, n_q * Hq, d, dtype, out, st);
}

}  // namespace slim
