// Causal attention with a sliding window and a few first tokens that stay visible, for the last n_q of n_k tokens: query i, at position p = n_k - n_q + i, sees key j if j <= p and
// (j > p - window or j < n_sinks).  A prompt (n_q = n_k), a follow-up prompt behind a cache, a decoded token (n_q = 1).
//
// A row is a (query, head) pair; the rows of a kv head are numbered query by query, head by head, so that consecutive rows share keys and any number of query heads per kv head
// fills the tiles.  What a tile of rows reads: the keys from the first one in its first query's window to its last query's position, and in front of them the first tokens that
// this stretch leaves behind.
#include "row_tile.h"
#include "routes.h"
#include <algorithm>

namespace slim {

struct SlidingRows {
    int n_q, n_k, G, Hkv, window, sinks;
    float scale_log2e;
};
// The keys that rows r0 .. r0 + count - 1 of a kv head see: [0, first) and [start, end); rows' first and last position.
struct SlidingSpan {
    int p0, p1, first, start, end;
    __device__ __forceinline__ SlidingSpan(const SlidingRows& a, int r0, int count) {
        const int off = a.n_k - a.n_q;
        p0 = off + min(r0 / a.G, a.n_q - 1);
        p1 = off + min((r0 + count - 1) / a.G, a.n_q - 1);
        start = max(0, p0 - a.window + 1);
        first = min(a.sinks, start);
        end = p1 + 1;
    }
};

// ---- few rows: 16 of them per workgroup, the units of 32 keys dealt to its waves and to gridDim.z workgroups
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

// Units u0, u0 + step, .. of the rows' keys.  p: position of row l16.
template <typename T, int D>
__device__ __forceinline__ void sliding_units(RowTile<T, D>& t, const T* __restrict__ k, const T* __restrict__ v, const SlidingRows& a, const SlidingSpan& sp, int p, int u0, int step,
                                              unsigned tile) {
    typedef RowTile<T, D> Tile;
    constexpr int NT = Tile::NT, NP = Tile::NP, KS = Tile::KS, V = Elem<T>::kVec, PC = 8 / V;      // 16-byte pieces of eight channels
    const int lane = threadIdx.x & 63, l16 = lane & 15, qr = lane >> 4;
    const size_t stride = (size_t)a.Hkv * D;
    const int u_first = (sp.first + kTileKeys - 1) / kTileKeys, n_units = u_first + (sp.end - sp.start + kTileKeys - 1) / kTileKeys;
    for (int u = u0; u < n_units; u += step) {
        const int j0 = u < u_first ? u * kTileKeys : sp.start + (u - u_first) * kTileKeys, have = min(kTileKeys, (u < u_first ? sp.first : sp.end) - j0);
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
        f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < KS; ++j) {
                bf16x8 x[NT];
                terms(kx[h][j], x);
                t.template add_scores<NT>(x, j, s[h]);
            }
        const bool whole = have == kTileKeys && j0 + kTileKeys - 1 <= sp.p0 && (j0 > sp.p1 - a.window || j0 + kTileKeys <= a.sinks);      // every row sees every key
        auto sees = [&](int key) { const int j = j0 + key; return key < have && j <= p && (j > p - a.window || j < a.sinks); };
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[h][e] = whole || sees(h * 16 + qr * 4 + e) ? s[h][e] * a.scale_log2e : -INFINITY;
        float w[8];
        t.weigh(s, w);
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
__global__ void __launch_bounds__(64 * kSlideWaves) sliding_rows_kernel(const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v, SlidingRows a, T* __restrict__ out,
                                                                        float* __restrict__ part) {
    typedef RowTile<T, D> Tile;
    __shared__ __align__(16) unsigned char lds[kSlideWaves * Tile::kLdsBytes];
    const int g = blockIdx.y, lane = threadIdx.x & 63, l16 = lane & 15, Hq = a.G * a.Hkv, rows = a.n_q * a.G;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r0 = blockIdx.x * kTileRows, count = min(kTileRows, rows - r0);
    const SlidingSpan sp(a, r0, count);
    const int r = min(r0 + l16, rows - 1), i = r / a.G;
    Tile t;
    t.begin(q + ((size_t)i * Hq + g * a.G + (r - i * a.G)) * D);
    sliding_units<T, D>(t, k + (size_t)g * D, v + (size_t)g * D, a, sp, a.n_k - a.n_q + i, blockIdx.z * kSlideWaves + wave, gridDim.z * kSlideWaves,
                        (unsigned)(uintptr_t)lds + wave * Tile::kLdsBytes);
    merge_waves<T, D, kSlideWaves>(t, lds, count, [&](int x, int dd, float acc, float l, float M) {
        const int i = (r0 + x) / a.G;
        const size_t row = (size_t)i * Hq + g * a.G + (r0 + x - i * a.G);
        if (gridDim.z == 1) {
            Elem<T>::st(out + row * D + dd, acc / l);
        } else {
            float* dst = part + ((size_t)blockIdx.z * a.n_q * Hq + row) * (D + 2);
            dst[dd] = acc;
            if (dd == 0) { dst[D] = M; dst[D + 1] = l; }
        }
    });
}

// Workgroups per row tile: about kSlideWgs in all, every wave the same number of units where that can be.
constexpr int kSlideWgs = 512;
static int sliding_splits(int n_q, int n_k, int G, int Hkv, int window, int sinks) {
    const long long tiles = ((long long)n_q * G + kTileRows - 1) / kTileRows * Hkv;
    const long long near = std::min<long long>(n_k, (long long)window + std::min<long long>(n_q, (kTileRows + G - 1) / G + 1));
    const long long units = (near + kTileKeys - 1) / kTileKeys + (std::min<long long>(sinks, n_k) + kTileKeys - 1) / kTileKeys;
    const long long most = std::max<long long>(1, std::min<long long>(kMergeParts, kSlideWgs / tiles));
    const long long rounds = std::max<long long>(1, (units + kSlideWaves * most - 1) / (kSlideWaves * most));
    return (int)std::max<long long>(1, std::min(most, (units + kSlideWaves * rounds - 1) / (kSlideWaves * rounds)));
}

size_t sliding_workspace_floats(int n_q, int n_k, int Hq, int Hkv, int d, int window, int sinks, int dtype) {
    const int splits = sliding_splits(n_q, n_k, Hq / Hkv, Hkv, window, sinks);
    return splits > 1 ? (size_t)splits * n_q * Hq * (d + 2) : 0;
}

int launch_sliding_attn(const void* q, const void* k, const void* v, int n_q, int n_k, int Hq, int Hkv, int d, int window, int sinks, float scale, int dtype, void* out,
                        float* part, hipStream_t st) {
    const SlidingRows a{n_q, n_k, Hq / Hkv, Hkv, window, sinks, scale * 1.4426950408889634f};
    const int splits = sliding_splits(n_q, n_k, a.G, Hkv, window, sinks);
    const long long tiles = ((long long)n_q * a.G + kTileRows - 1) / kTileRows;
    const dim3 grid((unsigned)tiles, Hkv, splits);
#define SLIM_SLIDE(T, D) hipLaunchKernelGGL((sliding_rows_kernel<T, D>), grid, dim3(64 * kSlideWaves), 0, st, (const T*)q, (const T*)k, (const T*)v, a, (T*)out, part)
    if (dtype == SLIM_BF16) SLIM_SLIDE(bf16_t, 128);
    else if (d == 32) SLIM_SLIDE(float, 32);
    else if (d == 64) SLIM_SLIDE(float, 64);
    else SLIM_SLIDE(float, 128);
#undef SLIM_SLIDE
    const int rc = check_launch();
    return rc || splits == 1 ? rc : launch_merge_rows(part, splits, n_q * Hq, d, dtype, out, st);
}

}  // namespace slim
