// Attention of 16 query rows of one kv head by one wave, 32 keys at a time, where few rows meet many keys (device code).
//
// A row is a (query, query head of the kv head) pair, so that the query heads that share a kv head share its loads, whatever their number.
//   S^T[key, row] = K . Q^T      16x16x32 matrix instructions; A: the lane (l16, qr) = (lane % 16, lane / 16) holds channels qr * D/4 .. + D/4 of key l16, eight of
//                                them an instruction (any order of the channels will do that both operands have)
//   O^T[d, row]   = V^T . P^T    the lane holds for row l16 the weights of keys 4 qr .. 4 qr + 3 of both halves of the 32 keys: what S^T left it, so nothing moves
//                                between lanes but the maximum; V comes from LDS through the transposing read, four keys of one channel at a time
// The wave's V tile is its own: rows of D bfloat16, 16-byte piece c of key r at c ^ (r % (D / 8)), which spreads both the writes (16 keys, one piece) and the
// transposing reads (16 keys, two pieces) over all banks.  LDS serves a wave's accesses in order, so no barrier is needed.
//
// float32 rows run in the same instructions: a float is the sum of three bfloat16 (its 24 bits, cut into three times eight: the second is below 2^-7 of the float, the third below 2^-15),
// products of the terms are exact, and of the nine the three with a + b > 2 are left out: 2^-22 of the floats' product twice and 2^-30, in the worst case 2^-21 together, all with the
// product's own sign (random floats: 2^-21.3 at most; results 2 to 4 10^-7 from 64 bits).  What comes from 4 bits is a single bfloat16, exactly.
#pragma once
#include "slim_common.h"

namespace slim {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4* LdsB64;
typedef __attribute__((address_space(3))) bf16x8* LdsB128;

constexpr int kTileRows = 16, kTileKeys = 32;

// Maximum over the four lanes with the same lane % 16.  (The elements leave the swap's result as whole numbers first: __builtin_bit_cast of a vector's element reads the vector's
// first one.)
__device__ __forceinline__ float max_over_rows(float v) {
    const unsigned x = __builtin_bit_cast(unsigned, v);
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const unsigned a0 = a[0], a1 = a[1];
    const unsigned y = __builtin_bit_cast(unsigned, fmaxf(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1)));
    const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    const unsigned b0 = b[0], b1 = b[1];
    return fmaxf(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}

// Eight floats as bfloat16 terms: one, rounded to nearest; it and what is left, rounded to nearest (2^-17 of the float may be missing); or three that add up to the float.
template <int NT> __device__ __forceinline__ void bf16_terms(const float* f, bf16x8* t) {
    if constexpr (NT <= 2) {
        const uint4 w = Elem<bf16_t>::pack(f);
        t[0] = __builtin_bit_cast(bf16x8, w);
        if constexpr (NT == 2) {
            float r[8];
            Elem<bf16_t>::unpack(w, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = f[i] - r[i];
            t[1] = __builtin_bit_cast(bf16x8, Elem<bf16_t>::pack(r));
        }
    } else {
        static_assert(NT == 3, "one to three terms");
        uint32_t w[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t u[3][2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float r = f[2 * i + e];
#pragma unroll
                for (int a = 0; a < 3; ++a) {
                    u[a][e] = __builtin_bit_cast(uint32_t, r) & 0xffff0000u;
                    r -= __builtin_bit_cast(float, u[a][e]);
                }
            }
#pragma unroll
            for (int a = 0; a < 3; ++a) w[a][i] = u[a][0] >> 16 | u[a][1];
        }
#pragma unroll
        for (int a = 0; a < 3; ++a) t[a] = __builtin_bit_cast(bf16x8, make_uint4(w[a][0], w[a][1], w[a][2], w[a][3]));
    }
}
// Eight channels of a dense row of T as terms.
template <typename T, int NT> __device__ __forceinline__ void row_terms(const T* p, bf16x8* t) {
    if constexpr (sizeof(T) == 2) {
        static_assert(NT == 1, "a bfloat16 is one term");
        t[0] = *reinterpret_cast<const bf16x8*>(p);
    } else {
        float f[8];
        Elem<float>::unpack(*reinterpret_cast<const uint4*>(p), f);
        Elem<float>::unpack(*reinterpret_cast<const uint4*>(p + 4), f + 4);
        bf16_terms<NT>(f, t);
    }
}

template <typename T, int D> struct RowTile {
    static constexpr int NT = sizeof(T) == 2 ? 1 : 3;    // terms of an operand that is a T
    static constexpr int NP = sizeof(T) == 2 ? 2 : 3;    // and of the weights: one term alone, rounded by up to 2^-8, would be off as much as the bfloat16 output's own rounding
    static constexpr int KS = D / 32, DT = D / 16, CH = D / 8;
    static constexpr int kLdsBytes = kTileKeys * D * 2;  // of a wave's V tile
    bf16x8 q[NT][KS];
    f32x4 o[DT];                                         // channel dt * 16 + 4 qr + e of row l16
    float m, mc, l;                                      // of row l16: largest score, that in the base-2 domain, the lane's share of the sum

    __device__ __forceinline__ void begin(const T* q_row) {          // of row l16
        const int qr = (threadIdx.x & 63) >> 4;
        begin(q_row, [&](int j) { return qr * (D / 4) + j * 8; });
    }
    // channel(j): the lane's eight channels of step j, in another order than the above.
    template <typename F> __device__ __forceinline__ void begin(const T* q_row, F channel) {
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            bf16x8 t[NT];
            row_terms<T, NT>(q_row + channel(j), t);
#pragma unroll
            for (int a = 0; a < NT; ++a) q[a][j] = t[a];
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        m = -INFINITY;
        mc = l = 0.f;
    }
    // Scores of 16 keys, from zero.  The products of first terms and the others are summed apart: among the large sums these would be rounded to their last place each time.
    struct Scores {
        f32x4 first = {0.f, 0.f, 0.f, 0.f}, rest = {0.f, 0.f, 0.f, 0.f};
        __device__ __forceinline__ f32x4 sum() const {
            if constexpr (NT == 1) return first;
            else return first + rest;
        }
    };
    // += K . Q^T over the eight channels of step j; k: NK terms of them.
    template <int NK> __device__ __forceinline__ void add_scores(const bf16x8* k, int j, Scores& s) const {
#pragma unroll
        for (int a = NK - 1; a >= 0; --a)
#pragma unroll
            for (int b = NT - 1; b >= 0; --b)
                if (a + b == 0) s.first = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[a], q[b][j], s.first, 0, 0, 0);
                else if (a + b < 3) s.rest = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[a], q[b][j], s.rest, 0, 0, 0);
    }
    // Scores of 32 keys, -infinity for those that row l16 does not see -> weights 2^(c s - mc) relative to the running maximum, which O and the sum follow.  The maximum is rounded
    // into the base-2 domain once and the difference from it once, where it is small: an error of the former is common to all weights of the row, and what the
    // reference leaves behind is rescaled by the difference of the rounded ones.
    __device__ __forceinline__ void weigh(const f32x4* s, float c, float* w) {
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        mx = fmaxf(m, max_over_rows(mx));
        if (__any(mx > m)) {
            const float now = mx == -INFINITY ? 0.f : mx * c;        // (a row that has seen no key yet)
            const float al = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - now);
            l *= al;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] *= al;
            m = mx;
            mc = now;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = __builtin_amdgcn_exp2f(fmaf(s[0][e], c, -mc));
            w[4 + e] = __builtin_amdgcn_exp2f(fmaf(s[1][e], c, -mc));
        }
        l += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    }
    // Byte offset of 16-byte piece c of key r in the V tile.
    __device__ static __forceinline__ unsigned v_piece(int r, int c) { return (unsigned)(r * (D * 2) + ((c ^ (r & (CH - 1))) << 4)); }
    // o += V^T . P^T with the term of V (NV in all, this one is number a) that lies in the wave's tile.
    template <int NV> __device__ __forceinline__ void add_values(const bf16x8* p, int a, unsigned lds_tile) {
        const int lane = threadIdx.x & 63, s16 = lane & 15, r = 4 * (lane >> 4) + (s16 >> 2);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) add_channels<NV>(p, a, dt, lds_tile + v_piece(r, dt * 2 + ((s16 & 3) >> 1)) + (s16 & 1) * 8);
    }
    // The same for channels 16 dt ..; at: where the lane reads them.
    template <int NV> __device__ __forceinline__ void add_channels(const bf16x8* p, int a, int dt, unsigned at) { add_read<NV>(p, a, dt, read_channels(at)); }
    __device__ static __forceinline__ bf16x8 read_channels(unsigned at) {
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsB64)at);
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsB64)(at + 16 * D * 2));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    template <int NV> __device__ __forceinline__ void add_read(const bf16x8* p, int a, int dt, bf16x8 v) {
        if constexpr (NT == 1) {
#pragma unroll
            for (int b = NP - 1; b >= 0; --b) o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[b], o[dt], 0, 0, 0);
        } else {                                         // float32: the terms' sum is rounded into the running values once
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = NP - 1; b >= 0; --b)
                if (a + b < 3) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[b], x, 0, 0, 0);
            o[dt] += x;
        }
    }
    // What the weights of row l16 are relative to, in the base-2 domain.
    __device__ __forceinline__ float reference() const { return m == -INFINITY ? m : mc; }
    // The row's sum in each of its four lanes, at the end.
    __device__ __forceinline__ void finish_sum() {
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
    }
};

// The results of a workgroup's NW waves for the same rows, merged: store(row, channel, values, sum, maximum) is called for the first `rows` of them.  lds: the waves' V tiles, which
// hold 16 rows of D floats each as well (16-byte pieces turned by the row).
template <typename T, int D, int NW, typename F> __device__ __forceinline__ void merge_waves(RowTile<T, D>& t, unsigned char* lds, int rows, F store, const int tid = threadIdx.x) {
    typedef RowTile<T, D> Tile;
    static_assert(Tile::kLdsBytes == kTileRows * D * 4, "O fits the V tile");
    __shared__ float ws_m[NW][kTileRows], ws_l[NW][kTileRows];
    const int lane = tid & 63, l16 = lane & 15, qr = lane >> 4, wave = tid >> 6;
    t.finish_sum();
    if (lane < kTileRows) { ws_m[wave][lane] = t.reference(); ws_l[wave][lane] = t.l; }
    float* mine = reinterpret_cast<float*>(lds + wave * Tile::kLdsBytes);
#pragma unroll
    for (int dt = 0; dt < Tile::DT; ++dt) *reinterpret_cast<f32x4*>(mine + l16 * D + (((dt * 4 + qr) ^ (l16 & (D / 4 - 1))) << 2)) = t.o[dt];
    __syncthreads();
    for (int i = tid; i < rows * D; i += 64 * NW) {
        const int r = i / D, dd = i % D;
        float M = -INFINITY, acc = 0.f, l = 0.f;
#pragma unroll
        for (int x = 0; x < NW; ++x) M = fmaxf(M, ws_m[x][r]);
#pragma unroll
        for (int x = 0; x < NW; ++x) {
            const float lx = ws_l[x][r], w = lx == 0.f ? 0.f : __builtin_amdgcn_exp2f(ws_m[x][r] - M);
            acc += w * reinterpret_cast<const float*>(lds + x * Tile::kLdsBytes)[r * D + (((dd >> 2) ^ (r & (D / 4 - 1))) << 2) + (dd & 3)];
            l += w * lx;
        }
        store(r, dd, acc, l, M);
    }
}

// Rows of partial results (D weighted values, maximum, sum) of up to kMergeParts splits -> rows of T: sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i.  part[split][row][D + 2].
constexpr int kMergeParts = 128;
int launch_merge_rows(const float* part, int n_parts, int rows, int head_dim, int dtype, void* out, hipStream_t st);

}  // namespace slim
