// A Key-Value cache in 4 bits: blocks written into their slots and read back, and a decoded token's attention over the slots as they lie (Section 4.3's pools, with
// 17/64 of the bytes to hold and to swap).
//
// A row is cut into groups of 32 channels.  A group has one power of two 2^e, e the smallest for which its largest magnitude stays below 7 * 2^e (so that rounding to
// 6 * 2^e, the largest value, is off by no more than half the step that the format would have there), and a code per channel: sign and the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6
// times 2^e, ties to the even code.  The values are bfloat16 and float32 numbers exactly, and both directions are single instructions for two channels
// (v_cvt_scalef32_pk_*), so what is read costs half an instruction per channel and no correction for a zero point.
// e is kept in [-125, 125]: every value but zero is a normal number.  A group with an infinity or a NaN is stored as byte 255, which the instruction that reads makes NaN.
//
// Layout of a slot (block B, H kv heads, heads of d): Keys' codes [H, B, d / 2], Values' codes, Keys' e + 127 [H, B, d / 32], Values' -- a kv head's rows lie together, as the
// attention reads them.
#include "row_tile.h"
#include <algorithm>
#include <mutex>

namespace slim {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// What lies where in a slot, for one kv head.
struct Kv4Head {
    size_t k, v, ks, vs;
    __device__ __forceinline__ Kv4Head(int g, int block, int Hkv, int d) {
        const size_t rows = (size_t)Hkv * block, at = (size_t)g * block;
        k = at * (d / 2);
        v = (rows + at) * (d / 2);
        ks = rows * d + at * (d / 32);
        vs = rows * d + (rows + at) * (d / 32);
    }
};

// Eight channels (four bytes of codes) as bfloat16; scale: 2^e.
__device__ __forceinline__ bf16x8 kv4_to_bf16(uint32_t c, float scale) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
    const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// ---- written and read back
// A wave takes 64 / (D / 8) rows of one kv head, Keys or Values, at a time, 8 channels a lane (four lanes a group), kSteps times in a row: what it reads is whole rows, what it writes
// lies together.  Bound by memory: 32768 tokens of 8 heads of 128 in bf16, in buffers that no cache holds, written 33.9 us (170 MB, 5.0 TB/s; a copy of that size on this card 5.2), read back
// 24.8 (6.9).  Past the caches go the rows that are read (without 38.0 us) and those that are written (without 51.8: the lines push out the codes), but not the codes that are
// written, four bytes a lane (with the read behind it 82 us for both instead of 59); four steps in a row instead of two 33.8 and 26.2.
constexpr int kSteps = 2;
struct Kv4Rows {
    const unsigned char* pool;
    size_t slot_bytes, layer_offset;
    const int* slot_of_block;                            // null: block b lies in slot b
    const int* blocks;                                   // read: list of blocks, null: 0, 1, ..
    int n_slots, n_blocks, block, Hkv, first, n;         // first, n: written: tokens first .. first + n - 1; read: n = prompt tokens
    int list, n_rows;                                    // read: entries of the list, rows that the output has room for
    int ldk, ldv;
};

template <typename T, int D>
__global__ void __launch_bounds__(256) kv4_write_kernel(const T* __restrict__ K, const T* __restrict__ V, Kv4Rows a) {
    constexpr int PC = D / 8, RPW = 64 / PC;             // lanes a row, rows a step
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, piece = lane % PC;
    const bool value = blockIdx.z;
    const int g = blockIdx.y;
    const int i0 = (blockIdx.x * 4 + wave) * (RPW * kSteps) + lane / PC;
    const T* src = value ? V + (size_t)g * D : K + (size_t)g * D;
    const size_t ld = value ? a.ldv : a.ldk;
    const Kv4Head at(g, a.block, a.Hkv, D);
    float f[kSteps][8];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const T* p = src + (size_t)min(i0 + s * RPW, a.n - 1) * ld + piece * 8;
        Elem<T>::unpack(load_stream16(p), f[s]);
        if constexpr (sizeof(T) == 4) Elem<T>::unpack(load_stream16(p + 4), f[s] + 4);
    }
    int b = (a.first + i0) / a.block, r = a.first + i0 - b * a.block;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        uint32_t mx = 0;                                 // magnitudes compare as whole numbers, NaN above infinity
#pragma unroll
        for (int i = 0; i < 8; ++i) mx = max(mx, __builtin_bit_cast(uint32_t, f[s][i]) & 0x7fffffffu);
        mx = max(mx, (uint32_t)__shfl_xor((int)mx, 1, 64));
        mx = max(mx, (uint32_t)__shfl_xor((int)mx, 2, 64));
        // + a quarter of a mantissa: from 1.75 times a power of two on the next power counts
        const int byte = mx >= 0x7f800000u ? 255 : min(max((int)((mx + (1u << 21)) >> 23) - 2, 2), 252);
        const float scale = kv4_scale(byte);
        uint32_t code = 0;
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f[s][0], f[s][1], scale, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f[s][2], f[s][3], scale, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f[s][4], f[s][5], scale, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, f[s][6], f[s][7], scale, 3);
        if (byte == 255) code = 0;
        if (i0 + s * RPW < a.n) {
            const int slot = a.slot_of_block ? a.slot_of_block[b] : b;
            if (slot >= 0 && slot < a.n_slots) {
                unsigned char* dst = const_cast<unsigned char*>(a.pool) + (size_t)slot * a.slot_bytes + a.layer_offset;
                *reinterpret_cast<uint32_t*>(dst + (value ? at.v : at.k) + (size_t)r * (D / 2) + piece * 4) = code;
                if (piece % 4 == 0) dst[(value ? at.vs : at.ks) + (size_t)r * (D / 32) + piece / 4] = (unsigned char)byte;
            }
        }
        r += RPW;
        while (r >= a.block) { r -= a.block; ++b; }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(256) kv4_read_kernel(T* __restrict__ K, T* __restrict__ V, Kv4Rows a) {
    constexpr int PC = D / 8, RPW = 64 / PC;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, piece = lane % PC;
    const bool value = blockIdx.z;
    const int g = blockIdx.y;
    const long long o0 = ((long long)blockIdx.x * 4 + wave) * (RPW * kSteps) + lane / PC;   // row of the output
    T* out = value ? V + (size_t)g * D : K + (size_t)g * D;
    const size_t ld = value ? a.ldv : a.ldk;
    const Kv4Head at(g, a.block, a.Hkv, D);
    int i = (int)(o0 / a.block), r = (int)(o0 - (long long)i * a.block);
    uint32_t code[kSteps], byte[kSteps];
    bool have[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        have[s] = false;
        if (i < a.list && o0 + s * RPW < a.n_rows) {
            const int b = a.blocks ? a.blocks[i] : i;
            if (b >= 0 && b < a.n_blocks && (long long)b * a.block + r < a.n) {
                const int slot = a.slot_of_block ? a.slot_of_block[b] : b;
                if (slot >= 0 && slot < a.n_slots) {
                    const unsigned char* src = a.pool + (size_t)slot * a.slot_bytes + a.layer_offset;
                    code[s] = *reinterpret_cast<const uint32_t*>(src + (value ? at.v : at.k) + (size_t)r * (D / 2) + piece * 4);
                    byte[s] = src[(value ? at.vs : at.ks) + (size_t)r * (D / 32) + piece / 4];
                    have[s] = true;
                }
            }
        }
        r += RPW;
        while (r >= a.block) { r -= a.block; ++i; }
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        if (!have[s]) continue;
        const uint4 v = __builtin_bit_cast(uint4, kv4_to_bf16(code[s], kv4_scale(byte[s])));
        T* dst = out + (size_t)(o0 + s * RPW) * ld + piece * 8;
        if constexpr (sizeof(T) == 2) {
            store_stream16(dst, v);
        } else {
            float f[8];
            Elem<bf16_t>::unpack(v, f);
            store_stream16(dst, Elem<float>::pack(f));
            store_stream16(dst + 4, Elem<float>::pack(f + 4));
        }
    }
}

int launch_kv4_write(const void* k, const void* v, int ldk, int ldv, int first, int n, int Hkv, int d, int block, int dtype, const int* slot_of_block, int n_blocks,
                     void* pool, int n_slots, size_t slot_bytes, size_t layer_offset, hipStream_t st) {
    const Kv4Rows a{(const unsigned char*)pool, slot_bytes, layer_offset, slot_of_block, nullptr, n_slots, n_blocks, block, Hkv, first, n, 0, 0, ldk, ldv};
    const int per_wg = 4 * kSteps * 512 / d;
    const dim3 grid((n + per_wg - 1) / per_wg, Hkv, 2);
#define SLIM_KV4(T, D) hipLaunchKernelGGL((kv4_write_kernel<T, D>), grid, dim3(256), 0, st, (const T*)k, (const T*)v, a)
#define SLIM_KV4_D(T) do { if (d == 32) SLIM_KV4(T, 32); else if (d == 64) SLIM_KV4(T, 64); else SLIM_KV4(T, 128); } while (0)
    if (dtype == SLIM_BF16) SLIM_KV4_D(bf16_t); else SLIM_KV4_D(float);
#undef SLIM_KV4
    return check_launch();
}

int launch_kv4_read(const void* pool, int n_slots, size_t slot_bytes, size_t layer_offset, const int* slot_of_block, const int* blocks, int list, int n_blocks, int block,
                    int n_tokens, int Hkv, int d, int dtype, void* k, void* v, int n_rows, int ldk, int ldv, hipStream_t st) {
    const Kv4Rows a{(const unsigned char*)pool, slot_bytes, layer_offset, slot_of_block, blocks, n_slots, n_blocks, block, Hkv, 0, n_tokens, list, n_rows, ldk, ldv};
    const int per_wg = 4 * kSteps * 512 / d;
    const long long rows = std::min<long long>(n_rows, blocks ? (long long)list * block : n_tokens);
    const dim3 grid((unsigned)((rows + per_wg - 1) / per_wg), Hkv, 2);
#define SLIM_KV4(T, D) hipLaunchKernelGGL((kv4_read_kernel<T, D>), grid, dim3(256), 0, st, (T*)k, (T*)v, a)
    if (dtype == SLIM_BF16) SLIM_KV4_D(bf16_t); else SLIM_KV4_D(float);
#undef SLIM_KV4
#undef SLIM_KV4_D
    return check_launch();
}

// ---- attention of one decoded token
// A loaded value whose first use is here: left alone, the compiler moves the shift that makes a scale of it behind the load, in front of the loop's end, and with it the wait.
__device__ __forceinline__ uint32_t used_here(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
}

// The units of 32 keys of the slots and of the response are dealt to the waves of gridDim.x workgroups per kv head; each workgroup leaves a partial result of the kv head's query
// heads, or, alone, the output.  The registers of a unit's codes are requested anew as soon as they are used.
// Bound, with many slots, by memory and by nine vector instructions (conversions, softmax) a matrix instruction: 2048 slots of 64 tokens, 32 / 8 heads, 28 us for 135 MB (4.8 TB/s; the
// loads alone 25); with few by the trips to memory one behind the other (slot map, codes, partial results): 128 slots 7.6 us and 2.2 for the merge.  Two units a turn: the same times.
constexpr int kQ4D = 128;
template <typename T, int NW>
__global__ void __launch_bounds__(64 * NW) decode_attn_kv4_kernel(
    const T* __restrict__ q, const unsigned char* __restrict__ pool, size_t slot_bytes, size_t layer_offset, const int* __restrict__ block_of_slot, int n_slots, int block,
    int n_prompt, const T* __restrict__ k_resp, const T* __restrict__ v_resp, int n_resp, int Hq, int Hkv, float scale_log2e, float* __restrict__ part, T* __restrict__ out) {
    constexpr int D = kQ4D;
    typedef RowTile<T, D> Tile;
    constexpr int NT = Tile::NT, NP = Tile::NP;
    extern __shared__ __align__(16) unsigned char lds[];
    const int g = blockIdx.y, lane = threadIdx.x & 63, l16 = lane & 15, qr = lane >> 4, G = Hq / Hkv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned tile = (unsigned)(uintptr_t)lds + wave * Tile::kLdsBytes;
    const int nb = (n_prompt + block - 1) / block, per_slot = (block + kTileKeys - 1) / kTileKeys;
    const int n_in_slots = n_slots * per_slot, n_units = n_in_slots + (n_resp + kTileKeys - 1) / kTileKeys, step = gridDim.x * NW;
    const Kv4Head head(g, block, Hkv, D);

    // The wave's units are u0, u0 + step, ..; those of a free slot or behind the end of a short block hold no key and are passed over.  64 of them are looked up at once, one a lane:
    // looked up one by one, each waited for block_of_slot.
    const int u0 = (int)blockIdx.x * NW + wave;
    int batch = u0, u_slot = 0, u_row = 0, u_rows = 0;   // the lane's unit: slot, first row, rows
    unsigned long long left = 0;                         // lanes whose units hold keys and have not been taken
    auto look_up = [&]() {
        const long long u = batch + (long long)lane * step;
        int b = -1;
        if (u < n_in_slots) {
            u_slot = (int)u / per_slot;
            u_row = ((int)u - u_slot * per_slot) * kTileKeys;
            b = block_of_slot[u_slot];
        }
        u_rows = b >= 0 && b < nb ? min(kTileKeys, min(block, n_prompt - b * block) - u_row) : 0;
        left = __ballot(u_rows > 0);
    };
    int rows = 0, c0 = 0;
    const unsigned char* base = nullptr;                 // of the unit's slot
    auto find = [&]() {                                  // the next unit; false: none is left
        while (!left) {
            if ((long long)batch + 64ll * step >= n_in_slots) return false;
            batch += 64 * step;
            look_up();
        }
        const int i = __builtin_ctzll(left);
        left &= left - 1;
        rows = __builtin_amdgcn_readlane(u_rows, i);
        c0 = __builtin_amdgcn_readlane(u_row, i);
        base = pool + (size_t)__builtin_amdgcn_readlane(u_slot, i) * slot_bytes + layer_offset;
        return true;
    };
    look_up();
    uint4 kx[2], vx[2];
    uint32_t ks[2], vs[2];                               // the e + 127 of a key's four groups
    // Addresses: a wave-uniform base and a 32-bit offset of the lane, the same for Keys and Values.  Rows behind the last key repeat it: their weight is 0.
    unsigned off[2];
    auto load_k = [&]() {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned r = min(l16 + 16 * h, rows - 1);
            off[h] = r * 4;
            kx[h] = load_stream16(base + head.k + (size_t)c0 * (D / 2) + (r * (D / 2) + qr * 16));
            ks[h] = *reinterpret_cast<const uint32_t*>(base + head.ks + (size_t)c0 * (D / 32) + off[h]);
        }
    };
    auto load_v = [&]() {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            vx[h] = load_stream16(base + head.v + (size_t)c0 * (D / 2) + (off[h] * 16 + qr * 16));
            vs[h] = *reinterpret_cast<const uint32_t*>(base + head.vs + (size_t)c0 * (D / 32) + off[h]);
        }
    };
    // the lane's group of a key
    auto scale_of = [&](uint32_t groups) { return kv4_scale(__builtin_amdgcn_ubfe(used_here(groups), qr * 8, 8)); };
    bool more = find();
    if (more) { load_k(); load_v(); }
    Tile t;
    t.begin(q + (size_t)(g * G + min(l16, G - 1)) * D);
    // the Query fragments are waited for here: waited for in the loop, they take the wait for the codes requested meanwhile with them in every turn
#pragma unroll
    for (int b = 0; b < NT; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(t.q[b][j]));
    float w[8];
    bf16x8 p[NP];
    auto masked = [&](f32x4* s, int have) {
        if (have == kTileKeys) return;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = s[h][e];
                s[h][e] = h * 16 + qr * 4 + e < have ? x : -INFINITY;
            }
    };
    while (more) {
        const int have = rows;
        more = find();                                   // none left: the last unit is requested once more, and not used
        f32x4 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            typename Tile::Scores sum;
            const uint32_t c[4] = {kx[h].x, kx[h].y, kx[h].z, kx[h].w};
            const float sc = scale_of(ks[h]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8 k = kv4_to_bf16(c[j], sc);
                t.template add_scores<1>(&k, j, sum);
            }
            s[h] = sum.sum();
        }
        __builtin_amdgcn_sched_barrier(0);
        load_k();                                        // the next unit's Keys fly under this one's Values
        __builtin_amdgcn_sched_barrier(0);
        masked(s, have);
        t.weigh(s, scale_log2e, w);
        bf16_terms<NP>(w, p);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t c[4] = {vx[h].x, vx[h].y, vx[h].z, vx[h].w};
            const float sc = scale_of(vs[h]);
#pragma unroll
            for (int j = 0; j < 4; ++j) *(LdsB128)(tile + Tile::v_piece(l16 + 16 * h, qr * 4 + j)) = kv4_to_bf16(c[j], sc);
        }
        __builtin_amdgcn_sched_barrier(0);
        load_v();
        __builtin_amdgcn_sched_barrier(0);
        t.template add_values<1>(p, 0, tile);
    }
    // response tokens: dense rows of T
    const size_t row_stride = (size_t)Hkv * D;
    for (int ui = n_in_slots + ((u0 - n_in_slots) % step + step) % step; ui < n_units; ui += step) {
        const int first = (ui - n_in_slots) * kTileKeys, have = min(kTileKeys, n_resp - first);
        f32x4 s[2];
        size_t at[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            typename Tile::Scores sum;
            at[h] = (size_t)(first + min(l16 + 16 * h, have - 1)) * row_stride + (size_t)g * D + qr * 32;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bf16x8 k[NT];
                row_terms<T, NT>(k_resp + at[h] + j * 8, k);
                t.template add_scores<NT>(k, j, sum);
            }
            s[h] = sum.sum();
        }
        masked(s, have);
        t.weigh(s, scale_log2e, w);
        bf16_terms<NP>(w, p);
        bf16x8 v[2][4][NT];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) row_terms<T, NT>(v_resp + at[h] + j * 8, v[h][j]);
#pragma unroll
        for (int a = 0; a < NT; ++a) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) *(LdsB128)(tile + Tile::v_piece(l16 + 16 * h, qr * 4 + j)) = v[h][j][a];
            t.template add_values<NT>(p, a, tile);
        }
    }
    merge_waves<T, D, NW>(t, lds, G, [&](int h, int dd, float acc, float l, float M) {
        const int row = g * G + h;
        if (gridDim.x == 1) {
            Elem<T>::st(out + (size_t)row * D + dd, l == 0.f ? 0.f : acc / l);
        } else {
            float* dst = part + ((size_t)blockIdx.x * Hq + row) * (D + 2);
            dst[dd] = acc;
            if (dd == 0) { dst[D] = M; dst[D + 1] = l; }
        }
    });
}

// A row takes NG groups of D / 4 lanes, four channels each; group j has the partials j, j + NG, ..  Everything is requested at once: the launch is one trip to memory.
constexpr int kMergeMost = 16;                           // partials of a group
template <typename T, int D, int NG>
__global__ void __launch_bounds__(256) merge_rows_kernel(const float* __restrict__ part, int n_parts, int rows, T* __restrict__ out) {
    constexpr int LN = D / 4, PER_WG = 256 / (LN * NG);
    static_assert(NG * kMergeMost >= (NG == 1 ? 1 : kMergeParts) && PER_WG >= 1, "all partials, within a workgroup");
    __shared__ float ms[NG][PER_WG], ls[NG][PER_WG];
    __shared__ __align__(16) float os[NG][PER_WG][D];
    const int tid = threadIdx.x, lane = tid % LN, grp = tid / LN % NG, x = tid / (LN * NG), row = blockIdx.x * PER_WG + x;
    const float* p = part + (size_t)min(row, rows - 1) * (D + 2);
    const size_t step = (size_t)rows * (D + 2);
    float m[kMergeMost], l[kMergeMost], M = -INFINITY;
    float2 v[kMergeMost][2];                             // (rows of D + 2 floats are aligned to eight bytes)
#pragma unroll
    for (int i = 0; i < kMergeMost; ++i) {
        const int at = grp + i * NG;
        m[i] = -INFINITY;
        l[i] = 0.f;
        v[i][0] = v[i][1] = make_float2(0.f, 0.f);
        if (at < n_parts) {
            const float* r = p + at * step;
            const float2 st = *reinterpret_cast<const float2*>(r + D);
            v[i][0] = *reinterpret_cast<const float2*>(r + lane * 4);
            v[i][1] = *reinterpret_cast<const float2*>(r + lane * 4 + 2);
            m[i] = st.x;
            l[i] = st.y;
        }
    }
#pragma unroll
    for (int i = 0; i < kMergeMost; ++i) M = fmaxf(M, m[i]);
    if constexpr (NG > 1) {
        if (lane == 0) ms[grp][x] = M;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NG; ++i) M = fmaxf(M, ms[i][x]);
    }
    float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kMergeMost; ++i) {
        const float w = l[i] == 0.f ? 0.f : __builtin_amdgcn_exp2f(m[i] - M);      // a partial without keys has no weight
        sum += w * l[i];
        o[0] += w * v[i][0].x;
        o[1] += w * v[i][0].y;
        o[2] += w * v[i][1].x;
        o[3] += w * v[i][1].y;
    }
    if constexpr (NG > 1) {
        if (lane == 0) ls[grp][x] = sum;
        *reinterpret_cast<f32x4*>(&os[grp][x][lane * 4]) = f32x4{o[0], o[1], o[2], o[3]};
        __syncthreads();
        if (grp != 0) return;
#pragma unroll
        for (int g = 1; g < NG; ++g) {
            sum += ls[g][x];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += os[g][x][lane * 4 + e];
        }
    }
    if (row >= rows) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) Elem<T>::st(out + (size_t)row * D + lane * 4 + e, sum == 0.f ? 0.f : o[e] / sum);
}

int launch_merge_rows(const float* part, int n_parts, int rows, int d, int dtype, void* out, hipStream_t st) {
#define SLIM_MERGE(T, D, NG) do { constexpr int per = 256 / (D / 4 * NG); \
        hipLaunchKernelGGL((merge_rows_kernel<T, D, NG>), dim3((rows + per - 1) / per), dim3(256), 0, st, part, n_parts, rows, (T*)out); } while (0)
#define SLIM_MERGE_D(T, D) do { if (n_parts <= kMergeMost) SLIM_MERGE(T, D, 1); else SLIM_MERGE(T, D, 8); } while (0)
    if (dtype == SLIM_BF16) SLIM_MERGE_D(bf16_t, 128);
    else if (d == 32) SLIM_MERGE_D(float, 32);
    else if (d == 64) SLIM_MERGE_D(float, 64);
    else SLIM_MERGE_D(float, 128);
#undef SLIM_MERGE_D
#undef SLIM_MERGE
    return check_launch();
}

// Workgroups per kv head and waves of a workgroup: every wave the same number of units where that can be, no more workgroups than the caller's workspace has room for (one partial per
// slot and per 64 response tokens).  256 workgroups of eight waves where that gives every wave a unit, else up to 512 of four; us, 32 / 8 heads, blocks of 64 tokens: 64 slots 8.5 / 8.2,
// 128 9.6 / 10.0, 512 13.5 / 14.9, 2048 30.3 / 32.2, 4096 51.6 / 53.7 (its loads alone 45); 512 of eight waves, which the registers keep from running together, 2048 slots 34.8.
struct Q4Plan { int waves, parts; };
static Q4Plan kv4_plan(int n_slots, int block, int n_resp, int Hkv) {
    const long long units = (long long)n_slots * ((block + kTileKeys - 1) / kTileKeys) + (n_resp + kTileKeys - 1) / kTileKeys;
    const int waves = units * Hkv >= 8 * 256 ? 8 : 4;
    const long long most = std::min<long long>(std::max(16, std::min(kMergeParts, (waves == 8 ? 256 : 512) / Hkv)), (long long)n_slots + (n_resp + 63) / 64);
    const long long rounds = std::max<long long>(1, (units + waves * most - 1) / (waves * most));
    return {waves, (int)std::max<long long>(1, std::min(most, (units + waves * rounds - 1) / (waves * rounds)))};
}

template <typename T, int NW>
static int launch_q4(const void* q, const void* pool, size_t slot_bytes, size_t layer_offset, const int* block_of_slot, int n_slots, int block, int n_prompt, const void* k_resp,
                     const void* v_resp, int n_resp, int Hq, int Hkv, float sl, void* out, float* part, int parts, hipStream_t st) {
    constexpr int smem = NW * RowTile<T, kQ4D>::kLdsBytes;
    if (smem >= 1 << 16) {
        static std::once_flag once;
        static hipError_t err = hipSuccess;
        std::call_once(once, [&] { err = hipFuncSetAttribute((const void*)decode_attn_kv4_kernel<T, NW>, hipFuncAttributeMaxDynamicSharedMemorySize, smem); });
        if (err != hipSuccess) return set_hip_error(err);
    }
    hipLaunchKernelGGL((decode_attn_kv4_kernel<T, NW>), dim3(parts, Hkv), dim3(64 * NW), smem, st, (const T*)q, (const unsigned char*)pool, slot_bytes, layer_offset, block_of_slot,
                       n_slots, block, n_prompt, (const T*)k_resp, (const T*)v_resp, n_resp, Hq, Hkv, sl, part, (T*)out);
    return check_launch();
}

int launch_decode_attn_kv4(const void* q, const void* pool, size_t slot_bytes, size_t layer_offset, const int* block_of_slot, int n_slots, int block, int n_prompt,
                           const void* k_resp, const void* v_resp, int n_resp, int Hq, int Hkv, float scale, int dtype, void* out, float* part, hipStream_t st) {
    const float sl = scale * 1.4426950408889634f;
    if (n_slots == 0) block = 1;
    const Q4Plan plan = kv4_plan(n_slots, block, n_resp, Hkv);
#define SLIM_Q4(T, NW) launch_q4<T, NW>(q, pool, slot_bytes, layer_offset, block_of_slot, n_slots, block, n_prompt, k_resp, v_resp, n_resp, Hq, Hkv, sl, out, part, plan.parts, st)
    const int rc = dtype == SLIM_BF16 ? (plan.waves == 8 ? SLIM_Q4(bf16_t, 8) : SLIM_Q4(bf16_t, 4)) : plan.waves == 8 ? SLIM_Q4(float, 8) : SLIM_Q4(float, 4);
#undef SLIM_Q4
    return rc || plan.parts == 1 ? rc : launch_merge_rows(part, plan.parts, Hq, kQ4D, dtype, out, st);
}

}  // namespace slim
