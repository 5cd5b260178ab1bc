// A Key-Value cache in 8 bits for a batch of requests: rows written into the slots that a map names, read back, and attention of each request's last tokens over its blocks where they lie.
//
// A slot holds, for each kv head, one power of two 2^e for the Keys of the block's rows and one for the Values', and a byte per channel: sign, four bits of exponent (bias 7), three of
// mantissa, largest 448, 127 not a number.  e is the smallest for which no magnitude is above 448 * 2^e, kept in [-117, 119], so that what a byte stands for is a bfloat16 and a
// float32 number exactly and zero or a normal one.  Both directions are single instructions for two channels (v_cvt_scalef32_pk_*).
//
// Layout of a slot (block B, H kv heads, heads of d): Keys' codes [H, B, d], Values' codes, e + 127 of Keys and Values [H, 2] -- a kv head's rows lie together, as the attention
// reads them.
#include "row_tile.h"
#include "batch.h"
#include <algorithm>
#include <mutex>
#include <type_traits>

namespace slim {

typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kKv8ByteLow = 10, kKv8ByteHigh = 246;      // e + 127 of -117 and 119
constexpr uint32_t kKv8NaN = 0x7f;

// What lies where in a slot, for one kv head.
struct Kv8Head {
    size_t k, v, e;
    __device__ __forceinline__ Kv8Head(int g, int block, int Hkv, int d) {
        const size_t rows = (size_t)Hkv * block, at = (size_t)g * block;
        k = at * d;
        v = (rows + at) * d;
        e = 2 * rows * d + 2 * g;
    }
};

__device__ __forceinline__ float kv8_power(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// Eight channels as bfloat16; power: 2^e.
__device__ __forceinline__ bf16x8 kv8_to_bf16(uint2 c, float power) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, power, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, power, true);
    const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, power, false), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, power, true);
    return bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}
// The same as float16.
__device__ __forceinline__ f16x8 kv8_to_f16(uint2 c, float power) {
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.x, power, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.x, power, true);
    const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.y, power, false), e = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.y, power, true);
    return f16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}
// Four finite floats as codes relative to 2^e, 448 for what is above.
__device__ __forceinline__ uint32_t kv8_codes(const float* f, float power) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_fmed3f(f[i], -448.f * power, 448.f * power);
    i16x2 c = {0, 0};
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, y[0], y[1], power, false);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, y[2], y[3], power, true);
    return __builtin_bit_cast(uint32_t, c);
}

// ---- written
// A run is a stretch of rows whose places follow each other in one block; its largest magnitude gives the exponent, and with it the codes.  Where rows in front of the run are in the block
// already, the larger exponent of both holds, and where it grows they are rounded again.
// A workgroup takes the runs that begin within its `chunk` rows of the map, for Keys or Values of `heads` kv heads.  A run of more than kKv8Short rows is the whole workgroup's, head by head:
// its rows stay in registers, up to kKv8Keep passes of them, and the next head's are on their way.  Shorter ones, the new tokens of a step, are a wave's, for as many heads as it has
// rows' lanes for (64 / (D / 8)).  Rows, old exponent and the run's length are requested together: two trips to memory.
// Bound by memory where there are many rows: 26381 of 24 prompts, 8 heads of 128, 161 MB, 41 us, 3.9 TB/s (a copy of as much takes 32); by the trips where there are few: 256 new tokens
// 5.4 us, 3 us of which a launch costs, and 10.4 where they raise their blocks' exponents.
constexpr int kKv8Keep = 4, kKv8Short = 8;
struct Kv8Write {
    const int* row_slot;
    unsigned char* pool;
    size_t slot_bytes, layer_offset;
    int n_rows, n_places, block, Hkv, ldk, ldv, chunk, heads;      // n_places: of the pool, n_slots * block; heads: of a workgroup, a divisor of 64 / (D / 8)
    Divide by_block;
};

// Largest finite magnitude (magnitudes compare alike as whole numbers).
__device__ __forceinline__ uint32_t largest(const float* f, uint32_t m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t x = __builtin_bit_cast(uint32_t, f[i]) & 0x7fffffffu;
        m = max(m, x >= 0x7f800000u ? 0u : x);
    }
    return m;
}
// e + 127 for the largest magnitude m: from just above 1.75 times a power of two on it counts as the next power.
__device__ __forceinline__ uint32_t exponent_byte(uint32_t m) { return (uint32_t)min(max((int)((m + 0x1fffffu) >> 23) - 8, kKv8ByteLow), kKv8ByteHigh); }
// Eight floats -> their codes.
__device__ __forceinline__ uint2 kv8_eight(const float* f, float power) {
    uint2 code = make_uint2(kv8_codes(f, power), kv8_codes(f + 4, power));
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) odd |= !(fabsf(f[i]) < INFINITY);
    if (odd) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(fabsf(f[i]) < INFINITY)) {
                uint32_t& w = i < 4 ? code.x : code.y;
                w = (w & ~(0xffu << (i % 4 * 8))) | kKv8NaN << (i % 4 * 8);
            }
    }
    return code;
}
// `bytes` codes, a multiple of 8, rounded again relative to a power that is 2^by times as large; by thread tid of n.
__device__ __forceinline__ void kv8_round_again(unsigned char* codes, size_t bytes, uint32_t by, int tid, int n) {
    const float up = kv8_power(127 - min(by, 100u));     // (a hundred and more: nothing is left but zeros)
    for (size_t i = (size_t)tid * 8; i < bytes; i += (size_t)n * 8) {
        uint2 c = *reinterpret_cast<const uint2*>(codes + i);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            uint32_t& w = x ? c.y : c.x;
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, up, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, up, true);
            const float f[4] = {lo[0], lo[1], hi[0], hi[1]};
            uint32_t now = kv8_codes(f, 1.f);
#pragma unroll
            for (int y = 0; y < 4; ++y)
                if ((w >> (8 * y) & 0x7fu) == kKv8NaN) now = (now & ~(0xffu << (8 * y))) | kKv8NaN << (8 * y);
            w = now;
        }
        *reinterpret_cast<uint2*>(codes + i) = c;
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(256) kv8_write_kernel(const T* __restrict__ K, const T* __restrict__ V, Kv8Write a) {
    constexpr int PC = D / 8, RPP = 256 / PC, HEADS = 64 / PC, NV = sizeof(T) / 2;      // lanes a row, rows a pass, heads of a wave, 16-byte loads a lane
    __shared__ uint32_t most_of[2][4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), piece = tid % PC, row = tid / PC;
    const bool value = blockIdx.z;
    const T* src = (value ? V : K) + piece * 8;
    const size_t ld = value ? a.ldv : a.ldk;
    auto place_of = [&](long long t) {                   // of row t, -1: none
        const int p = t >= 0 && t < a.n_rows ? a.row_slot[t] : -1;
        return p >= 0 && p < a.n_places ? p : -1;
    };
    auto load = [&](const T* p, uint4* c) {
        c[0] = load_stream16(p);
        if constexpr (NV == 2) c[1] = load_stream16(p + 4);
    };
    auto unpack = [&](const uint4* c, float* f) {
        Elem<T>::unpack(c[0], f);
        if constexpr (NV == 2) Elem<T>::unpack(c[1], f + 4);
    };
    auto old_byte = [&](const unsigned char* p, int r0) { return r0 > 0 ? (uint32_t)min(max((int)*p, kKv8ByteLow), kKv8ByteHigh) : (uint32_t)kKv8ByteLow; };

    const long long first = (long long)blockIdx.x * a.chunk;
    unsigned long long shorts, longs;
    int place = -1;
    {
        bool start = false, is_long = false;
        if (lane < a.chunk) {
            place = place_of(first + lane);
            const int before = place_of(first + lane - 1), far = place_of(first + lane + kKv8Short);
            if (place >= 0) {
                const int r = place - a.by_block(place) * a.block;
                start = r == 0 || before != place - 1;
                is_long = start && r < a.block - kKv8Short && far == place + kKv8Short;
            }
        }
        shorts = __ballot(start && !is_long);
        longs = __ballot(is_long);
    }

    const int g0 = blockIdx.y * a.heads, g1 = min(g0 + a.heads, a.Hkv);
    if (g0 % HEADS != 0) shorts = 0;
    const int g_short = min(g0 + lane / PC, a.Hkv - 1);
    const bool mine = g0 + lane / PC < a.Hkv;            // (lanes without a head do as the last one's, but write nothing)
    const Kv8Head at(g_short, a.block, a.Hkv, D);
    for (int number = 0; shorts; ++number) {
        const int i0 = __builtin_ctzll(shorts);
        shorts &= shorts - 1;
        if (number % 4 != wave) continue;
        const int p0 = __builtin_amdgcn_readlane(place, i0), slot = a.by_block(p0), r0 = p0 - slot * a.block;
        const long long t0 = first + i0;
        const int longest = (int)min((long long)min(kKv8Short, a.block - r0), a.n_rows - t0);
        uint4 c[kKv8Short][NV];
#pragma unroll
        for (int i = 0; i < kKv8Short; ++i)
            load(src + (size_t)g_short * D + (size_t)(t0 + min(i, longest - 1)) * ld, c[i]);
        unsigned char* base = a.pool + (size_t)slot * a.slot_bytes + a.layer_offset;
        unsigned char* codes = base + (value ? at.v : at.k);
        unsigned char* exponent = base + at.e + (value ? 1 : 0);
        const uint32_t before = old_byte(exponent, r0);
        const int n = __builtin_ctzll(~__ballot(lane < longest && place_of(t0 + lane) == p0 + lane));      // rows of the run
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kKv8Short; ++i) {
            float f[8];
            unpack(c[i], f);
            const uint32_t now = largest(f, m);
            m = i < n ? now : m;
        }
#pragma unroll
        for (int o = 1; o < PC; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
        const uint32_t byte = max(before, exponent_byte(m));
        const float power = kv8_power(byte);
        if (mine) {
#pragma unroll
            for (int i = 0; i < kKv8Short; ++i)
                if (i < n) {
                    float f[8];
                    unpack(c[i], f);
                    *reinterpret_cast<uint2*>(codes + (size_t)(r0 + i) * D + piece * 8) = kv8_eight(f, power);
                }
            if (piece == 0) *exponent = (unsigned char)byte;
        }
        unsigned long long grown = r0 > 0 ? __ballot(mine && piece == 0 && byte > before) : 0;
        while (grown) {
            const int x = __builtin_ctzll(grown);
            grown &= grown - 1;
            const Kv8Head there(g0 + x / PC, a.block, a.Hkv, D);
            kv8_round_again(base + (value ? there.v : there.k), (size_t)r0 * D, (uint32_t)__builtin_amdgcn_readlane((int)(byte - before), x), lane, 64);
        }
    }

    for (int turn = 0; longs;) {
        const int i0 = __builtin_ctzll(longs);
        longs &= longs - 1;
        const int p0 = __builtin_amdgcn_readlane(place, i0), slot = a.by_block(p0), r0 = p0 - slot * a.block;
        const long long t0 = first + i0;
        const int longest = (int)min((long long)a.block - r0, a.n_rows - t0);
        unsigned char* base = a.pool + (size_t)slot * a.slot_bytes + a.layer_offset;
        uint4 keep[kKv8Keep][NV];
        uint32_t before;
        auto request = [&](int g) {                      // a head's rows (the last one again where the block has no more) and exponent
            const T* rows = src + (size_t)g * D;
#pragma unroll
            for (int i = 0; i < kKv8Keep; ++i) load(rows + (size_t)(t0 + min(i * RPP + row, longest - 1)) * ld, keep[i]);
            before = old_byte(base + Kv8Head(g, a.block, a.Hkv, D).e + (value ? 1 : 0), r0);
        };
        request(g0);
        int n = 0;                                       // rows of the run
        while (n < longest) {
            const bool same = n + lane < longest && place_of(t0 + n + lane) == p0 + n + lane;
            const unsigned long long end = ~__ballot(same);
            n += end ? __builtin_ctzll(end) : 64;
            if (end) break;
        }
        for (int g = g0; g < g1; ++g, ++turn) {
            const T* rows = src + (size_t)g * D;
            const Kv8Head at(g, a.block, a.Hkv, D);
            unsigned char* codes = base + (value ? at.v : at.k);
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < kKv8Keep; ++i) {
                float f[8];
                unpack(keep[i], f);
                const uint32_t now = largest(f, m);
                m = i * RPP + row < n ? now : m;
            }
            for (int i = kKv8Keep * RPP + row; i < n; i += RPP) {
                uint4 c[NV];
                float f[8];
                load(rows + (size_t)(t0 + i) * ld, c);
                unpack(c, f);
                m = largest(f, m);
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
            if (lane == 0) most_of[turn & 1][wave] = m;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < 4; ++w) m = max(m, most_of[turn & 1][w]);
            const uint32_t was = before, byte = max(was, exponent_byte(m));
            const float power = kv8_power(byte);
            auto eight = [&](const uint4* c) {
                float f[8];
                unpack(c, f);
                return kv8_eight(f, power);
            };
            uint2 code[kKv8Keep];
#pragma unroll
            for (int i = 0; i < kKv8Keep; ++i) code[i] = eight(keep[i]);
            if (g + 1 < g1) request(g + 1);              // on its way while this head's codes are written
#pragma unroll
            for (int i = 0; i < kKv8Keep; ++i)
                if (i * RPP + row < n) *reinterpret_cast<uint2*>(codes + (size_t)(r0 + i * RPP + row) * D + piece * 8) = code[i];
            for (int i = kKv8Keep * RPP + row; i < n; i += RPP) {
                uint4 c[NV];
                load(rows + (size_t)(t0 + i) * ld, c);
                *reinterpret_cast<uint2*>(codes + (size_t)(r0 + i) * D + piece * 8) = eight(c);
            }
            if (byte > was && r0 > 0) kv8_round_again(codes, (size_t)r0 * D, byte - was, tid, 256);
            if (tid == 0) base[at.e + (value ? 1 : 0)] = (unsigned char)byte;
        }
    }
}

int launch_kv8_write(const void* k, const void* v, int ldk, int ldv, const int* row_slot, int n_rows, int Hkv, int d, int block, int dtype, void* pool, int n_slots, size_t slot_bytes,
                     size_t layer_offset, hipStream_t st) {
    // Few rows in small chunks, so that there are workgroups for all CUs, many in the largest, which look at the map least: 256 tokens of 8 heads 6.2 us in chunks of 4, 37 of 64 (whose waves
    // take run after run); 26381 rows 78 and 42.  Four heads a workgroup: with 4, 2, 1 those take 41.9, 42.3 and 44.6.
    const int chunk = (int)std::min<long long>(64, std::max<long long>(4, (long long)n_rows * Hkv * 2 / 4096));
    const int heads = 4;
    const Kv8Write a{row_slot, (unsigned char*)pool, slot_bytes, layer_offset, n_rows, n_slots * block, block, Hkv, ldk, ldv, chunk, heads, Divide(block)};
    const dim3 grid((n_rows - 1) / chunk + 1, (Hkv - 1) / heads + 1, 2);
#define SLIM_KV8(T, D) hipLaunchKernelGGL((kv8_write_kernel<T, D>), grid, dim3(256), 0, st, (const T*)k, (const T*)v, a)
    if (dtype == SLIM_BF16) { if (d == 64) SLIM_KV8(bf16_t, 64); else SLIM_KV8(bf16_t, 128); }
    else if (d == 64) SLIM_KV8(float, 64);
    else SLIM_KV8(float, 128);
#undef SLIM_KV8
    return check_launch();
}

// ---- read back
// Codes once, rows once: a lane takes eight channels of kKv8Steps rows, a wave the rows of its head that lie side by side.  Bound by memory: 9856 tokens of 8 heads of 128 (60 MB) 11.4 us,
// 32768 (201 MB) 24.3, what its launch and the lookup of a slot cost beside it: 64 tokens 3.0.  One, two, four rows: 9856 tokens 10.8, 11.4, 12.3 us, 32768 26.6, 24.3, 26.0.
constexpr int kKv8Steps = 2;
struct Kv8Read {
    const unsigned char* pool;
    size_t slot_bytes, layer_offset;
    const int* slots;                                    // null: block b lies in slot b
    int n_slots, n_tokens, block, Hkv, ldk, ldv;
};

template <typename T, int D>
__global__ void __launch_bounds__(256) kv8_read_kernel(T* __restrict__ K, T* __restrict__ V, Kv8Read a) {
    constexpr int PC = D / 8, RPW = 64 / PC;             // lanes a row, rows a step
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, piece = lane % PC;
    const bool value = blockIdx.z;
    const int g = blockIdx.y;
    const int t0 = (blockIdx.x * 4 + wave) * (RPW * kKv8Steps) + lane / PC;
    T* out = (value ? V : K) + (size_t)g * D + piece * 8;
    const size_t ld = value ? a.ldv : a.ldk;
    const Kv8Head at(g, a.block, a.Hkv, D);
    int b = t0 / a.block, r = t0 - b * a.block;
    uint2 code[kKv8Steps];
    uint32_t byte[kKv8Steps];
    bool have[kKv8Steps];
#pragma unroll
    for (int s = 0; s < kKv8Steps; ++s) {
        have[s] = false;
        if (t0 + s * RPW < a.n_tokens) {
            const int slot = a.slots ? a.slots[b] : b;
            if (slot >= 0 && slot < a.n_slots) {
                const unsigned char* src = a.pool + (size_t)slot * a.slot_bytes + a.layer_offset;
                code[s] = *reinterpret_cast<const uint2*>(src + (value ? at.v : at.k) + (size_t)r * D + piece * 8);
                byte[s] = src[at.e + (value ? 1 : 0)];
                have[s] = true;
            }
        }
        r += RPW;
        while (r >= a.block) { r -= a.block; ++b; }
    }
#pragma unroll
    for (int s = 0; s < kKv8Steps; ++s) {
        if (!have[s]) continue;
        const uint4 v = __builtin_bit_cast(uint4, kv8_to_bf16(code[s], kv8_power(byte[s])));
        T* dst = out + (size_t)(t0 + s * RPW) * ld;
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

int launch_kv8_read(const void* pool, int n_slots, size_t slot_bytes, size_t layer_offset, const int* slots, int n_tokens, int Hkv, int d, int block, int dtype, void* k, void* v,
                    int ldk, int ldv, hipStream_t st) {
    const Kv8Read a{(const unsigned char*)pool, slot_bytes, layer_offset, slots, n_slots, n_tokens, block, Hkv, ldk, ldv};
    const int per_wg = 4 * kKv8Steps * 512 / d;
    const dim3 grid((n_tokens - 1) / per_wg + 1, Hkv, 2);
#define SLIM_KV8(T, D) hipLaunchKernelGGL((kv8_read_kernel<T, D>), grid, dim3(256), 0, st, (T*)k, (T*)v, a)
    if (dtype == SLIM_BF16) { if (d == 64) SLIM_KV8(bf16_t, 64); else SLIM_KV8(bf16_t, 128); }
    else if (d == 64) SLIM_KV8(float, 64);
    else SLIM_KV8(float, 128);
#undef SLIM_KV8
    return check_launch();
}

// ---- attention
// A request's rows are its (query, query head of the kv head) pairs, query by query, head by head; a tile is 16 of them, or 32 in batches of longer drafts.  A piece is up to 16 keys of one
// block.  The pieces of all tiles of all requests, one behind the other, are cut into equal shares, one workgroup a share, so that requests of any lengths keep all workgroups busy to the
// end.  A workgroup goes through its share tile by tile; its waves take two pieces in turn, from wherever they lie.  A tile that lies in one share is written at once, one that several
// share is left as partial results, which a second kernel merges.  The lengths are known to the GPU alone, so that each wave forms the sums over the requests for itself, 64 of them at a time.
// The Keys' codes become bfloat16 in the lanes that read them, in the order of the matrix instruction; the Values' go through LDS, whose transposing read gives the other operand.  The
// next pieces' codes are requested as soon as the registers of the present ones are free.
// Bound by the codes' way from memory: 256 requests of one token, 32 heads over 8 of 128, of 751 MB altogether, 150 us and 5 to merge, 4.9 TB/s (a kernel that only reads them 145); one of
// 131072 tokens, 268 MB, 54 and 5 (52); 48 requests with up to 4 drafts, 279 MB, 73 and 5 (65).
constexpr int kPiece = 16;
constexpr int kBatchWaves = 4;
// Workgroups: as many as run together, three a CU, and where the registers leave two (float32 heads of 128, tiles of 32 rows) 512.  With 768 and 512, 256 requests of 64 to 8192 tokens: bfloat16
// heads of 128 150 and 157 us, of 64 105 and 114, float32 heads of 64 115 and 129, of 128 239 and 204; 64 drafts of 8 queries, heads of 64, 52 and 45.  (Where the requests are as many as the
// shares of a head and alike, nothing is shared: 64 of 4000 tokens, 8 heads of 64, 61 and 55.)
constexpr int kBatchGrid = 768;
template <typename T, int D, int NR> constexpr int batch_grid() { return NR == 1 && (sizeof(T) == 2 || D == 64) ? kBatchGrid : 512; }
constexpr int kBatchLeast = 2 * 2 * kBatchWaves;         // pieces of a share: two turns of its waves (one request of 500 to 4000 tokens 13 us; with one turn 13, with four 14 to 16, with eight
                                                         // 14 to 20); of tiles of 32 rows, whose turns are longer, one (16 queries of a request of 512 or 2048 tokens 17 and 21 us, with two 23 and 25)
constexpr int kBatchTile = 8;                            // what beginning and ending a tile counts for, in pieces (256 requests 156 us, with 2 165, with 24 156)
constexpr int kFewRows = 64, kManyRows = 256, kManyGrid = 256;      // rows of a request up to which tiles have 16 or 32 rows; rows of the tiles for more; their workgroups
constexpr int kFewPartRows = 512 * 2 * 2 * kTileRows, kPartRows = kFewPartRows + kManyGrid * 2 * kManyRows;      // rows of partial results

struct BatchAttnArgs {
    const int *row_start, *lens, *table;
    const unsigned char* pool;
    size_t slot_bytes, layer_offset;
    float* part;                                         // rows of D + 4: values, maximum, sum; [shares][2][rows of a tile]: of the tile that a share begins within, and of the one that it leaves unfinished
    int2* where;                                         // of row (t, h): its row of `part` in the share that begins its tile, and 2 * the number of shares + 1 for tiles of many rows
    float scale_log2e;
    int R, max_blocks, n_slots, n_rows, block, per_block, Hq, Hkv, ldq, ldo;      // per_block: pieces
    int few, tile_rows;                                  // requests of more rows (of a kv head) are left to the kernel for many; rows of the tiles of the others
    Divide by_block, by_piece, by_group, by_shares;      // by block, per_block, Hq / Hkv, the shares of a kv head (few rows)
};

struct BatchRequest {
    int lo, n, len;                                      // first row of the step, rows of it, tokens
    __device__ __forceinline__ int rows(const BatchAttnArgs& a) const { return n * (a.Hq / a.Hkv); }      // of a kv head
    template <int TR> __device__ __forceinline__ int tiles(const BatchAttnArgs& a) const { return (rows(a) + TR - 1) / TR; }
    __device__ __forceinline__ int pieces(const BatchAttnArgs& a) const {
        const int whole = a.by_block(len);
        return whole * a.per_block + (len - whole * a.block + kPiece - 1) / kPiece;
    }
    template <int TR> __device__ __forceinline__ long long cost(const BatchAttnArgs& a) const { return (long long)tiles<TR>(a) * (pieces(a) + kBatchTile); }
    __device__ __forceinline__ bool many(const BatchAttnArgs& a) const { return n > 0 && rows(a) > a.few; }
};
__device__ __forceinline__ BatchRequest batch_request(const BatchAttnArgs& a, int r) {
    BatchRequest x = {0, 0, 0};
    if (r < a.R) {
        x.lo = min(max(a.row_start[r], 0), a.n_rows);
        x.n = min(max(a.row_start[r + 1], x.lo), a.n_rows) - x.lo;
        x.len = min(max(a.lens[r], 0), a.max_blocks * a.block);
    }
    return x;
}
// Of lane i, which is the same in the whole wave.
__device__ __forceinline__ int wave_value(int v, int i) { return __builtin_amdgcn_readlane(v, i); }
__device__ __forceinline__ long long wave_value(long long v, int i) {
    return (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32) | (unsigned)__builtin_amdgcn_readlane((int)v, i));
}
__device__ __forceinline__ long long wave_prefix(long long v, int lane) {      // sum of the lanes up to this one
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long x = __shfl_up(v, o, 64);
        if (lane >= o) v += x;
    }
    return v;
}
// A loaded value whose first use is here (left alone, the compiler moves what is made of it behind the load, and with it the wait).
__device__ __forceinline__ uint32_t first_used_here(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
}

template <typename T, int D, int NW, int NR>
__global__ void __launch_bounds__(64 * NW, sizeof(T) == 2 && NR == 1 ? 3 : 2) batch_attn_kv8_kernel(const T* __restrict__ q, T* __restrict__ out, BatchAttnArgs a) {
    typedef RowTile<T, D> Tile;
    constexpr int NP = Tile::NP, NT = Tile::NT, KS = Tile::KS, PC = D / 64, TR = NR * kTileRows;      // PC: 16-byte pieces of a lane's channels
    extern __shared__ __align__(256) unsigned char lds[];
    const int G = a.Hq / a.Hkv;
    // The kv head goes fastest: with eight of them each XCD has its own.
    const int g = blockIdx.x % a.Hkv, share_of = blockIdx.x / a.Hkv, shares = gridDim.x / a.Hkv;
    int r0 = 0;                                          // x: of request r0 + the lane
    const int lane_in = threadIdx.x & 63;
    auto request = [&](int r) {
        BatchRequest x = batch_request(a, r);
        if (x.many(a)) x.n = 0;
        return x;
    };
    BatchRequest x = request(lane_in);
    long long mine = x.template cost<TR>(a), end = a.R == 1 ? mine : wave_prefix(mine, lane_in);
    long long total = wave_value(end, a.R == 1 ? 0 : 63);      // (in scalar registers, with all that follows from it)
    for (int r = 64; r < a.R; r += 64) total += wave_value(wave_prefix(request(r + lane_in).template cost<TR>(a), lane_in), 63);
    const long long share = max((long long)kBatchLeast / NR, total < 1ll << 30 ? (long long)a.by_shares((int)total + shares - 1) : (total + shares - 1) / shares), begin = share * share_of;
    long long left_over = min(total - begin, share);     // of the share
    if (left_over <= 0) return;
    long long at = begin;                                // of the share's beginning, counted from request r0's, then from its own request's
    int i_req;
    while (true) {
        const unsigned long long behind = __ballot(end > at);
        if (behind) {
            i_req = __builtin_ctzll(behind);
            at -= wave_value(end - mine, i_req);
            break;
        }
        at -= wave_value(end, 63);
        r0 += 64;
        if (r0 >= a.R) return;
        x = request(r0 + lane_in);
        mine = x.template cost<TR>(a);
        end = wave_prefix(mine, lane_in);
    }
    int tile = 0, from = (int)at;
    const int apart = wave_value(x.pieces(a), i_req) + kBatchTile;
    if (at >= apart) {
        tile = (int)(at / apart);
        from = (int)(at - (long long)tile * apart);
    }

    const Kv8Head head(g, a.block, a.Hkv, D);
    while (true) {
        const BatchRequest me{wave_value(x.lo, i_req), wave_value(x.n, i_req), wave_value(x.len, i_req)};
        const int pieces = me.pieces(a);
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                        // (what follows from it would be kept in registers from tile to tile)
        const int lane = tid & 63, l16 = lane & 15, qr = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const unsigned tile_lds = (unsigned)(uintptr_t)lds + wave * Tile::kLdsBytes;
        const int r = r0 + i_req, take = (int)min((long long)(pieces + kBatchTile - from), left_over);
        const int row0 = tile * TR, rows = min(TR, me.rows(a) - row0);
        const int p0 = me.len - me.n + row0 / G, p1 = me.len - me.n + (row0 + rows - 1) / G;      // positions of the first and the last row
        const int limit = p1 + 1;                            // (zero and below if there are more rows than tokens: then no piece is found)
        const int* table = a.table + (size_t)r * a.max_blocks;

        // The wave's pieces, in pairs: u0, u0 + 1, u0 + 2 NW, ..  64 of them are looked up at once, one a lane, and the table entries of the next 64 are on their way.  A piece of a block that no
        // slot has, or behind the last row, has no keys and is passed over.
        const int last = limit <= 0 ? 0 : a.by_block(limit - 1) * a.per_block + (limit - 1 - a.by_block(limit - 1) * a.block) / kPiece + 1;
        const int u_end = min(last, from + take);
        constexpr int kBatch = 64 * NW;
        int u = from + 2 * wave + (lane >> 1) * 2 * NW + (lane & 1);      // the lane's
        int batch = __builtin_amdgcn_readfirstlane(u) - kBatch;
        int u_slot = 0, u_pos = 0, u_rows = 0, next_slot = u < u_end ? table[a.by_piece(u)] : -1;
        unsigned long long left = 0;
        int have[2], c0[2], pos[2];
        const unsigned char* base[2];
        auto find = [&]() {                                  // the next two pieces; false: none is left
            while (!left) {
                batch += kBatch;
                if (batch >= u_end) return false;
                const int b = a.by_piece(u), row = (u - b * a.per_block) * kPiece;
                u_slot = next_slot;
                u_pos = b * a.block + row;
                u_rows = u_slot >= 0 && u_slot < a.n_slots ? min(kPiece, min(a.block - row, limit - u_pos)) : 0;
                left = __ballot(u_rows > 0);
                u += kBatch;
                next_slot = u < u_end ? table[a.by_piece(u)] : -1;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h == 1 && !left) {                       // a single one: the other half repeats it, unseen
                    have[1] = 0;
                    c0[1] = c0[0];
                    pos[1] = pos[0];
                    base[1] = base[0];
                    break;
                }
                const int i = __builtin_ctzll(left);
                left &= left - 1;
                have[h] = __builtin_amdgcn_readlane(u_rows, i);
                pos[h] = __builtin_amdgcn_readlane(u_pos, i);
                c0[h] = pos[h] - a.by_block(pos[h]) * a.block;
                base[h] = a.pool + (size_t)__builtin_amdgcn_readlane(u_slot, i) * a.slot_bytes + a.layer_offset;
            }
            return true;
        };

        uint4 kx[2][PC], vx[2][PC];
        uint32_t ke[2], ve[2];                               // e + 127
        // Addresses: a wave-uniform base and a 32-bit offset of the lane.  Rows behind the last key repeat it: not seen.  A lane's channels are 16 in a row of each 64, so that an instruction
        // takes 64 bytes in a row of each key.
        auto row_offset = [&](int h) { return (unsigned)(min(l16, max(have[h], 1) - 1) * D + qr * 16); };
        auto channel = [&](int j) { return j / 2 * 64 + qr * 16 + j % 2 * 8; };
        auto load_k = [&]() {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned char* at = base[h] + head.k + (size_t)c0[h] * D;
                const unsigned off = row_offset(h);
#pragma unroll
                for (int c = 0; c < PC; ++c) kx[h][c] = *reinterpret_cast<const uint4*>(at + (off + c * 64));
                ke[h] = base[h][head.e + (lane & 0)];
            }
        };
        auto load_v = [&]() {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned char* at = base[h] + head.v + (size_t)c0[h] * D;
                const unsigned off = row_offset(h);
#pragma unroll
                for (int c = 0; c < PC; ++c) vx[h][c] = *reinterpret_cast<const uint4*>(at + (off + c * 64));
                ve[h] = base[h][head.e + 1 + (lane & 0)];
            }
        };
        auto half_of = [](const uint4& c, int j) { return j % 2 ? make_uint2(c.z, c.w) : make_uint2(c.x, c.y); };
        bool more = find();
        if (more) { load_k(); load_v(); }

        // the lane's rows, one in each 16
        int p[NR];
        Tile t[NR];
#pragma unroll
        for (int y = 0; y < NR; ++y) {
            const int lrow = row0 + min(y * kTileRows + l16, rows - 1), token = a.by_group(lrow);
            p[y] = me.len - me.n + token;
            t[y].begin(q + (size_t)(me.lo + token) * a.ldq + (size_t)(g * G + lrow - token * G) * D, channel);
            // waited for here: waited for in the loop, the Query fragments take the wait for the codes requested meanwhile with them in every turn
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int j = 0; j < KS; ++j) asm volatile("" : "+v"(t[y].q[b][j]));
        }
        // Where the lane writes and reads the wave's V tile: one address each, whose bits 4 .. 7 are turned for the pieces and channels.  (Hidden from the compiler in every turn: it would keep
        // them all in registers, and the Query fragments out of them.)
        const int vr = 4 * qr + (l16 >> 2);
        unsigned v_to = tile_lds + Tile::v_piece(l16, qr * 2), v_from = tile_lds + Tile::v_piece(vr, (l16 & 3) >> 1) + (l16 & 1) * 8;
        while (more) {
            asm volatile("" : "+v"(v_to), "+v"(v_from));
            const bool whole = have[0] == kPiece && have[1] == kPiece && max(pos[0], pos[1]) + kPiece - 1 <= p0;      // every row sees every key
            int seen[NR][2];                                 // keys that the lane's rows see
#pragma unroll
            for (int y = 0; y < NR; ++y)
#pragma unroll
                for (int h = 0; h < 2; ++h) seen[y][h] = min(have[h], p[y] + 1 - pos[h]);
            more = find();                                   // none left: the last pieces are requested once more, and not used
            f32x4 s[NR][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                typename Tile::Scores sum[NR];
                const float kp = kv8_power(first_used_here(ke[h]));
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                    const bf16x8 k = kv8_to_bf16(half_of(kx[h][j / 2], j), kp);
#pragma unroll
                    for (int y = 0; y < NR; ++y) t[y].template add_scores<1>(&k, j, sum[y]);
                }
#pragma unroll
                for (int y = 0; y < NR; ++y) s[y][h] = sum[y].sum();
            }
            __builtin_amdgcn_sched_barrier(0);
            load_k();                                        // the next pieces' Keys fly under these Values
            __builtin_amdgcn_sched_barrier(0);
            if (!whole) {
#pragma unroll
                for (int y = 0; y < NR; ++y)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = s[y][h][e];
                            s[y][h][e] = qr * 4 + e < seen[y][h] ? x : -INFINITY;
                        }
            }
            bf16x8 pw[NR][NP];
#pragma unroll
            for (int y = 0; y < NR; ++y) {
                float w[8];
                t[y].weigh(s[y], a.scale_log2e, w);
                bf16_terms<NP>(w, pw[y]);
            }
            float vp[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) vp[h] = kv8_power(first_used_here(ve[h]));
            if (!whole) {
                // Values that some row does not see and that are not numbers: their weight is 0, which a product would turn into an undefined sum.  They become zeros here, and what makes a row
                // that sees one of them undefined is its sum.
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    bool odd = false;
#pragma unroll
                    for (int c = 0; c < PC; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t& x = i == 0 ? vx[h][c].x : i == 1 ? vx[h][c].y : i == 2 ? vx[h][c].z : vx[h][c].w;
                            const uint32_t bytes = (((x & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u) * 0xffu;
                            odd |= bytes != 0;
                            x &= ~bytes;
                        }
                    const unsigned long long lanes = __ballot(odd);
                    if (lanes) {
                        const unsigned keys = (unsigned)(lanes | lanes >> 16 | lanes >> 32 | lanes >> 48) & 0xffffu;
#pragma unroll
                        for (int y = 0; y < NR; ++y)
                            if (keys & ((1u << max(seen[y][h], 0)) - 1u)) t[y].l = NAN;
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < KS; ++j) *(LdsB128)((v_to ^ ((j / 2 * 8 + j % 2) << 4)) + h * (16 * D * 2)) = kv8_to_bf16(half_of(vx[h][j / 2], j), vp[h]);
            __builtin_amdgcn_sched_barrier(0);
            load_v();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int dt = 0; dt < Tile::DT; ++dt) {
                const bf16x8 v = Tile::read_channels(v_from ^ (dt << 5));
#pragma unroll
                for (int y = 0; y < NR; ++y) t[y].template add_read<1>(pw[y], 0, dt, v);
            }
        }

        const bool whole_tile = from == 0 && take >= pieces;
        if (from < pieces || whole_tile) {                // (else nothing but the tile's end is left in this share)
            if (from == 0 && tid < rows) {
                const int i = row0 + tid, n = i / G;
                const long long to = begin + share - left_over + pieces - 1;      // (what the share has taken so far is share - left_over, but for the last one, which ends with its tile)
                const int n_shares = whole_tile ? 1 : (int)(to / share) - share_of + 1;
                a.where[(size_t)(me.lo + n) * a.Hq + g * G + i - n * G] = make_int2((blockIdx.x * 2 + 1) * TR + tid, 2 * n_shares);
            }
            float* part = a.part + (size_t)(blockIdx.x * 2 + (from == 0)) * TR * (D + 4);
#pragma unroll
            for (int y = 0; y < NR; ++y) {
                const int in_half = rows - y * kTileRows;
                if (y > 0 && in_half <= 0) break;
                merge_waves<T, D, NW>(t[y], lds, min(kTileRows, in_half), [&](int i, int dd, float acc, float l, float M) {
                    i += y * kTileRows;
                    if (whole_tile) {
                        const int x = row0 + i, n = x / G;
                        Elem<T>::st(out + (size_t)(me.lo + n) * a.ldo + (size_t)(g * G + x - n * G) * D + dd, l == 0.f ? 0.f : acc / l);
                    } else {
                        float* dst = part + i * (D + 4);
                        dst[dd] = acc;
                        if (dd == 0) { dst[D] = M; dst[D + 1] = l; }
                    }
                }, tid);
                __syncthreads();                             // the waves' tiles are read before they are written again
            }
        }
        left_over -= take;
        if (left_over <= 0) return;
        from = 0;
        if (++tile == me.template tiles<TR>(a)) {
            tile = 0;
            unsigned long long more_rows = __ballot(x.n > 0) & ~((2ull << i_req) - 1);
            while (!more_rows) {
                r0 += 64;
                if (r0 >= a.R) return;
                x = request(r0 + lane_in);
                more_rows = __ballot(x.n > 0);
            }
            i_req = __builtin_ctzll(more_rows);
        }
    }
}

// ---- requests of many rows (bfloat16)
// Tiles of 256 rows, 32 a wave; the eight waves turn 64 keys at a time into bfloat16 Keys and float16 Values in LDS, once for all of them, and each forms, in 32x32x16 matrix instructions,
//   S^T[key, row] = K . Q^T       32 keys; the lane (l32, h) = (lane % 32, lane / 32) is left scores of row l32: keys 8 i + 4 h + 0 .. 3, i < 4
//   O^T[d, row]   = V^T . P^T     whose operand P^T is what the lane holds: V comes through the transposing read in the same order of keys
// A phase stands for 32 keys: their weights, beside the scores of the 32 behind and the values of the 32 before, a matrix instruction and a lane's arithmetic in turn.  It reads the Values in its
// first half, the Keys of the next phase in its second.  Four buffers of 64 keys: Values of the keys before, the present and the next keys, and the ones being filled; a barrier each 64 keys.
// A weight is 2^(score - reference), the sum of the softmax that of the weights, unrounded; what a key's block holds beside it, or behind what the row sees, touches neither.  Two loops:
//   Where the exponents e of the Values' blocks that a workgroup's part of a tile meets lie within kManySpan of each other (nearly always): a weight is rounded to one float16, a Value is
//   code * 2^(e - largest e + kManyShift) in float16, exact (with kManySpan 12 and kManyShift 7 from 2^-14, the smallest normal one, to 57344), and the results are multiplied by the power
//   that is left.  The reference of a row is a whole number, 10 below its largest score when it was set, and is set anew, by a power of two, only when a score is more than 15 above it: nothing
//   is rescaled in nearly all phases.  Weights from 2^-14 on (2^-23 of the row's largest or less) are off by 2^-11 of themselves, smaller ones by 2^-25 (2^-34 of the largest): so a result is
//   off by 2^-11 of sum p |v| and 2^-34 of sum |v|.
//   Where they are further apart, that last sum may be anything beside the first, and a weight has to keep its places however small it is: two bfloat16 terms (2^-17 of itself), Values as
//   bfloat16 with their powers, the reference the running maximum.  So too, in a second pass over the same keys, where at the end of the first loop the last sum can be more than 2^-10 of a row's
//   largest result (one key takes nearly everything and has Values of next to nothing).  One buffer, filled and read in turn: 358 us for a call of 1511 queries behind 9856 tokens where the other loop takes 240 to 250.
// Bound by issue: 1511 queries behind 9856 tokens, 28 heads over 4 of 128, 230 GFLOP in 250 us
// by themselves and 280 to 290 one call behind the other, 0.92 and 0.8 PFLOP/s, where a library product of 8192^3 reaches 1.37 and matrix instructions alone 1.75; the matrix units are
// busy half of the time, and beside 16 of their instructions a wave has some 105 others of the vector ALU and 28 of LDS, which its SIMD's two waves do not hide altogether.  Weights of one bfloat16 took 243 us of an earlier form's 247, with an error of 2.4 10^-3 from 64 bits where rounding the output leaves 1.7.  That form
// without the exponentials took 57 us less, without LDS 39: no one of them bounds it alone.  16 rows a wave 484 us; 64 rows a wave, with all 512 registers, as 32.
constexpr int kManyKeys = 64;
template <int D> struct ManyTile {
    // Rows of D 16-bit numbers and 16 bytes (Keys: 16 keys' same piece of 16 bytes) or 64 (Values: four keys' same 64 bytes) cover all banks once, and every address of a lane is one base and a constant.
    static constexpr int kRowK = D * 2 + 16, kRowV = D * 2 + 64, kSide = kManyKeys * kRowK, kBuffer = kSide + kManyKeys * kRowV;      // a key; the Keys; both
    static constexpr int kFlags = 4 * kBuffer, kSpans = kFlags + 32, kLost = kSpans + 32, kLists = kLost + 32, kLdsBytes = kLists + 8 * 64 * 16;      // four; a bit for each of their keys with a
                                                               // Value that is not a number; the exponents that the waves have met, and whether they have a row that float16 is not enough for; a wave's pieces
    static constexpr int KS = D / 16, DT = D / 32;
};
constexpr float kManyAbove = 10.f, kManyRoom = 15.f;     // where the largest weight begins, and how far it may grow: 2^10, 2^15
constexpr int kManySpan = 12, kManyShift = 7, kManyFar = 64;      // of the Values' exponents, see above; their magnitude (partial results are not divided by their sums, and stay far from float32's ends)

template <int D>
__global__ void __launch_bounds__(512, 2) batch_attn_many_kernel(const bf16_t* __restrict__ q, bf16_t* __restrict__ out, BatchAttnArgs a) {
    typedef ManyTile<D> Tile;
    constexpr int KS = Tile::KS, DT = Tile::DT, PR = D / 16;      // PR: 16-byte pieces of a key's codes
    extern __shared__ __align__(16) unsigned char lds[];
    const int G = a.Hq / a.Hkv, g = blockIdx.x % a.Hkv, share_of = blockIdx.x / a.Hkv, shares = gridDim.x / a.Hkv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, h = lane >> 5;
    const unsigned lds0 = (unsigned)(uintptr_t)lds;

    // What a tile costs: the tokens that its last row sees, and some for beginning and ending it, times G so that it is a whole number: each of a request's tiles kManyRows more.  (64, 256 or
    // 1024 tokens for it make no difference to long requests.)
    constexpr int kManyTile = 256;
    auto tiles_of = [&](const BatchRequest& x) { return (x.rows(a) + kManyRows - 1) / kManyRows; };
    auto first_cost = [&](const BatchRequest& x) { return (long long)G * (max(x.len - x.n, 0) + kManyTile) + kManyRows; };
    auto cost_to = [&](const BatchRequest& x, long long tiles) { return tiles * first_cost(x) + tiles * (tiles - 1) / 2 * kManyRows; };
    auto request = [&](int r) {
        BatchRequest x = batch_request(a, r);
        if (!x.many(a)) x.n = 0;
        return x;
    };
    int r0 = 0;
    BatchRequest x = request(lane);
    auto cost = [&](const BatchRequest& x) { return cost_to(x, tiles_of(x)); };
    long long total = cost(x);
    for (int r = 64; r < a.R; r += 64) total += cost(request(r + lane));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
    total = wave_value(total, 0);
    // (A new prompt of 512 tokens 37 us in shares of 256 tokens' cost at least, 55 without.)
    const long long share = max((long long)G * 256, (total + shares - 1) / shares), begin = share * share_of;
    long long left_over = min(total - begin, share);
    if (left_over <= 0) return;
    long long at = begin;
    int i_req;
    while (true) {
        const long long mine = cost(x), end = wave_prefix(mine, lane);
        const unsigned long long behind = __ballot(end > at);
        if (behind) {
            i_req = __builtin_ctzll(behind);
            at -= wave_value(end - mine, i_req);
            break;
        }
        at -= wave_value(end, 63);
        r0 += 64;
        if (r0 >= a.R) return;
        x = request(r0 + lane);
    }
    BatchRequest me{wave_value(x.lo, i_req), wave_value(x.n, i_req), wave_value(x.len, i_req)};
    int tile = 0;                                        // the one that position `at` lies in: the last one whose beginning is not behind it
    for (int n = tiles_of(me); n > 1;) {
        const int half = n >> 1;
        if (cost_to(me, tile + half) <= at) tile += half;
        n -= half;
    }
    long long from_cost = at - cost_to(me, tile);
    const Kv8Head head(g, a.block, a.Hkv, D);

    while (true) {
        const long long tile_cost = first_cost(me) + (long long)tile * kManyRows, take = min(tile_cost - from_cost, left_over);
        const int row0 = tile * kManyRows, rows = min(kManyRows, me.rows(a) - row0), before = me.len - me.n;
        const int p0 = before + a.by_group(row0), limit = before + a.by_group(row0 + rows - 1) + 1;
        const int* table = a.table + (size_t)(r0 + i_req) * a.max_blocks;
        const int last = limit <= 0 ? 0 : a.by_block(limit - 1) * a.per_block + (limit - 1 - a.by_block(limit - 1) * a.block) / kPiece + 1;
        auto piece_at = [&](long long c) { return c >= tile_cost ? last : (int)((double)last * ((double)c / (double)tile_cost)); };
        const int u_begin = piece_at(from_cost), u_end = piece_at(from_cost + take);

        // The pieces, looked up 64 at once by every wave for itself, one a lane; those with keys are listed in LDS: where the Keys begin, exponents | rows << 16 | 1 << 24 if there are 16 which all
        // rows of the tile see, position.  Four make 64 keys; the list is filled up with pieces without rows.  Slots are requested two lookups ahead, exponents one.
        int u, batch;
        auto slot_at = [&](int u) { return u < u_end ? table[a.by_piece(u)] : -1; };
        auto exponents_at = [&](int slot) {
            return slot >= 0 && slot < a.n_slots ? *reinterpret_cast<const uint16_t*>(a.pool + (size_t)slot * a.slot_bytes + a.layer_offset + head.e) : (uint16_t)0;
        };
        int slot_1, slot_2, at_list, n_list;             // (lists in fours)
        uint32_t e_1;
        auto begin_pieces = [&]() {
            u = u_begin + lane;
            batch = u_begin - 64;
            slot_1 = slot_at(u);
            slot_2 = slot_at(u + 64);
            e_1 = exponents_at(slot_1);
            at_list = n_list = 0;
        };
        begin_pieces();
        // The Values' exponents of all blocks in the tile's part, a block a lane, all waves together: the largest, and how far the smallest lies below it.
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        int e_top, e_low;                                // + 127
        {
            u16x2 span = {0, 0};                         // largest byte, 255 - smallest
            const int b_end = u_begin < u_end ? a.by_piece(u_end - 1) + 1 : 0;
            for (int b = u_begin < u_end ? a.by_piece(u_begin) + (int)threadIdx.x : 0; b < b_end; b += 512) {
                const int slot = table[b];
                if (slot >= 0 && slot < a.n_slots) {
                    const int byte = min(max((int)a.pool[(size_t)slot * a.slot_bytes + a.layer_offset + head.e + 1], kKv8ByteLow), kKv8ByteHigh);
                    span = __builtin_elementwise_max(span, u16x2{(unsigned short)byte, (unsigned short)(255 - byte)});
                }
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) span = __builtin_elementwise_max(span, __builtin_bit_cast(u16x2, __shfl_xor(__builtin_bit_cast(int, span), o, 64)));
            uint32_t* spans = reinterpret_cast<uint32_t*>(lds + Tile::kSpans);
            if (lane == 0) spans[wave] = __builtin_bit_cast(uint32_t, span);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) span = __builtin_elementwise_max(span, __builtin_bit_cast(u16x2, spans[i]));
            const int both = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, span));
            e_top = both == 0 ? 127 : both & 0xffff;     // (no block: nothing is read)
            e_low = both == 0 ? 127 : 255 - (both >> 16 & 0xffff);
        }
        const bool apart = e_top - e_low > kManySpan || e_top > 127 + kManyFar || e_low < 127 - kManyFar;
        int e_shift = apart ? 0 : 127 - e_top + kManyShift;                                            // added to a Value's exponent when it becomes a number
        float left_power = kv8_power((uint32_t)(127 - e_shift));                                       // and what a result is multiplied by for it
        uint4* list = reinterpret_cast<uint4*>(lds + Tile::kLists) + wave * 64;
        auto advance = [&]() {                           // to the next four; false: there are none, and the last ones stay
            if (at_list + 1 < n_list) {
                ++at_list;
                return true;
            }
            while (true) {
                batch += 64;
                if (batch >= u_end) return false;
                const int b = a.by_piece(u), row = (u - b * a.per_block) * kPiece, pos = b * a.block + row;
                const int rows = slot_1 >= 0 && slot_1 < a.n_slots ? min(kPiece, min(a.block - row, limit - pos)) : 0;
                const size_t from = (size_t)a.pool + (size_t)max(slot_1, 0) * a.slot_bytes + a.layer_offset + head.k + (size_t)row * D;
                const uint4 entry = make_uint4((unsigned)from, (unsigned)(from >> 32), e_1 | (unsigned)max(rows, 0) << 16 | (rows == kPiece && pos + kPiece - 1 <= p0 ? 1u << 24 : 0u), (unsigned)pos);
                u += 64;
                e_1 = exponents_at(slot_2);
                slot_1 = slot_2;
                slot_2 = slot_at(u + 64);
                const unsigned long long have = __ballot(rows > 0);
                if (!have) continue;
                const int count = __builtin_popcountll(have), number = __builtin_amdgcn_mbcnt_hi((unsigned)(have >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)have, 0));
                if (rows > 0) list[number] = entry;
                n_list = (count + 3) / 4;
                at_list = 0;
                if (rows > 0 && number == 0)
                    for (int i = count; i < n_list * 4; ++i) list[i] = make_uint4(entry.x, entry.y, entry.z & 0xffffu, entry.w);
                return true;
            }
        };
        // A thread's codes of 64 keys: 16 channels of key threadIdx.x / PR (of heads of 64 the first half of the threads).
        const int my_key = threadIdx.x / PR, my_piece = threadIdx.x % PR;
        const bool mine = D == 128 || my_key < kManyKeys;
        const size_t values_apart = head.v - head.k;
        uint4 kx, vx, entry;
        float kp, vp;
        uint2 info_new;                                  // of lanes 0 .. 3: exponents, rows, position
        auto read_list = [&]() {
            entry = list[at_list * 4 + (D == 128 ? wave >> 1 : wave & 3)];
            const uint4 e = list[at_list * 4 + (lane & 3)];
            info_new = make_uint2(e.z, e.w);
        };
        auto load = [&]() {
            const unsigned char* from = (const unsigned char*)((size_t)entry.y << 32 | entry.x);
            const unsigned off = min(my_key & 15, max((int)(entry.z >> 16 & 31u), 1) - 1) * D + my_piece * 16;
            kx = *reinterpret_cast<const uint4*>(from + off);
            vx = *reinterpret_cast<const uint4*>(from + values_apart + off);
            kp = kv8_power(entry.z & 0xffu);
            vp = kv8_power((uint32_t)(min(max((int)(entry.z >> 8 & 0xffu), kKv8ByteLow), kKv8ByteHigh) + e_shift));
        };
        auto all_full = [](const uint2& info) { return (__ballot(info.x >> 24 & 1u) & 15u) == 15u; };
        // Values of the next keys that are not numbers become zeros, a bit each, where some row does not see all of them (as for few rows).
        auto clear_odd = [&](int buffer) {
            bool odd = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t& x = i == 0 ? vx.x : i == 1 ? vx.y : i == 2 ? vx.z : vx.w;
                const uint32_t bytes = (((x & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u) * 0xffu;
                odd |= bytes != 0;
                x &= ~bytes;
            }
            const unsigned long long lanes = __ballot(odd);
            unsigned bits = 0;                           // of the wave's 64 / PR keys
#pragma unroll
            for (int i = 0; i < 64 / PR; ++i) bits |= (lanes >> (i * PR) & ((1ull << PR) - 1)) ? 1u << i : 0u;
            unsigned char* flags = lds + Tile::kFlags + buffer * 8;
            if (lane == 0 && mine) {
                if constexpr (D == 128) flags[wave] = (unsigned char)bits;
                else *reinterpret_cast<uint16_t*>(flags + wave * 2) = (uint16_t)bits;
            }
        };
        const unsigned fill_k = lds0 + my_key * Tile::kRowK + my_piece * 32, fill_v = lds0 + Tile::kSide + my_key * Tile::kRowV + my_piece * 32;
        // A part of the keys' way into a buffer: eight channels of Keys (part 0, 1) or Values (2, 3; as float16, or as bfloat16 too).
        auto fill_part = [&](int buffer, int part, auto bf16_values) {
            const uint4 c = part < 2 ? kx : vx;
            const uint2 half = part % 2 ? make_uint2(c.z, c.w) : make_uint2(c.x, c.y);
            const bf16x8 x = part < 2 ? kv8_to_bf16(half, kp) : bf16_values.value ? kv8_to_bf16(half, vp) : __builtin_bit_cast(bf16x8, kv8_to_f16(half, vp));
            if (mine) *(LdsB128)((part < 2 ? fill_k : fill_v) + buffer * Tile::kBuffer + part % 2 * 16) = x;
        };

        auto first_keys = [&]() {
            if (!advance()) return false;
            read_list();
            load();
            return true;
        };
        const bool any = first_keys();
        // Query fragments: the lane's row, channels 16 c + 8 h ..
        const int lrow = row0 + min(wave * 32 + l32, rows - 1), token = a.by_group(lrow), my_pos = before + token;
        const bf16_t* q_row = q + (size_t)(me.lo + token) * a.ldq + (size_t)(g * G + lrow - token * G) * D + h * 8;
        bf16x8 qf[KS];
#pragma unroll
        for (int c = 0; c < KS; ++c) qf[c] = *reinterpret_cast<const bf16x8*>(q_row + c * 16);
        f32x16 o[DT];
        // of row l32: reference in the base-2 domain, weights' exponent that it moves above (-inf: not set yet; in the loop of two terms the largest score itself), the lane's share of the sum
        float mc, lim, l;
        auto begin_rows = [&]() {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
            mc = l = 0.f;
            lim = -INFINITY;
        };
        begin_rows();
        // Addresses of the lane in a buffer: K fragments (key l32, channels 16 c + 8 h: pieces 2 c + h), V fragments (keys 16 m + 4 h + .., channels 32 d + ..).
        const unsigned k_from = lds0 + l32 * Tile::kRowK + h * 16;
        const unsigned v_from = lds0 + Tile::kSide + (4 * h + (lane >> 2 & 3)) * Tile::kRowV + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
        bf16x8 kf[KS];
        f16x8 vf[DT][2], pf[2][2];
        f32x16 s[2];                                     // of 32 keys, and of the next
        float top[2];                                    // the lane's largest exponent of a weight
        auto read_k = [&](int buffer, int sub, int c) { kf[c] = *(LdsB128)(k_from + buffer * Tile::kBuffer + sub * (32 * Tile::kRowK) + c * 32); };
        auto read_v = [&](int buffer, int sub, int d, int m) {
            const unsigned from = v_from + buffer * Tile::kBuffer + (sub * 32 + m * 16) * Tile::kRowV + d * 64;
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsB64)from), hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsB64)(from + 8 * Tile::kRowV));
            vf[d][m] = __builtin_bit_cast(f16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        auto largest_of = [&](int y) {
            float mx = s[y][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) mx = __builtin_elementwise_maximum(mx, s[y][i]);
            return mx;
        };
        auto top_of = [&](float score) { return fmaf(score, a.scale_log2e, -mc); };
        auto score = [&](int y, int c) {
            if (c == 0)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[y][i] = 0.f;
            s[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[c], qf[c], s[y], 0, 0, 0);
        };
        auto value = [&](int y, int m, int d) { o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[d][m], pf[y][m], o[d], 0, 0, 0); };
        // What the row does not see of 32 keys; where values that are not numbers became zeros, a row that sees one of them is undefined by its sum.
        auto hide = [&](f32x16& scores, int y, const uint2& info, int buffer) {
            const unsigned odd = *reinterpret_cast<const uint32_t*>(lds + Tile::kFlags + buffer * 8 + y * 4);
            unsigned seen_keys = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int seen = min((int)((unsigned)__builtin_amdgcn_readlane(info.x, y * 2 + j) >> 16 & 31u), my_pos + 1 - __builtin_amdgcn_readlane(info.y, y * 2 + j));
                seen_keys |= ((1u << max(seen, 0)) - 1u) << (16 * j);
                const int mine = seen - 4 * h;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float v = scores[8 * j + i];
                    scores[8 * j + i] = (i & 3) + 8 * (i >> 2) < mine ? v : -INFINITY;
                }
            }
            if (odd & seen_keys) l = NAN;
        };
        // Moves the reference of rows that have a score too far above it, and with it what the weights so far have left: results, sum, and the weights before, whose values are still to come.
        auto settle = [&](int y) {
            if (!__any(top[y] > lim)) return;
            const float mx = fmaxf(top[y], __shfl_xor(top[y], 32, 64));
            if (mx > lim) {
                const float to = ceilf(mx + mc) - kManyAbove, al = lim == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - to);
                l *= al;
                mc = to;
                lim = kManyRoom;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] *= al;
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int i = 0; i < 8; ++i) pf[1 - y][m][i] = (_Float16)((float)pf[1 - y][m][i] * al);
            }
        };
        // A phase: the weights of keys y beside the scores of the next (kf) and the values of those before (vf), a matrix instruction (32 cycles) and what a lane computes meanwhile, in this order: a
        // weight or two, the rounding and sum of those before, the largest of the new scores, and more(i): reads, conversions.
        auto phase = [&](int y, auto more) {
            constexpr int NM = KS + 2 * DT, EP = 16 / NM, kDone = D == 128 ? NM - 2 : NM;
            const int z = 1 - y;
            float w[16], sum = 0.f, mx = 0.f;
            uint32_t words[2][4];
            auto round_pair = [&](int i) {
                words[i / 4][i % 4] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{w[2 * i], w[2 * i + 1]}, f16x2));
                sum += w[2 * i] + w[2 * i + 1];
                asm volatile("" : "+v"(words[i / 4][i % 4]), "+v"(sum));
            };
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                if (i < KS) score(z, i);
                else value(z, (i - KS) / DT, (i - KS) % DT);
#pragma unroll
                for (int e = 0; e < EP; ++e) {
                    w[i * EP + e] = __builtin_amdgcn_exp2f(top_of(s[y][i * EP + e]));
                    asm volatile("" : "+v"(w[i * EP + e]));      // (formed in this place)
                }
                if (EP == 1 ? i >= 2 && i % 2 == 0 : i >= 1) round_pair(EP == 1 ? i / 2 - 1 : i - 1);
                // from three instructions behind the last scores' on, 16 of them over the instructions that are left (heads of 128: up to the last but two, as the next phase begins with their largest)
                constexpr int kFrom = KS + 2, kEach = (16 + kDone - kFrom - 1) / (kDone - kFrom);
                if (i >= kFrom) {
#pragma unroll
                    for (int e = (i - kFrom) * kEach; e < (i - kFrom + 1) * kEach && e < 16; ++e)
                        mx = e == 0 ? s[z][e] : __builtin_elementwise_maximum(mx, s[z][e]);      // (fmaxf costs a second instruction for each score)
                    asm volatile("" : "+v"(mx));
                }
                if (i == kDone) {
                    top[z] = top_of(mx);
                    asm volatile("" : "+v"(top[z]));
                }
                more(i);
                __builtin_amdgcn_sched_barrier(0);
            }
            round_pair(7);
            if (kDone == NM) top[z] = top_of(mx);
            l += sum;
#pragma unroll
            for (int m = 0; m < 2; ++m) pf[y][m] = __builtin_bit_cast(f16x8, make_uint4(words[m][0], words[m][1], words[m][2], words[m][3]));
            asm volatile("" : "+v"(pf[y][0]), "+v"(pf[y][1]), "+v"(l));
        };

        constexpr std::false_type as_f16;
        constexpr std::true_type as_bf16;
        int loop = __builtin_amdgcn_readfirstlane(!any ? 0 : apart ? 2 : 1);
        if (loop == 1) {
            // Two tiles of 64 keys in LDS, a third in registers, on its way.  Turn i reads the Values of tiles i - 1 and i and the Keys of i + 1, and fills the buffer of i + 2, which is that of
            // i - 2: turn i - 1 was the last to read it, turn i + 1 is the first to read what it gets.  So one barrier, at a turn's end, keeps both apart.
            uint2 info = info_new, info_1, info_2;
            bool whole = all_full(info);
            if (!whole) clear_odd(0);
#pragma unroll
            for (int i = 0; i < 4; ++i) fill_part(0, i, as_f16);
            bool next = advance();
            read_list();
            load();
            info_1 = info_new;
            bool whole_1 = all_full(info_1);
            if (!whole_1) clear_odd(1);
#pragma unroll
            for (int i = 0; i < 4; ++i) fill_part(1, i, as_f16);
            bool after = next && advance();
            read_list();
            load();
            info_2 = info_new;
            bool whole_2 = all_full(info_2);
            __syncthreads();
#pragma unroll
            for (int c = 0; c < KS; ++c) read_k(0, 0, c);
#pragma unroll
            for (int m = 0; m < 2; ++m) pf[1][m] = f16x8{};      // (the first phase's values: nothing, or undefined where they are undefined for all rows)
#pragma unroll
            for (int c = 0; c < KS; ++c) score(0, c);
            top[0] = top_of(largest_of(0));
#pragma unroll
            for (int c = 0; c < KS; ++c) read_k(0, 1, c);
            int buffer = 0, behind = 0;                  // of the present keys, of those before
            while (true) {
                const int ahead = (buffer + 1) & 3, filled = (buffer + 2) & 3;
                if (!whole) {
                    hide(s[0], 0, info, buffer);
                    top[0] = top_of(largest_of(0));
                }
                settle(0);
                phase(0, [&](int i) {
                    if (i < 2 * DT) read_v(behind, behind == buffer ? 0 : 1, i % DT, i / DT);
                    if (i >= 2 * DT && i - 2 * DT < KS) read_k(ahead, 0, i - 2 * DT);      // (behind the last keys: whatever lies there, not used)
                });
                if (!whole) {
                    hide(s[1], 1, info, buffer);
                    top[1] = top_of(largest_of(1));
                }
                settle(1);
                if (!whole_2) clear_odd(filled);
                phase(1, [&](int i) {
                    if (i < 2 * DT) read_v(buffer, 0, i % DT, i / DT);
                    if (i >= 2 * DT && i - 2 * DT < KS) read_k(ahead, 1, i - 2 * DT);
                    if (i >= KS && (i - KS) % (2 * DT / 4) == 0) fill_part(filled, (i - KS) / (2 * DT / 4), as_f16);      // (behind the last keys: the last codes again, not used)
                });
                __syncthreads();
                if (!next) break;
                info = info_1;
                info_1 = info_2;
                whole = whole_1;
                whole_1 = whole_2;
                next = after;
                after = after && advance();
                read_list();
                load();
                info_2 = info_new;
                whole_2 = all_full(info_2);
                behind = buffer;
                buffer = ahead;
            }
#pragma unroll
            for (int i = 0; i < 2 * DT; ++i) read_v(buffer, 1, i % DT, i / DT);
#pragma unroll
            for (int i = 0; i < 2 * DT; ++i) value(1, i / DT, i % DT);
            // What small weights have lost is 2^-25 times the sum of the Values, 2^16 each, at most: where that is more than 2^-10 of a row's largest result, once more in two terms.
            float most = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(o[d][i]));
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            const unsigned long long lost = __ballot(lim != -INFINITY && most < (float)(u_end - u_begin) * (kPiece * 2.f));
            uint32_t* flags = reinterpret_cast<uint32_t*>(lds + Tile::kLost);
            if (lane == 0) flags[wave] = lost != 0;
            __syncthreads();
            uint32_t any_lost = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) any_lost |= flags[i];
            if (__builtin_amdgcn_readfirstlane(any_lost)) {
                loop = 2;
                e_shift = 0;
                left_power = 1.f;
                begin_pieces();
                first_keys();
                begin_rows();
            }
        }
        if (loop == 2) {
            for (bool next = true; next;) {
                const uint2 info = info_new;
                const bool whole = all_full(info);
                if (!whole) clear_odd(0);
#pragma unroll
                for (int i = 0; i < 4; ++i) fill_part(0, i, as_bf16);
                next = advance();
                read_list();
                load();
                __syncthreads();
#pragma unroll 1
                for (int y = 0; y < 2; ++y) {
#pragma unroll
                    for (int c = 0; c < KS; ++c) read_k(0, y, c);
#pragma unroll
                    for (int c = 0; c < KS; ++c) score(0, c);
                    if (!whole) hide(s[0], y, info, 0);
                    float mx = largest_of(0);
                    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                    if (__any(mx > lim)) {
                        const float now = fmaxf(mx, lim), to = now == -INFINITY ? 0.f : now * a.scale_log2e, al = lim == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - to);
                        lim = now;
                        mc = to;
                        l *= al;
#pragma unroll
                        for (int d = 0; d < DT; ++d) o[d] *= al;
                    }
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        float w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = __builtin_amdgcn_exp2f(top_of(s[0][8 * m + i]));
                        l += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
                        bf16x8 terms[2];
                        bf16_terms<2>(w, terms);
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            read_v(0, y, d, m);
#pragma unroll
                            for (int t = 1; t >= 0; --t) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[d][m]), terms[t], o[d], 0, 0, 0);
                        }
                    }
                }
                __syncthreads();
            }
        }
        __syncthreads();                                 // the buffers are read before they are written again

        const bool whole_tile = from_cost == 0 && take == tile_cost;
        if (from_cost == 0 && threadIdx.x < rows) {
            const int i = row0 + threadIdx.x, n = a.by_group(i);
            const long long to = begin + share - left_over + tile_cost - 1;      // (what the share has taken so far is share - left_over, but for the last one, which ends with its tile)
            const int n_shares = whole_tile ? 1 : (int)(to / share) - share_of + 1;
            a.where[(size_t)(me.lo + n) * a.Hq + g * G + i - n * G] = make_int2(kFewPartRows + (blockIdx.x * 2 + 1) * kManyRows + threadIdx.x, 2 * n_shares + 1);
        }
        l += __shfl_xor(l, 32, 64);
        const int in_tile = wave * 32 + l32;
        if (in_tile < rows) {
            if (whole_tile) {
                bf16_t* dst = out + (size_t)(me.lo + token) * a.ldo + (size_t)(g * G + lrow - token * G) * D + 4 * h;
                const float inv = l == 0.f ? 0.f : left_power / l;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<uint2*>(dst + d * 32 + i * 8) =
                            make_uint2(pack_bf16x2(o[d][4 * i] * inv, o[d][4 * i + 1] * inv), pack_bf16x2(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv));
            } else {
                float* dst = a.part + (size_t)(kFewPartRows + (blockIdx.x * 2 + (from_cost == 0)) * kManyRows + in_tile) * (D + 4);
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(dst + d * 32 + i * 8 + 4 * h) = f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]} * left_power;
                if (h == 0) { dst[D] = mc; dst[D + 1] = l; }
            }
        }
        left_over -= take;
        if (left_over <= 0) return;
        from_cost = 0;
        if (++tile == tiles_of(me)) {
            tile = 0;
            unsigned long long more_rows = __ballot(x.n > 0) & ~((2ull << i_req) - 1);
            while (!more_rows) {
                r0 += 64;
                if (r0 >= a.R) return;
                x = request(r0 + lane);
                more_rows = __ballot(x.n > 0);
            }
            i_req = __builtin_ctzll(more_rows);
            me = BatchRequest{wave_value(x.lo, i_req), wave_value(x.n, i_req), wave_value(x.len, i_req)};
        }
    }
}

// The partial results of a row (t, h), merged: a group of D / 4 lanes takes one in NG of them, four channels a lane.
template <typename T, int D, int NG>
__global__ void __launch_bounds__(256) batch_merge_kernel(T* __restrict__ out, BatchAttnArgs a) {
    constexpr int LN = D / 4, PER = 256 / (LN * NG);     // lanes a group, rows a workgroup
    __shared__ float ms[NG][PER], ls[NG][PER];
    __shared__ __align__(16) float os[NG][PER][D];
    const int tid = threadIdx.x, c = tid % LN, grp = tid / LN % NG, x = tid / (LN * NG);
    const long long row = (long long)blockIdx.x * PER + x;
    const int t = (int)(row / a.Hq);
    int first = 0, n = 0, apart = 0, back = 0;           // in rows of `part`: from share to share, from the first one's second tile to the others' first
    const int2 at = a.where[min(row, (long long)a.n_rows * a.Hq - 1)];
    if (t >= max(a.row_start[0], 0) && t < min(a.row_start[a.R], a.n_rows)) {
        const bool many = at.y & 1;
        first = at.x;
        n = at.y >> 1;
        back = many ? kManyRows : a.tile_rows;
        apart = 2 * a.Hkv * back;
        if (n <= 1 || first < back || first - back + (long long)(n - 1) * apart >= (many ? kPartRows : kFewPartRows)) n = 0;
    }
    const float* p = a.part + (size_t)first * (D + 4);
    float M = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    constexpr int kAtOnce = NG == 1 ? 3 : 8;             // requested together (NG 1, two or three partial results a row in most cases: 1511 queries of 28 heads 13.5, 12.8, 13.9 and 19.0 us with 2, 3, 4 and 8)
    for (int y0 = grp; y0 < n; y0 += NG * kAtOnce) {
        float2 st[kAtOnce];
        f32x4 v[kAtOnce];
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b) {
            const int y = min(y0 + b * NG, n - 1);       // the first one is what its share has left unfinished
            const float* s = p + (y == 0 ? 0ll : (long long)y * apart - back) * (D + 4);
            st[b] = *reinterpret_cast<const float2*>(s + D);
            v[b] = *reinterpret_cast<const f32x4*>(s + c * 4);
        }
        float now = M;
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b) {
            if (y0 + b * NG >= n) st[b].y = 0.f;
            if (st[b].y != 0.f) now = fmaxf(now, st[b].x);         // (a partial result without keys has no weight)
        }
        const float al = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(M - now);
        M = now;
        l *= al;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] *= al;
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b) {
            const float w = st[b].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(st[b].x - M);
            l += w * st[b].y;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += w * v[b][e];
        }
    }
    if constexpr (NG > 1) {
        if (c == 0) { ms[grp][x] = M; ls[grp][x] = l; }
        *reinterpret_cast<f32x4*>(&os[grp][x][c * 4]) = f32x4{o[0], o[1], o[2], o[3]};
        __syncthreads();
        if (grp != 0) return;
        float top = M;
#pragma unroll
        for (int y = 1; y < NG; ++y) top = fmaxf(top, ms[y][x]);
        float al = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(M - top);
        l *= al;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] *= al;
#pragma unroll
        for (int y = 1; y < NG; ++y) {
            al = ls[y][x] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ms[y][x] - top);
            l += ls[y][x] * al;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += al * os[y][x][c * 4 + e];
        }
    }
    if (n == 0) return;
    T* dst = out + (size_t)t * a.ldo + (size_t)(row - (long long)t * a.Hq) * D + c * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) Elem<T>::st(dst + e, l == 0.f ? 0.f : o[e] / l);
}

static size_t batch_part_bytes(int n_rows, int Hq, int Hkv, int d) {
    const bool many = (long long)n_rows * (Hq / Hkv) > kFewRows;      // (of either type, so that one workspace serves both)
    return align_up((size_t)(many ? kPartRows : kFewPartRows) * (d + 4) * sizeof(float), 256);
}
size_t batch_attn_kv8_workspace_bytes(int n_rows, int Hq, int Hkv, int d) { return batch_part_bytes(n_rows, Hq, Hkv, d) + align_up((size_t)n_rows * Hq * sizeof(int2), 256); }

// Raises a kernel's LDS limit, once on each device.
constexpr int kDevices = 64;
struct Raised { std::once_flag once[kDevices]; hipError_t err[kDevices] = {}; };
template <typename K> static int raise_lds(K kernel, int bytes, Raised& raised) {
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return set_hip_error(e);
    if (dev < 0 || dev >= kDevices) return SLIM_UNSUPPORTED;
    std::call_once(raised.once[dev], [&] { raised.err[dev] = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); });
    return raised.err[dev] == hipSuccess ? SLIM_OK : set_hip_error(raised.err[dev]);
}

template <typename T, int D, int NR>
static int launch_few(const void* q, void* out, BatchAttnArgs& a, hipStream_t st) {
    const int shares = std::max(1, batch_grid<T, D, NR>() / a.Hkv);
    const long long rows = (long long)a.n_rows * a.Hq;
    a.by_shares = Divide(shares);
    a.tile_rows = NR * kTileRows;
    constexpr int NW = kBatchWaves, smem = NW * RowTile<T, D>::kLdsBytes;
    static_assert(smem < 1 << 16 && batch_grid<T, D, NR>() * 2 * NR * kTileRows <= kFewPartRows, "within the limit that needs no raising, and the workspace");
    hipLaunchKernelGGL((batch_attn_kv8_kernel<T, D, NW, NR>), dim3(shares * a.Hkv), dim3(64 * NW), smem, st, (const T*)q, (T*)out, a);
    const int rc = check_launch();
    if (rc || shares == 1) return rc;                    // (no tile is shared)
    constexpr int kOne = 256 / (D / 4);                  // rows of a workgroup without groups
    // Many rows have few partial results each, and a group of lanes for each is enough (256 new tokens of 32 heads 5.1 us, with kOne groups 11.5); few have many (131072 tokens 5.2, with one 15.9).
    if (rows >= kBatchGrid * 4)
        hipLaunchKernelGGL((batch_merge_kernel<T, D, 1>), dim3((unsigned)((rows + kOne - 1) / kOne)), dim3(256), 0, st, (T*)out, a);
    else
        hipLaunchKernelGGL((batch_merge_kernel<T, D, kOne>), dim3((unsigned)rows), dim3(256), 0, st, (T*)out, a);
    return check_launch();
}

template <typename T, int D>
static int launch_batch_attn(const void* q, void* out, BatchAttnArgs& a, hipStream_t st) {
    if constexpr (sizeof(T) == 2) {
        // The host knows only how many rows there are altogether, and from them what the batch can hold.
        // A request of more than kFewRows takes the kernel for many, if it is launched: empty, that costs 3 to 5 us.  It is where rows and requests leave room for two of its tiles beside a token
        // for each request, or for more than 16 rows a request: 255 new tokens behind 1400 with 64, 256, 512 queries behind 8192 take 203, 230, 265 us with it, 178, 265, 376 without.
        // kFewRows: 8 requests of 8192 tokens with 64 rows each take 70 us in tiles of 32 rows, 81 in those for many, with 96 rows 89 and 84, with 128 96 and 86.
        const int G = a.Hq / a.Hkv;
        const long long rows = (long long)a.n_rows * G;
        const bool longer = rows > (long long)kTileRows * a.R;
        if (rows > kFewRows && (longer || (long long)(a.n_rows - a.R) * G > 2 * kManyRows)) {
            constexpr int many_smem = ManyTile<D>::kLdsBytes;
            static Raised raised;
            if (const int rc = raise_lds(batch_attn_many_kernel<D>, many_smem, raised)) return rc;
            a.few = kFewRows;
            hipLaunchKernelGGL((batch_attn_many_kernel<D>), dim3(std::max(1, kManyGrid / a.Hkv) * a.Hkv), dim3(512), many_smem, st, (const bf16_t*)q, (bf16_t*)out, a);
            if (const int rc = check_launch()) return rc;
        }
        // Tiles of 32 rows read the keys half as often: 64 requests of 4096 tokens and 20 rows 110 us, with tiles of 16 rows 195; of 2048 tokens and 64 rows 121 and 193; a single request of
        // 2048 tokens and 64 rows, which leaves workgroups free, 21 and 18.
        if (longer) return launch_few<T, D, 2>(q, out, a, st);
    }
    return launch_few<T, D, 1>(q, out, a, st);
}

int launch_batch_attn_kv8(const void* q, int ldq, const int* row_start, const int* lens, const int* table, int R, int n_rows, int max_blocks, const void* pool, int n_slots, size_t slot_bytes,
                          size_t layer_offset, int block, int Hq, int Hkv, int d, float scale, int dtype, void* out, int ldo, void* workspace, hipStream_t st) {
    const int per_block = (block + kPiece - 1) / kPiece;
    BatchAttnArgs a{row_start, lens, table, (const unsigned char*)pool, slot_bytes, layer_offset, (float*)workspace, (int2*)((char*)workspace + batch_part_bytes(n_rows, Hq, Hkv, d)),
                    scale * 1.4426950408889634f, R, max_blocks, n_slots, n_rows, block, per_block, Hq, Hkv, ldq, ldo, 0x7fffffff, kTileRows, Divide(block), Divide(per_block), Divide(Hq / Hkv), Divide(1)};
    if (dtype == SLIM_BF16) return d == 64 ? launch_batch_attn<bf16_t, 64>(q, out, a, st) : launch_batch_attn<bf16_t, 128>(q, out, a, st);
    return d == 64 ? launch_batch_attn<float, 64>(q, out, a, st) : launch_batch_attn<float, 128>(q, out, a, st);
}

}  // namespace slim
