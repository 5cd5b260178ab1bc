// Tables of a batch of requests, from their lengths: the rows of the step, where they go in the pool of blocks, and the slots that new blocks take from a list of free ones.
//
//   row_start[r] = sum of n_new below r;   had(r) = ceil(lens[r] / block), need(r) = ceil((lens[r] + n_new[r]) / block);   first(r) = used + sum of need - had below r
//   block_table[r, had(r) + i] = free_slots[first(r) + i];   row t of request r: position lens[r] + t - row_start[r], and the entry of its block times block plus its row there
//
// One launch: every workgroup forms both sums for itself in LDS, since a row needs all of them in front of it, and takes a share of the rows and of the new blocks (there are no
// more new blocks than rows).  A row finds its request by bisection of row_start; its block's slot comes from the table where the block was there and from the list where it is new, so
// that no workgroup reads what another one writes.  What is read and written is small (32768 rows: 0.26 MB); bound by the trips to memory one behind the other: 4.4 us for 256 requests of a
// token, 4.3 for 37 prompts of 26028, of which 2.5 are a launch's.
#include "slim_common.h"
#include "batch.h"
#include <algorithm>

namespace slim {

constexpr int kMapThreads = 256;

struct BatchMapArgs {
    const int *lens, *n_new, *free_slots, *used;
    int *table, *lens_out, *row_start, *row_pos, *row_slot, *info;
    int R, block, max_blocks, n_free, n_slots, n_rows;
};

// Largest i in [0, n) with v[i] <= x; v ascending, v[0] <= x.
__device__ __forceinline__ int last_not_above(const int* v, int n, int x) {
    int lo = 0;
    while (n > 1) {
        const int half = n >> 1;
        if (v[lo + half] <= x) lo += half;
        n -= half;
    }
    return lo;
}

__global__ void __launch_bounds__(kMapThreads) batch_map_kernel(BatchMapArgs a) {
    extern __shared__ int lds[];
    int* start = lds;                                    // [R + 1]
    int* first = lds + a.R + 1;                          // [R + 1], without `used`
    __shared__ long long wave_rows[kMapThreads / 64], wave_blocks[kMapThreads / 64];
    __shared__ int wave_err[kMapThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (a.R + kMapThreads - 1) / kMapThreads, r0 = min(a.R, tid * per), r1 = min(a.R, r0 + per);
    const long long room = (long long)a.max_blocks * a.block;
    auto request = [&](int r, int& rows, int& blocks) {  // false: its lengths are not ones that a table has room for
        const int len = a.lens[r], n = a.n_new[r];
        const long long end = (long long)len + n;
        if (len < 0 || n < 0 || end > room) { rows = blocks = 0; return false; }
        rows = n;
        blocks = (int)((end + a.block - 1) / a.block - ((long long)len + a.block - 1) / a.block);
        return true;
    };
    long long rows = 0, blocks = 0;
    int err = 0;
    for (int r = r0; r < r1; ++r) {
        int n, b;
        if (!request(r, n, b)) err = 1;
        rows += n;
        blocks += b;
    }
    long long row_sum = rows, block_sum = blocks;        // of the wave's lanes up to this one
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long x = __shfl_up(row_sum, o, 64), y = __shfl_up(block_sum, o, 64);
        if (lane >= o) { row_sum += x; block_sum += y; }
    }
    if (lane == 63) { wave_rows[wave] = row_sum; wave_blocks[wave] = block_sum; }
    const bool bad = __any(err);
    if (lane == 0) wave_err[wave] = bad;
    __syncthreads();
    long long row_at = row_sum - rows, block_at = block_sum - blocks, all_rows = 0, taken = 0;
    err = 0;
#pragma unroll
    for (int w = 0; w < kMapThreads / 64; ++w) {
        if (w < wave) { row_at += wave_rows[w]; block_at += wave_blocks[w]; }
        all_rows += wave_rows[w];
        taken += wave_blocks[w];
        err |= wave_err[w];
    }
    const int used = a.used ? *a.used : 0;
    if (all_rows > a.n_rows) err |= 2;
    if (used < 0 || used + taken > a.n_free) err |= 4;
    if (err) all_rows = taken = 0;
    for (int r = r0; r < r1; ++r) {                      // (with an error the sums may be beyond 32 bits, and are not used)
        int n, b;
        request(r, n, b);
        start[r] = err ? 0 : (int)row_at;
        first[r] = err ? 0 : (int)block_at;
        row_at += n;
        block_at += b;
    }
    __syncthreads();

    if (blockIdx.x == 0) {
        for (int r = tid; r < a.R; r += kMapThreads) {
            a.row_start[r] = start[r];
            a.lens_out[r] = a.lens[r] + (err ? 0 : a.n_new[r]);
        }
        if (tid == 0) {
            a.row_start[a.R] = (int)all_rows;
            a.info[0] = (int)all_rows;
            a.info[1] = (int)taken;
            a.info[2] = err;
            a.info[3] = used + (int)taken;
        }
    }
    for (long long t = (long long)blockIdx.x * kMapThreads + tid; t < a.n_rows; t += (long long)gridDim.x * kMapThreads) {
        int pos = 0, place = -1;
        if (t < all_rows) {
            const int r = last_not_above(start, a.R, (int)t), len = a.lens[r];
            pos = len + (int)t - start[r];
            const int b = pos / a.block, had = (int)(((long long)len + a.block - 1) / a.block);
            const int slot = b < had ? a.table[(size_t)r * a.max_blocks + b] : a.free_slots[used + first[r] + b - had];
            if (slot >= 0 && slot < a.n_slots) place = slot * a.block + (pos - b * a.block);
        }
        a.row_pos[t] = pos;
        a.row_slot[t] = place;
        if (t < taken) {
            const int r = last_not_above(first, a.R, (int)t);
            const int had = (int)(((long long)a.lens[r] + a.block - 1) / a.block);
            a.table[(size_t)r * a.max_blocks + had + (int)t - first[r]] = a.free_slots[used + t];
        }
    }
}

int launch_batch_map(const int* lens, const int* n_new, int R, int block, int* table, int max_blocks, const int* free_slots, int n_free, const int* used, int n_slots, int n_rows,
                     int* lens_out, int* row_start, int* row_pos, int* row_slot, int* info, hipStream_t st) {
    const BatchMapArgs a{lens, n_new, free_slots, used, table, lens_out, row_start, row_pos, row_slot, info, R, block, max_blocks, n_free, n_slots, n_rows};
    const int grid = std::min((n_rows - 1) / kMapThreads + 1, 1024);
    hipLaunchKernelGGL(batch_map_kernel, dim3(grid), dim3(kMapThreads), 2 * (R + 1) * sizeof(int), st, a);
    return check_launch();
}

}  // namespace slim
