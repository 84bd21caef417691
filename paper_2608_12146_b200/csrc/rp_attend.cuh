// What the attention kernels share: the list of blocks of tokens that the CTAs take, and how they share it out.
#pragma once

#include "rp_tensor.cuh"

struct AttendHead { int status, count, pad[2]; };       // front of the workspace; items [count] behind it: (sample, block of its tokens)
struct AttendClear { void *x; i64 token, head; int heads, d, bytes; };
struct AttendPlan {
    const i64 *start;
    i64 T;
    int N, rows, causal, by_key, most;                  // most: room for items
    AttendHead *head;
    int2 *items;
    AttendClear clear[3];                                // outputs whose rows of no sample are cleared
    int n_clear;
};
int rp_launch_attend_plan(const AttendPlan &A, cudaStream_t stream);
int rp_attend_check(const rp_attend_config *a, i64 T, int N);
int rp_attend_view(const rp_view *v, i64 T, int heads, RpOpDevice &dev);

// The attention kernels have twelve warps: eight for the softmax, in two groups of four (a warp reaches the 32 rows of tensor memory that go by its number), one that
// copies, one that issues the products, two that wait.  The latter four give registers to the former eight: 4 * 32 * 72 + 8 * 32 * 216 = 12 * 32 * 168.
#define ATTEND_THREADS 384
#define ATTEND_COPY_WARP 8
#define ATTEND_MMA_WARP 9
__device__ __forceinline__ void rp_many_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 216;"); }
__device__ __forceinline__ void rp_few_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 72;"); }

// The CTA's item of a round, -1 when there is none: rounds go through the list forwards and backwards in turn, so that who gets the largest of one
// round gets the smallest of the next.
__device__ __forceinline__ int rp_attend_item(int round, int total)
{
    const int n = gridDim.x, b = round & 1 ? n - 1 - blockIdx.x : blockIdx.x;
    const i64 at = (i64)round * n + b;
    return at < total ? (int)at : -1;
}

// A block of tokens: its sample's first token and length, its own first token inside the sample.
struct AttendTile {
    i64 base;
    int len, row0;
    __device__ __forceinline__ AttendTile(const int2 *items, const i64 *start, i64 T, int item, int rows)
    {
        const int2 it = items[item];
        base = max(start[it.x], (i64)0);
        len = (int)(min(start[it.x + 1], T) - base);
        row0 = it.y * rows;
    }
};
// Tiles of 128 keys that the i-th tile of 128 queries of a block sees.
__device__ __forceinline__ int rp_attend_tiles(const AttendTile &t, int i, int causal)
{
    const int seen = causal ? min(t.len, t.row0 + 128 * i + 128) : t.len;
    return (seen + 127) >> 7;
}

// Rows [from, to) of a tile in shared memory become 0, by one warp, before the tensor cores read them.  (A row is 128 bytes of each panel; the swizzle moves
// 16-byte pieces inside a row only.)
template <int D, int ROWS = 128>
__device__ __forceinline__ void rp_clear_rows(unsigned char *tile, int from, int to, int lane)
{
    for (int p = 0; p < D / 64; ++p)
        for (int x = max(from, 0) * 8 + lane; x < to * 8; x += 32) *(uint4 *)(tile + p * ROWS * 128 + x * 16) = make_uint4(0, 0, 0, 0);
    fence_async();
    __syncwarp();
}

// A copy that was under way when a wait ran out: two seconds at most.
__device__ __forceinline__ void rp_drain(u32 bar, u32 parity)
{
    const u64 since = rp_nanoseconds();
    while (!bar_try(bar, parity) && rp_nanoseconds() - since < 2000000000ull) { }
}
