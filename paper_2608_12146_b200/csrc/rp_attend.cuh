// What the attention kernels share: the list of blocks of tokens that the CTAs take, and how they share it out.
#pragma once

#include "rp_tensor.cuh"

struct AttendHead { int status, count, ticket, pad; };  // front of the workspace; items [count] behind it: (sample, block of its tokens); ticket: items taken so far
struct AttendClear { void *x; i64 token, head; int heads, d, bytes; };
struct AttendPlan {
    const i64 *start;
    i64 T;
    int N, rows, causal, by_key, most;                  // most: room for items
    AttendHead *head;
    int2 *items;
};
struct AttendClears { AttendClear x[3]; int n; };       // outputs whose rows of no sample are cleared

// By one CTA of 1024 threads: lists the blocks of `rows` tokens of all samples, those with the most tiles of others first.
// Work of a block: queries (by_key 0) see the keys up to them, keys (by_key 1) are seen by the queries from them on.
#define PLAN_BUCKETS 1024
static __device__ __noinline__ void rp_attend_plan(const AttendPlan &A)
{
    __shared__ int count[PLAN_BUCKETS];
    __shared__ int from[PLAN_BUCKETS], sums[32];
    for (int x = threadIdx.x; x < PLAN_BUCKETS; x += 1024) count[x] = 0;
    __syncthreads();
    for (int pass = 0; pass < 2; ++pass) {
        // A lane a sample; samples of many blocks then by the whole warp, one after the other.  (4096 samples of 8 tokens, 8 heads on 2: 891 us with a warp a
        // sample, 729 so.)
        const int lane = threadIdx.x & 31;
        for (int i0 = threadIdx.x & ~31; i0 < A.N; i0 += 1024) {
            const int i = i0 + lane;
            const i64 lo = i < A.N ? max(A.start[i], (i64)0) : 0, hi = i < A.N ? min(A.start[i + 1], A.T) : 0;
            const int blocks = hi > lo ? (int)((hi - lo + A.rows - 1) / A.rows) : 0;
            const auto take = [&](int sample, int n, int b) {
                const int work = !A.causal ? n : A.by_key ? n - b : b + 1;
                const int bucket = PLAN_BUCKETS - 1 - min(work - 1, PLAN_BUCKETS - 1);
                if (pass == 0) atomicAdd(&count[bucket], 1);
                else {
                    const int at = atomicAdd(&from[bucket], 1);
                    if (at < A.most) A.items[at] = make_int2(sample, b);
                }
            };
            if (blocks <= 4)
                for (int b = 0; b < blocks; ++b) take(i, blocks, b);
            for (u32 many = __ballot_sync(0xffffffffu, blocks > 4); many; many &= many - 1) {
                const int who = __ffs((int)many) - 1, n = __shfl_sync(0xffffffffu, blocks, who);
                for (int b = lane; b < n; b += 32) take(i0 + who, n, b);
            }
        }
        __syncthreads();
        if (pass == 0) {
            // a thread a bucket
            const int warp = threadIdx.x >> 5, c = count[threadIdx.x];
            int x = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            if (lane == 31) sums[warp] = x;
            __syncthreads();
            int before = warp ? sums[lane < warp ? lane : 0] : 0;
            if (lane >= warp) before = 0;
            before = __reduce_add_sync(0xffffffffu, before);
            from[threadIdx.x] = before + x - c;
            if (threadIdx.x == 1023) { A.head->count = min(before + x, A.most); A.head->status = 0; A.head->ticket = 0; }
            __syncthreads();
        }
    }
}
// By CTAs of 1024 threads, this one the b-th of n: clears the rows that no sample holds.
static __device__ __noinline__ void rp_attend_clear(const AttendClears &A, const i64 *start, int N, i64 T, int b, int n)
{
    i64 head = start[0], tail = start[N];
    head = min(max(head, (i64)0), T); tail = min(max(tail, head), T);
    const i64 gone = head + T - tail;
    for (int o = 0; o < A.n; ++o) {
        const AttendClear &C = A.x[o];
        const i64 width = (i64)C.heads * C.d;
        for (i64 x = (i64)b * 1024 + threadIdx.x; x < gone * width; x += (i64)n * 1024) {
            i64 t = x / width;
            const i64 h = x % width / C.d, i = x % C.d;
            t = t < head ? t : tail + t - head;
            const i64 at = t * C.token + h * C.head + i;
            if (C.bytes == 2) ((unsigned short *)C.x)[at] = 0; else ((float *)C.x)[at] = 0.0f;
        }
    }
}
extern i64 g_attend_wait_ns;             // limit of the kernels' waits (rp_debug_set_wait_limit)
int rp_attend_check(const rp_attend_config *a, i64 T, int N);
int rp_attend_view(const rp_view *v, i64 T, int heads, RpOpDevice &dev);
// Is one of the first `n_out` views the same memory as another of them or as one of the `n` behind them?
static inline bool rp_attend_shared(const rp_view *const *v, int n_out, int n)
{
    for (int i = 0; i < n_out; ++i)
        for (int j = i + 1; j < n_out + n; ++j)
            if (v[i] && v[j] && v[i]->x && v[i]->x == v[j]->x) return true;
    return false;
}

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
