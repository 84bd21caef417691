// Gradient of the attention inside the samples of a packed row.
//
//   p = exp(scale q k^T - lse), ds = p (do v^T - delta), delta = sum_d do o;   dv = p^T do, dk = scale ds^T q, dq = scale ds k
//
// float16 has few powers of two: a sample's gradients of scores are multiplied with one that puts the norm of its largest row of do between 8 and 16 before they are
// rounded (so that values to a norm of 2047 cannot leave the range, and gradients of 10^-4 keep their bits), weights with 2^15; both are taken out of the sums.
//
// Two kernels: one takes 128 keys and goes through the queries that see them (dk, dv), one takes 128 queries and goes through the keys that they see
// (dq).  Each output is summed by one CTA in a fixed order: no additions from several CTAs to one place, whose order would change the last bits.  The price is
// that scores and do v^T are worked out twice, 14 multiply-adds a pair and element in place of 10.  Bound by the hand-overs between the warp that issues products and
// those of the softmax: at 4096 tokens the tensor cores are busy for 22 % (keys, which also wait for the largest block) and 56 % (queries) of the time.
// With a window (WINDOW) blocks of keys are seen by a few tiles of queries, blocks of queries see a few tiles of keys, and the sample's first block is seen by all of its
// queries when there are first tokens: it is cut into chunks, whose sums for the first tokens meet in a kernel of their own.  A row of 32768 tokens of one sample, 16 heads on
// 4, 128 wide: 371 us with a window of 128, 929 with 1024 (1037 with 4 first tokens).
#include <algorithm>

#include "rp_attend.cuh"

struct GradArgs {
    const int2 *items;
    AttendHead *head;
    const i64 *start;
    i64 T;
    int Hq, Hk, share, d, causal;
    int window, sinks;
    float *parts;                            // sums of chunks for the first tokens: [place][Hk][dv, dk][sinks][d]
    float scale;
    const float2 *stats;                     // [Hq][T]: lse / ln 2, delta
    const u32 *tops;                         // float16: [samples] square of the norm of the largest row of do, as bits
    void *x[2];                              // dv, dk, or dq
    i64 token[2], hd[2];
    int *status;
    u64 wait_ns;
};

// Before the two kernels: CTA 0 lists the blocks of keys, CTA 1 those of queries, the others clear the rows that no sample holds and work out lse / ln 2 and delta of
// every token and query head: 16 lanes a head, 16 bytes of do and o a lane.
struct StatsArgs {
    const void *o, *g;
    const float *lse;
    i64 o_token, o_head, g_token, g_head, l_token, l_head;
    int H, d;
    float2 *stats;
    float *norms;                            // float16: [H][T] squares of the norms of the rows of do
    u32 *tops;
};
template <typename X> struct Narrow { static constexpr bool value = !std::is_same<X, bf16>::value; };
template <typename X>
__global__ void __launch_bounds__(1024) k_attend_prepare(AttendPlan keys, AttendPlan queries, AttendClears C, StatsArgs A)
{
    rp_let_next_launch_start();
    if (blockIdx.x == 0) { rp_attend_plan(keys); return; }
    if (blockIdx.x == 1) { rp_attend_plan(queries); return; }
    const int b = blockIdx.x - 2, n = gridDim.x - 2, lane = threadIdx.x & 15;
    rp_attend_clear(C, keys.start, keys.N, keys.T, b, n);
    if constexpr (Narrow<X>::value)
        for (int i = b * 1024 + threadIdx.x; i < keys.N; i += n * 1024) A.tops[i] = 0;
    // 64 rows of a CTA: heads of a token, tokens; two steps are worked on while the next two are on their way (all lanes go round as often)
    constexpr int AHEAD = 2;
    const i64 T = keys.T;
    const int heads = max(min(A.H, 64), 1), tokens = 64 / heads, row = threadIdx.x >> 4, dt = row / heads;
    for (int h0 = 0; h0 < A.H; h0 += heads) {
        const int h = h0 + row % heads;
        const bool mine = dt < tokens && h < A.H;
        const X *o = (const X *)A.o + h * A.o_head + lane * 8, *g = (const X *)A.g + h * A.g_head + lane * 8;
        Pack8<X> p[2][AHEAD], q[2][AHEAD];
        float l[2][AHEAD];
        const auto fetch = [&](i64 t0, Pack8<X> *p, Pack8<X> *q, float *l) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const i64 t = t0 + (i64)u * n * tokens + dt;
                p[u] = Pack8<X>(); q[u] = Pack8<X>(); l[u] = 0.0f;
                if (mine && t < T && lane * 8 < A.d) { p[u] = rp_load8(o + t * A.o_token); q[u] = rp_load8(g + t * A.g_token); }
                if (mine && t < T && lane == 0) l[u] = A.lse[t * A.l_token + h * A.l_head];
            }
        };
        const auto work = [&](i64 t0, const Pack8<X> *p, const Pack8<X> *q, const float *l) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const i64 t = t0 + (i64)u * n * tokens + dt;
                float a[8], c[8], sum = 0.0f;
                rp_open8(p[u], a); rp_open8(q[u], c);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf(a[i], c[i], sum);
#pragma unroll
                for (int i = 1; i < 16; i <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, i);
                if (mine && t < T && lane == 0) A.stats[h * T + t] = make_float2(l[u] * RP_LOG2E, sum);
                if constexpr (Narrow<X>::value) {
                    float norm = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) norm = fmaf(c[i], c[i], norm);
#pragma unroll
                    for (int i = 1; i < 16; i <<= 1) norm += __shfl_xor_sync(0xffffffffu, norm, i);
                    if (mine && t < T && lane == 0) A.norms[h * T + t] = norm;
                }
            }
        };
        const i64 step = (i64)AHEAD * n * tokens, from = (i64)b * tokens;
        fetch(from, p[0], q[0], l[0]);
        for (i64 t0 = from; t0 < T; t0 += 2 * step) {
            fetch(t0 + step, p[1], q[1], l[1]);
            work(t0, p[0], q[0], l[0]);
            fetch(t0 + 2 * step, p[0], q[0], l[0]);
            work(t0 + step, p[1], q[1], l[1]);
        }
    }
}

// The largest of a sample's rows of do, for float16 (infinities and NaN, which no factor mends, do not count): a thread a token.
static __device__ __forceinline__ void rp_attend_tops(const i64 *start, int N, i64 T, int H, const float *norms, u32 *tops, int block)
{
    const i64 t = (i64)block * 256 + threadIdx.x;
    float top = 0.0f;
    for (int h = 0; t < T && h < H; ++h) {
        const float x = norms[h * T + t];
        if (x < INFINITY) top = fmaxf(top, x);
    }
    const int i = t < T ? rp_sample_of(start, N, t) : -1;
    u32 bits = i >= 0 && i < N ? __float_as_uint(top) : 0u;
    if (__all_sync(0xffffffffu, i == __shfl_sync(0xffffffffu, i, 0))) {
        bits = __reduce_max_sync(0xffffffffu, bits);
        if (threadIdx.x & 31) bits = 0;
    }
    if (bits) atomicMax(tops + i, bits);
}
__global__ void __launch_bounds__(256) k_attend_tops(const i64 *start, int N, i64 T, int H, const float *norms, u32 *tops) { rp_attend_tops(start, N, T, H, norms, tops, blockIdx.x); }

// With a window: delta of the tokens that see few keys (32 at most) from its definition, sum_j p_j do v_j.  o is as large as v there, and what its rounding leaves in do o is
// as much as the rounding of their scores' gradients (samples of 60 tokens: gradients of queries and keys 1.6 times as far off as with their own rounding alone, 1.42 so;
// from the 33rd key on it is a sixth of that rounding and less).  Those are each sample's first tokens (k_attend_first), and where the window and the first tokens that stay
// visible are as few, all of them (k_attend_few).
// A sample's first tokens: a warp half of a sample's and a query head's.  Behind `first` such CTAs those for float16's largest rows.
#define FIRST_TOKENS 32
struct FirstArgs {
    const i64 *start;
    i64 T;
    int N, H, share, d, window, sinks;
    float scale;
    const void *q, *k, *v, *g;
    i64 q_token, q_head, k_token, k_head, v_token, v_head, g_token, g_head;
    const float *lse;
    i64 l_token, l_head;
    float2 *stats;
    const float *norms;
    u32 *tops;
    int first;
};
template <typename X>
__global__ void __launch_bounds__(256) k_attend_first(const FirstArgs A)
{
    rp_let_next_launch_start();              // (nothing here is over before the launch in front is: the next one need only wait for this)
    if ((int)blockIdx.x < A.first && threadIdx.x >= 64) return;              // (two warps a CTA: there are few, and their loads go to many lines)
    if ((int)blockIdx.x >= A.first) { rp_wait_for_launch_before(); rp_attend_tops(A.start, A.N, A.T, A.H, A.norms, A.tops, blockIdx.x - A.first); return; }
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    for (i64 unit = (i64)blockIdx.x * 2 + (threadIdx.x >> 5); unit < (i64)A.N * A.H * 2; unit += (i64)A.first * 2) {
        const int i = (int)(unit / (2 * A.H)), h = (int)(unit % (2 * A.H)) >> 1, r0 = 16 * (int)(unit & 1), hk = h / A.share;
        const i64 base = max(A.start[i], (i64)0);
        const int n = (int)min(min(A.start[i + 1], A.T) - base, (i64)FIRST_TOKENS);
        if (r0 >= n) { rp_wait_for_launch_before(); continue; }
        // (rows behind the sample's end are read as its last one: nothing comes of them)
        const int r[2] = { min(r0 + g, n - 1), min(r0 + g + 8, n - 1) };
        // (a lane's eight elements are places 2t, 2t + 1, 2t + 8, 2t + 9 of one product and of the next: the order of a sum's terms is free)
        const X *q = (const X *)A.q + base * A.q_token + h * A.q_head + 8 * t, *o = (const X *)A.g + base * A.g_token + h * A.g_head + 8 * t;
        const X *k = (const X *)A.k + base * A.k_token + hk * A.k_head + 8 * t, *v = (const X *)A.v + base * A.v_token + hk * A.v_head + 8 * t;
        float s[4][4] = { }, dp[4][4] = { };
#pragma unroll 2
        for (int c = 0; c < A.d; c += 32) {
            const bool there = c + 8 * t < A.d;
            const auto at = [&](const X *x, i64 row) { return there ? *(const uint4 *)(x + row + c) : make_uint4(0, 0, 0, 0); };
            const uint4 q0 = at(q, r[0] * A.q_token), q1 = at(q, r[1] * A.q_token), o0 = at(o, r[0] * A.g_token), o1 = at(o, r[1] * A.g_token);
            const u32 a[2][4] = { { q0.x, q1.x, q0.y, q1.y }, { q0.z, q1.z, q0.w, q1.w } }, b[2][4] = { { o0.x, o1.x, o0.y, o1.y }, { o0.z, o1.z, o0.w, o1.w } };
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int j = min(8 * x + g, n - 1);
                const uint4 kk = at(k, j * A.k_token), vv = at(v, j * A.v_token);
                const u32 e[2][2] = { { kk.x, kk.y }, { kk.z, kk.w } }, f[2][2] = { { vv.x, vv.y }, { vv.z, vv.w } };
#pragma unroll
                for (int y = 0; y < 2; ++y) { rp_multiply(s[x], a[y], e[y], X()); rp_multiply(dp[x], b[y], f[y], X()); }
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int row = r0 + g + 8 * u;
            const float lse = A.lse[(base + r[u]) * A.l_token + h * A.l_head];
            float delta = 0.0f;
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int j = 8 * x + 2 * t + y;
                    const bool sees = j <= row && j < n && (row - j < A.window || j < A.sinks);
                    delta += sees ? rp_exp2((s[x][2 * u + y] * A.scale - lse) * RP_LOG2E) * dp[x][2 * u + y] : 0.0f;
                }
            delta += __shfl_xor_sync(0xffffffffu, delta, 1);
            delta += __shfl_xor_sync(0xffffffffu, delta, 2);
            rp_wait_for_launch_before();                     // (it writes a delta here, too)
            if (row < n && t == 0) A.stats[(i64)h * A.T + base + row].y = delta;
        }
    }
}
// Every token, where none sees more than 32 keys; this takes the place of the statistics that come from o (which, in samples of 1000 tokens, leave gradients of queries and
// keys 1.53 times as far off with a window of 16 as with their own rounding alone, 1.78 times with 4, 2.26 with 2; 1.41 to 1.42 so).  A CTA takes a block of 128 tokens of a
// sample and some of a key head's query heads, a warp 16 of the tokens, whose q and do stay in registers.  Their keys are tiles of 8: those of the first tokens, then the window's,
// from as many before the 16 up to themselves.  All of the block's lie in shared memory, neighbouring rows 64 bytes off each other's banks.  By blocks of the sample, so that its
// bits do not depend on what else is in the row.
// 16384 tokens of two samples, 16 heads on 4, 128 wide (q and do: 134 MB): 49 us with a window of 16, 70 with 28 and 4 first tokens; the whole gradient 230 and 305 us, where delta
// from o takes 211 and 262.  It waits for q and do, which a warp asks for between two pieces of work.
#define FEW_KEYS 32
struct FewArgs {
    FirstArgs of;
    const AttendHead *head;                  // the blocks of queries
    const int2 *items;
    int parts;                               // a key head's query heads are dealt out to as many CTAs
    int ahead, before, tiles;                // tiles of first tokens, of keys before a warp's tokens, in all: 7 at most
};
template <int D> struct FewRow { unsigned char at[2 * D + 64]; };
__device__ __forceinline__ void copy_piece(void *to, const void *from, bool there)       // 16 bytes, or as many zeros, in the background
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(rp_smem(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void pieces_copied() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// A lane's part of what 16 rows see of some tiles: rows lane / 4 and 8 on, of each tile the keys 2 (lane % 4) and 1 on; sees(tile, key, row) as bits.
template <typename Sees> __device__ __forceinline__ u32 few_mask(int tiles, const Sees &sees)
{
    const int lane = threadIdx.x & 31;
    u32 mask = 0;
    for (int i = 0; i < 4 * tiles; ++i) mask |= sees(i >> 2, 2 * (lane & 3) + (i & 1), (lane >> 2) + 8 * (i >> 1 & 1)) ? 1u << i : 0u;
    return mask;
}
template <typename X, int D>
__global__ void __launch_bounds__(256, 2) k_attend_few(const FewArgs F)
{
    extern __shared__ __align__(16) unsigned char raw[];
    const FirstArgs &A = F.of;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, ahead = F.ahead, before = F.before, tiles = F.tiles, rows = 112 + 8 * tiles;
    FewRow<D> *const keys = (FewRow<D> *)raw, *const values = keys + rows;
    rp_let_next_launch_start();
    rp_wait_for_launch_before();             // the list of blocks; float16's largest rows are 0
    const int each = A.H / A.share * F.parts;            // units of a block
    const i64 total = (i64)F.head->count * each;
    // (behind all first tokens and the window's reach of them, what a place sees is the same everywhere)
    const u32 mask_far = few_mask(tiles, [&](int x, int e, int row) {
        const int back = row + 8 * before - 8 * (x - ahead) - e;
        return x < ahead ? 8 * x + e < A.sinks : back >= 0 && back < A.window;
    });
    for (i64 unit = blockIdx.x; unit < total; unit += gridDim.x) {
        const int item = (int)(unit / each), hk = (int)(unit % each) / F.parts, part = (int)(unit % each) % F.parts;
        const AttendTile block(F.items, A.start, A.T, item, 128);
        const X *const k = (const X *)A.k + block.base * A.k_token + hk * A.k_head, *const v = (const X *)A.v + block.base * A.v_token + hk * A.v_head;
        const int near0 = block.row0 - 8 * before;       // the key behind the first tokens' rows
        __syncthreads();                                 // (the block before has been read)
        for (int x = threadIdx.x; x < rows * (D / 8); x += 256) {
            const int y = x / (D / 8), c = x % (D / 8), j = min(max(y < 8 * ahead ? y : near0 + y - 8 * ahead, 0), block.len - 1);
            const bool there = 8 * c < A.d;
            copy_piece(keys[y].at + 16 * c, k + j * A.k_token + (there ? 8 * c : 0), there);
            copy_piece(values[y].at + 16 * c, v + j * A.v_token + (there ? 8 * c : 0), there);
        }
        pieces_copied();
        __syncthreads();
        const int w0 = 16 * (threadIdx.x >> 5), r0 = block.row0 + w0, near = r0 - 8 * before;
        if (r0 >= block.len) continue;
        const u32 mask = near >= A.sinks ? mask_far : few_mask(tiles, [&](int x, int e, int row) {
            const int j = x < ahead ? 8 * x + e : near + 8 * (x - ahead) + e, y = r0 + row;
            return j >= 0 && j <= y && (x >= ahead || j < near) && (y - j < A.window || j < A.sinks);
        });
        // (rows behind the sample's end are read as its last one: nothing comes of them)
        const int r[2] = { min(r0 + g, block.len - 1), min(r0 + g + 8, block.len - 1) };
        float top = 0.0f;
        for (int h = hk * A.share + part; h < (hk + 1) * A.share; h += F.parts) {
            // (a lane's eight elements are places 2t, 2t + 1, 2t + 8, 2t + 9 of one product and of the next: the order of a sum's terms is free)
            const X *const q = (const X *)A.q + block.base * A.q_token + h * A.q_head + 8 * t, *const o = (const X *)A.g + block.base * A.g_token + h * A.g_head + 8 * t;
            u32 a[D / 16][4], b[D / 16][4];
            float delta[2] = { 0.0f, 0.0f }, lse[2], norm[2] = { 0.0f, 0.0f };
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                lse[u] = A.lse[(block.base + r[u]) * A.l_token + h * A.l_head];
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint4 x = make_uint4(0, 0, 0, 0), y = x;
                    if (32 * c + 8 * t < A.d) { x = *(const uint4 *)(q + r[u] * A.q_token + 32 * c); y = *(const uint4 *)(o + r[u] * A.g_token + 32 * c); }
                    a[2 * c][u] = x.x; a[2 * c][2 + u] = x.y; a[2 * c + 1][u] = x.z; a[2 * c + 1][2 + u] = x.w;
                    b[2 * c][u] = y.x; b[2 * c][2 + u] = y.y; b[2 * c + 1][u] = y.z; b[2 * c + 1][2 + u] = y.w;
                }
            }
            if constexpr (Narrow<X>::value) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        Pack8<X> p;
                        float w[8];
                        p.w[0] = make_uint4(b[2 * c][u], b[2 * c][2 + u], b[2 * c + 1][u], b[2 * c + 1][2 + u]);
                        rp_open8(p, w);
#pragma unroll
                        for (int i = 0; i < 8; ++i) norm[u] = fmaf(w[i], w[i], norm[u]);
                    }
            }
            u32 bits = mask;
#pragma unroll 1
            for (int x = 0; x < tiles; ++x, bits >>= 4) {
                const int y = (x < ahead ? 0 : w0) + 8 * x + g;
                const unsigned char *const kr = keys[y].at + 16 * t, *const vr = values[y].at + 16 * t;
                float s[4] = { }, dp[4] = { };
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    const uint4 kk = *(const uint4 *)(kr + 64 * c), vv = *(const uint4 *)(vr + 64 * c);
                    const u32 e[2][2] = { { kk.x, kk.y }, { kk.z, kk.w } }, f[2][2] = { { vv.x, vv.y }, { vv.z, vv.w } };
#pragma unroll
                    for (int z = 0; z < 2; ++z) { rp_multiply(s, a[2 * c + z], e[z], X()); rp_multiply(dp, b[2 * c + z], f[z], X()); }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) delta[i >> 1] += bits & 1u << i ? rp_exp2((s[i] * A.scale - lse[i >> 1]) * RP_LOG2E) * dp[i] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const auto over_row = [](float x) {
                    x += __shfl_xor_sync(0xffffffffu, x, 1);
                    return x + __shfl_xor_sync(0xffffffffu, x, 2);
                };
                const int row = r0 + g + 8 * u;
                const float sum = over_row(delta[u]);
                if (row < block.len && t == 0) A.stats[(i64)h * A.T + block.base + row] = make_float2(lse[u] * RP_LOG2E, sum);
                if constexpr (Narrow<X>::value) {
                    const float n = over_row(norm[u]);
                    if (row < block.len && n < INFINITY) top = fmaxf(top, n);          // (infinities and NaN, which no factor mends, do not count)
                }
            }
        }
        if constexpr (Narrow<X>::value) {
            const u32 bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
            if (lane == 0 && bits) atomicMax(A.tops + F.items[item].x, bits);
        }
    }
}
template <typename X, int D>
static int launch_few(const FewArgs &F, cudaLaunchConfig_t &how)
{
    how.dynamicSmemBytes = 2 * sizeof(FewRow<D>) * (112 + 8 * F.tiles);
    RP_CUDA(cudaFuncSetAttribute(k_attend_few<X, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(2 * sizeof(FewRow<D>) * (112 + 8 * 7))));
    RP_CUDA(cudaLaunchKernelEx(&how, k_attend_few<X, D>, F));
    return RP_OK;
}
// Power of two for the gradients of a sample's scores, from its largest row.
__device__ __forceinline__ float ds_scale(u32 top)
{
    const int e = (int)(__float_as_uint(sqrtf(__uint_as_float(top))) >> 23) - 127;         // 2^e <= norm < 2^(e + 1)
    return top ? __uint_as_float((u32)(127 + 3 - e) << 23) : 1.0f;
}

// One row of an accumulator in tensor memory, D columns, goes out.
template <typename X, int D>
__device__ __forceinline__ void store_row(u32 at, X *out, int d, bool there, float f)
{
#pragma unroll
    for (int c = 0; c < D; c += 32) {
        u32 o[32];
        tmem_load32(at + c, o);
        tmem_loaded();
        float v[32];
#pragma unroll
        for (int x = 0; x < 32; ++x) v[x] = __uint_as_float(o[x]) * f;
#pragma unroll
        for (int x = 0; x < 32; x += 8)
            if (there && c + x < d) rp_store8(out + c + x, rp_close8<X>(v + x));
        __syncwarp();
    }
}

// The same for 32 rows of a warp, through `rows` in shared memory (2 D bytes a row): pieces of 16 bytes side by side go out together.  (Each lane its own row: 32 lines
// an instruction.)
template <typename X, int D>
__device__ __forceinline__ void store_rows(u32 at, X *out, i64 step, int d, int left, float f, unsigned char *rows, int lane)
{
    constexpr int PIECES = D / 8, EACH = 32 / PIECES;
    const auto place = [](int row, int piece) { return row * (2 * D) + ((piece ^ (PIECES == 8 ? row & 7 : row >> 1 & 3)) << 4); };
    u32 o[D];
#pragma unroll
    for (int c = 0; c < D; c += 32) tmem_load32(at + c, o + c);
    tmem_loaded();
#pragma unroll
    for (int x = 0; x < PIECES; ++x) {
        float v[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) v[y] = __uint_as_float(o[8 * x + y]) * f;
        *(Pack8<X> *)(rows + place(lane, x)) = rp_close8<X>(v);
    }
    __syncwarp();
#pragma unroll
    for (int x = 0; x < PIECES; ++x) {
        const int row = x * EACH + lane / PIECES, piece = lane % PIECES;
        const Pack8<X> w = *(const Pack8<X> *)(rows + place(row, piece));
        if (row < left && 8 * piece < d) rp_store8(out + row * step + 8 * piece, w);
    }
    __syncwarp();
}

// The same in 32 bits.
template <int D>
__device__ __forceinline__ void store_part(u32 at, float *out, int d, bool there, float f)
{
#pragma unroll
    for (int c = 0; c < D; c += 32) {
        u32 o[32];
        tmem_load32(at + c, o);
        tmem_loaded();
#pragma unroll
        for (int x = 0; x < 32; x += 4)
            if (there && c + x < d)
                *(float4 *)(out + c + x) = make_float4(__uint_as_float(o[x]) * f, __uint_as_float(o[x + 1]) * f, __uint_as_float(o[x + 2]) * f, __uint_as_float(o[x + 3]) * f);
        __syncwarp();
    }
}

// Where a chunk of a first block's queries leaves the sums for the first tokens.  Chunks of a sample start `chunk` tokens apart and a sample with several is longer than
// that, so no two of those that start in one stretch of as many tokens are both the first of their sample, and no two both are not.
__device__ __forceinline__ i64 part_place(i64 base, int chunk, int tokens) { return 2 * ((int)base / tokens + chunk) + (chunk > 0); }           // (rows: less than 2^30)

// ---------------------------------------------------------------------------------------
// keys: dk and dv
// ---------------------------------------------------------------------------------------
// Tiles of 128 queries: scores, do v^T and the two sums fill the tensor memory (2 * 128 + 2 * head_dim columns).  Both groups of four warps work on a tile, 64 columns
// each.  The products come in the order dv(j), s(j + 1), dk(j), do v^T(j + 1): while the weights of a tile are worked out, the tensor cores add up dk of the one
// before and multiply do v^T of this one; while the gradients of its scores are, dv of this and scores of the next.  Weights and gradients lie as operands where the
// scores and the products of their group were.  (Tiles of 64 queries, two of them at a time, one for each group: 435 us
// for what took 249 then; 268 now, see the launch.)
template <int D> struct KeySmem {
    static constexpr int TILE = 128 * D * 2, STAGES = 2;
    alignas(1024) unsigned char k[TILE];
    alignas(1024) unsigned char v[TILE];
    alignas(1024) unsigned char q[STAGES][TILE];
    alignas(1024) unsigned char g[STAGES][TILE];
    alignas(16) float stats[2][2][2][64];    // [turn][group][lse / ln 2, delta][column]
    u64 kv_full, kv_empty, q_full[STAGES], q_empty[STAGES], s_full, dp_full, p_full, ds_full, st_full[2], acc_full, acc_empty, done;
    u32 tmem;
    Waits waits;
};

// A block of keys, and the tiles of queries that see it.
template <bool WINDOW> struct KeyItem {
    AttendTile t;
    int chunk, first, per;
    __device__ __forceinline__ KeyItem(const GradArgs &A, int item) : t(A.items, A.start, A.T, item, 128), chunk(0)
    {
        if (!WINDOW) {
            first = A.causal ? t.row0 >> 7 : 0;
            per = ((t.len + 127) >> 7) - first;
            return;
        }
        if (t.row0 < 0) { chunk = -t.row0 >> 7; t.row0 = 0; }
        const AttendRange r(t.len, t.row0 >> 7, chunk, A.window, A.sinks);
        first = r.first;
        per = r.per;
    }
};

template <typename X, int D, bool WINDOW>
__global__ void __launch_bounds__(ATTEND_THREADS, 1)
k_attend_keys(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
              const __grid_constant__ CUtensorMap map_g, const GradArgs A)
{
    typedef KeySmem<D> Smem;
    constexpr int STAGES = Smem::STAGES, PANELS = D / 64, PANEL = 128 * 128;
    extern __shared__ __align__(1024) unsigned char raw[];
    Smem &sm = *(Smem *)(raw + ((1024 - (rp_smem(raw) & 1023)) & 1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        bar_init(rp_smem(&sm.kv_full), 1); bar_init(rp_smem(&sm.kv_empty), 1);
        for (int s = 0; s < STAGES; ++s) { bar_init(rp_smem(&sm.q_full[s]), 1); bar_init(rp_smem(&sm.q_empty[s]), 1); }
        bar_init(rp_smem(&sm.s_full), 1); bar_init(rp_smem(&sm.dp_full), 1); bar_init(rp_smem(&sm.p_full), 8); bar_init(rp_smem(&sm.ds_full), 8);
        for (int i = 0; i < 2; ++i) bar_init(rp_smem(&sm.st_full[i]), 4);
        bar_init(rp_smem(&sm.acc_full), 1); bar_init(rp_smem(&sm.acc_empty), 8); bar_init(rp_smem(&sm.done), 1);
        sm.waits.start(A.wait_ns);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == ATTEND_COPY_WARP) tmem_alloc(rp_smem(&sm.tmem), 512);
    tmem_before();
    __syncthreads();
    tmem_after();
    const u32 tm = rp_uniform(sm.tmem);
    rp_wait_for_launch_before();             // the list of blocks and the statistics: nothing of them before this line
    rp_let_next_launch_start();              // the queries' kernel, which needs these too, takes the SMs that run out of work here
    const int total = rp_uniform(A.head->count * A.Hk);
    Waits *const waits = &sm.waits;

    if (warp >= 8) {
        rp_few_registers();
        if (warp == ATTEND_COPY_WARP && lane == 0) {
            tma_prefetch(&map_q); tma_prefetch(&map_k); tma_prefetch(&map_v); tma_prefetch(&map_g);
            u32 blocks = 0, fill = 0;                   // copies of keys and values and into the ring so far
            bool ok = true;
            for (int n = 0; ok; ++n) {
                const int at = rp_attend_item(n, total);
                if (at < 0) break;
                const KeyItem<WINDOW> item(A, at / A.Hk);
                const AttendTile &t = item.t;
                const int hk = at % A.Hk, first = item.first, per = item.per;
                if (!(ok = bar_place(n, rp_smem(&sm.kv_empty), (n - 1) & 1, waits))) break;
                ++blocks;
                bar_expect(rp_smem(&sm.kv_full), 2 * Smem::TILE);
                for (int p = 0; p < PANELS; ++p) {
                    tma_load3(rp_smem(sm.k) + p * PANEL, &map_k, p * 64, hk, (int)t.base + t.row0, rp_smem(&sm.kv_full));
                    tma_load3(rp_smem(sm.v) + p * PANEL, &map_v, p * 64, hk, (int)t.base + t.row0, rp_smem(&sm.kv_full));
                }
                for (int h = hk * A.share; ok && h < (hk + 1) * A.share; ++h)
                    for (int j = 0; j < per; ++j, ++fill) {
                        const u32 s = fill % STAGES, turn = fill / STAGES;
                        if (!(ok = bar_place(turn, rp_smem(&sm.q_empty[s]), (turn - 1) & 1, waits))) break;
                        bar_expect(rp_smem(&sm.q_full[s]), 2 * Smem::TILE);
                        waits->copied = fill + 1;
                        for (int p = 0; p < PANELS; ++p) {
                            tma_load3(rp_smem(sm.q[s]) + p * PANEL, &map_q, p * 64, h, (int)t.base + (first + j) * 128, rp_smem(&sm.q_full[s]));
                            tma_load3(rp_smem(sm.g[s]) + p * PANEL, &map_g, p * 64, h, (int)t.base + (first + j) * 128, rp_smem(&sm.q_full[s]));
                        }
                    }
            }
            // nobody may leave while copies are under way (whoever should have waited for them may have given up)
            for (u32 f = fill > (u32)STAGES ? fill - STAGES : 0; f < fill; ++f) rp_drain(rp_smem(&sm.q_full[f % STAGES]), (f / STAGES) & 1);
            if (blocks) rp_drain(rp_smem(&sm.kv_full), (blocks - 1) & 1);
        }
        if (warp == ATTEND_MMA_WARP) {
            const u32 shape_s = mma_shape<X>(128, false), shape_o = mma_shape<X>(D, true);
            u32 base = 0;                               // tiles of the items before
            for (int n = 0;; ++n) {
                const int at = rp_attend_item(n, total);
                if (at < 0 || rp_uniform(waits->gave_up)) break;
                const KeyItem<WINDOW> item(A, at / A.Hk);
                const int len = rp_uniform(item.t.len), first = (int)rp_uniform(item.first), per = (int)rp_uniform(item.per), nt = per * A.share;
                int tile = first;                       // of queries: the next to arrive
                // 128 keys against a tile's queries, or their values against the gradients
                auto against = [&](u32 to, const unsigned char *keys, const unsigned char *queries, u32 bar) {
                    const u32 a = mma_operand(rp_smem(keys), true, 0), b = mma_operand(rp_smem(queries), true, 0);
                    if (rp_elect()) {
#pragma unroll
                        for (int x = 0; x < D / 16; ++x) {
                            const u32 off = ((x / 4) * PANEL + (x % 4) * 32) >> 4;
                            mma_ss(to, a + off, b + off, shape_s, x > 0);
                        }
                        mma_commit(bar);
                    }
                    __syncwarp();
                };
                auto arrived = [&](u32 f) {     // a tile's queries and gradients
                    const u32 s = f % STAGES;
                    bar_hold(rp_smem(&sm.q_full[s]), (f / STAGES) & 1, waits);
                    // queries behind the sample's end are another sample's: their weights are 0, and 0 times NaN would not be
                    const int left = len - tile * 128;
                    if (left < 128) { rp_clear_rows<D>(sm.q[s], left, 128, lane); rp_clear_rows<D>(sm.g[s], left, 128, lane); }
                    tile = tile + 1 == first + per ? first : tile + 1;
                };
                // a tile's weights (or gradients of its scores) times its gradients (or queries)
                auto add = [&](u32 to, u32 weights, const unsigned char *rows, bool more) {
                    const u32 b = mma_operand(rp_smem(rows), false, PANEL);
                    if (rp_elect()) {
#pragma unroll
                        for (int x = 0; x < 8; ++x) mma_ts(to, weights + (x / 4) * 64 + (x % 4) * 8, b + x * (2048 >> 4), shape_o, more || x > 0);
                    }
                    __syncwarp();
                };
                bar_hold(rp_smem(&sm.kv_full), n & 1, waits);
                arrived(base);
                against(tm, sm.k, sm.q[base % STAGES], rp_smem(&sm.s_full));
                against(tm + 128, sm.v, sm.g[base % STAGES], rp_smem(&sm.dp_full));
                if (nt == 1) mma_commit_warp(rp_smem(&sm.kv_empty));
                if (n) bar_hold(rp_smem(&sm.acc_empty), (n - 1) & 1, waits);
                for (int j = 0; j < nt; ++j) {
                    const u32 f = base + j, s = f % STAGES, s1 = (f + 1) % STAGES;
                    if (j + 1 < nt) arrived(f + 1);         // (mostly before the weights have)
                    bar_hold(rp_smem(&sm.p_full), f & 1, waits);
                    tmem_after();
                    add(tm + 256, tm, sm.g[s], j > 0);
                    if (j + 1 < nt) against(tm, sm.k, sm.q[s1], rp_smem(&sm.s_full));
                    bar_hold(rp_smem(&sm.ds_full), f & 1, waits);
                    tmem_after();
                    add(tm + 256 + D, tm + 128, sm.q[s], j > 0);
                    mma_commit_warp(rp_smem(&sm.q_empty[s]));
                    if (j + 1 < nt) {
                        against(tm + 128, sm.v, sm.g[s1], rp_smem(&sm.dp_full));
                        if (j + 2 == nt) mma_commit_warp(rp_smem(&sm.kv_empty));
                    } else
                        mma_commit_warp(rp_smem(&sm.acc_full));
                }
                base += nt;
            }
            // nobody may leave while products are under way
            mma_commit_warp(rp_smem(&sm.done));
            if (lane == 0) rp_drain(rp_smem(&sm.done), 0);
        }
    } else {
        rp_many_registers();
        const int b = warp >> 2, row = threadIdx.x & 127;
        const u32 lanes = (u32)(warp & 3) << 21, ts = tm + lanes + b * 64, td = tm + lanes + 128 + b * 64;
        const f2 sl2 = rp_f2(A.scale * RP_LOG2E, A.scale * RP_LOG2E);
        u32 f = 0;                                      // tiles so far
        for (int n = 0;; ++n) {
            const int at = rp_attend_item(n, total);
            if (at < 0) break;
            const KeyItem<WINDOW> item(A, at / A.Hk);
            const AttendTile &t = item.t;
            const int hk = at % A.Hk, first = item.first, per = item.per, nt = per * A.share, r = t.row0 + row;
            bool ok = true;
            float c1 = 1.0f;                            // float16: the factors of ds (without the weights') and of the outputs
            if constexpr (Narrow<X>::value) c1 = ds_scale(A.tops[A.items[at / A.Hk].x]);
            const f2 c2 = rp_f2(c1 * (1.0f / 32768.0f), c1 * (1.0f / 32768.0f));
            auto stats = [&](int j) {                   // of one column of a tile
                const int q = (first + j % per) * 128 + b * 64 + row;
                return row < 64 && q < t.len ? A.stats[(i64)(hk * A.share + j / per) * A.T + t.base + q] : make_float2(0.0f, 0.0f);
            };
            float2 next = stats(0);
            for (int j = 0; j < nt; ++j, ++f) {
                const int q0 = (first + j % per) * 128 + b * 64;
                // (two places in turn: who has come to a tile's barrier has read the tile before)
                float (*st)[64] = sm.stats[f & 1][b];
                if (row < 64) {
                    st[0][row] = Narrow<X>::value ? 15.0f - next.x : -next.x;
                    st[1][row] = Narrow<X>::value ? -next.y * (c1 * (1.0f / 32768.0f)) : -next.y;
                }
                if (j + 1 < nt) next = stats(j + 1);
                bar_arrive_warp(rp_smem(&sm.st_full[b]), lane);
                if (!(ok = bar_wait_warp(rp_smem(&sm.st_full[b]), f & 1, waits))) break;
                if (!(ok = bar_wait_warp(rp_smem(&sm.s_full), f & 1, waits))) break;
                tmem_after();
                u32 s[64];
                float p[64];
                tmem_load32(ts, s);
                tmem_load32(ts + 32, s + 32);
                tmem_loaded();
#pragma unroll
                for (int c = 0; c < 64; c += 4) {
                    const ulonglong2 l = *(const ulonglong2 *)&st[0][c];         // (of the other sign)
                    rp_parts(rp_exp2(rp_fma(rp_f2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), sl2, f2{ l.x })), p[c], p[c + 1]);
                    rp_parts(rp_exp2(rp_fma(rp_f2(__uint_as_float(s[c + 2]), __uint_as_float(s[c + 3])), sl2, f2{ l.y })), p[c + 2], p[c + 3]);
                }
                const bool behind = q0 + 64 > t.len || (WINDOW && q0 + 63 >= t.row0 + A.window), before = A.causal && q0 < t.row0 + 128;
                if (WINDOW && before != behind) {
                    // (one comparison a column, where one will do)
                    const int lo = r - q0, hi = (r >= A.sinks ? min(t.len, r + A.window) : t.len) - q0;
                    if (before) {
#pragma unroll
                        for (int c = 0; c < 64; ++c) p[c] = c >= lo ? p[c] : 0.0f;
                    } else {
#pragma unroll
                        for (int c = 0; c < 64; ++c) p[c] = c < hi ? p[c] : 0.0f;
                    }
                } else if (before || behind) {
                    const int lo = A.causal ? r - q0 : 0, hi = (WINDOW && r >= A.sinks ? min(t.len, r + A.window) : t.len) - q0;
#pragma unroll
                    for (int c = 0; c < 64; ++c) p[c] = c >= lo && c < hi ? p[c] : 0.0f;
                }
#pragma unroll
                for (int c = 0; c < 32; ++c) s[c] = rp_pair(p[2 * c], p[2 * c + 1], X());
                tmem_store32(ts, s);
                tmem_stored();
                tmem_before();
                bar_arrive_warp(rp_smem(&sm.p_full), lane);
                if (!(ok = bar_wait_warp(rp_smem(&sm.dp_full), f & 1, waits))) break;
                tmem_after();
                tmem_load32(td, s);
                tmem_load32(td + 32, s + 32);
                tmem_loaded();
                auto less = [&](f2 dp, f2 delta) { return Narrow<X>::value ? rp_fma(dp, c2, delta) : rp_add(dp, delta); };
#pragma unroll
                for (int c = 0; c < 64; c += 4) {
                    const ulonglong2 e = *(const ulonglong2 *)&st[1][c];         // (of the other sign)
                    float a, z;
                    rp_parts(rp_mul(rp_f2(p[c], p[c + 1]), less(rp_f2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), f2{ e.x })), a, z);
                    s[c / 2] = rp_pair(a, z, X());
                    rp_parts(rp_mul(rp_f2(p[c + 2], p[c + 3]), less(rp_f2(__uint_as_float(s[c + 2]), __uint_as_float(s[c + 3])), f2{ e.y })), a, z);
                    s[c / 2 + 1] = rp_pair(a, z, X());
                }
                tmem_store32(td, s);
                tmem_stored();
                tmem_before();
                bar_arrive_warp(rp_smem(&sm.ds_full), lane);
            }
            if (ok) ok = bar_wait_warp(rp_smem(&sm.acc_full), n & 1, waits) && !waits->gave_up;
            tmem_after();
            // the first group hands over dv, the second dk
            X *out = b ? (X *)A.x[1] + (t.base + r) * A.token[1] + hk * A.hd[1] : (X *)A.x[0] + (t.base + r) * A.token[0] + hk * A.hd[0];
            const float f0 = Narrow<X>::value ? 1.0f / 32768.0f : 1.0f, f1 = Narrow<X>::value ? A.scale / c1 : A.scale;      // (c1: a power of two)
            bool mine = r < t.len;
            if (WINDOW && A.sinks > 0 && t.row0 == 0 && t.len > rp_attend_chunk(A.window) * 128) {
                // one of several chunks: the first tokens' sums meet those of the others; the rest of the keys are seen in the first chunk alone
                const bool ahead = mine && r < A.sinks;
                const i64 place = part_place(t.base, item.chunk, rp_attend_chunk(A.window) * 128);
                if (__any_sync(0xffffffffu, ahead))
                    store_part<D>(tm + lanes + 256 + b * D, A.parts + (((place * A.Hk + hk) * 2 + b) * A.sinks + r) * A.d, A.d, ahead, !ok ? NAN : b ? f1 : f0);
                mine = mine && !ahead && item.chunk == 0;
            }
            store_row<X, D>(tm + lanes + 256 + b * D, out, A.d, mine, !ok ? NAN : b ? f1 : f0);
            tmem_before();
            bar_arrive_warp(rp_smem(&sm.acc_empty), lane);
        }
    }
    __syncwarp();
    __syncthreads();
    if (threadIdx.x == 0 && sm.waits.gave_up) *A.status = RP_ERR_TIMEOUT;
    if (warp == ATTEND_COPY_WARP) tmem_free(tm, 512);
}

// ---------------------------------------------------------------------------------------
// queries: dq
// ---------------------------------------------------------------------------------------
// Tiles of 128 keys, 64 columns to each of the two groups of four warps.  q and do, which all tiles of a block share, lie in tensor memory as the operands of their
// products: from shared memory a product of 128 x 128 x 16 reads all of the 128 bytes that a cycle of it has, with the copies coming in beside (220 us for what
// took 166 then; 144 now).  They come through the ring that brings keys and values, ahead of these: each lane reads its row there and puts it into tensor memory.  Scores are multiplied while the weights of the tile before are worked out (as soon as those have been read), dq of a
// tile and do v^T of the next while the weights of the next are.  Columns: scores 128, do v^T 128 (and in its place ds as operand), dq, q and do 64 each.
template <int D> struct QuerySmem {
    static constexpr int TILE = 128 * D * 2, STAGES = 3;
    alignas(1024) unsigned char k[STAGES][TILE];
    alignas(1024) unsigned char v[STAGES][TILE];
    u64 q_full, kv_full[STAGES], kv_empty[STAGES], s_full, s_empty, dp_full, ds_full, acc_full, item_full[2], item_empty[2], done;
    u32 tmem;
    alignas(16) volatile int item[2][4];     // the item, its sample's first row and length, its own first row
    alignas(16) unsigned char rows[8][64 * D / 2];      // of each warp, what it hands over
    int taken, handled[8];                   // when a wait has run out: blocks that the CTA took, blocks that each warp of the softmax handed over
    Waits waits;
};

template <typename X, int D, bool WINDOW>
__global__ void __launch_bounds__(ATTEND_THREADS, 1)
k_attend_queries(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const __grid_constant__ CUtensorMap map_g, const GradArgs A)
{
    typedef QuerySmem<D> Smem;
    constexpr int STAGES = Smem::STAGES, PANELS = D / 64, PANEL = 128 * 128;
    extern __shared__ __align__(1024) unsigned char raw[];
    Smem &sm = *(Smem *)(raw + ((1024 - (rp_smem(raw) & 1023)) & 1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { bar_init(rp_smem(&sm.kv_full[s]), 1); bar_init(rp_smem(&sm.kv_empty[s]), 1); }
        bar_init(rp_smem(&sm.q_full), 8); bar_init(rp_smem(&sm.s_full), 1); bar_init(rp_smem(&sm.s_empty), 8); bar_init(rp_smem(&sm.dp_full), 1);
        bar_init(rp_smem(&sm.ds_full), 8); bar_init(rp_smem(&sm.acc_full), 1); bar_init(rp_smem(&sm.done), 1);
        for (int i = 0; i < 2; ++i) { bar_init(rp_smem(&sm.item_full[i]), 1); bar_init(rp_smem(&sm.item_empty[i]), 9); }
        sm.waits.start(A.wait_ns);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == ATTEND_COPY_WARP) tmem_alloc(rp_smem(&sm.tmem), 512);
    tmem_before();
    __syncthreads();
    tmem_after();
    const u32 tm = rp_uniform(sm.tmem);
    const int total = rp_uniform(A.head->count * A.Hq);
    Waits *const waits = &sm.waits;

    if (warp >= 8) {
        rp_few_registers();
        if (warp == ATTEND_COPY_WARP && lane == 0) {
            tma_prefetch(&map_q); tma_prefetch(&map_k); tma_prefetch(&map_v); tma_prefetch(&map_g);
            u32 fill = 0;
            int taken = 0;
            bool ok = true;
            for (int n = 0; ok; ++n) {
                // the next of the list for whoever is free: CTAs start as the keys' kernel leaves them an SM
                if (!(ok = bar_place(n > 1, rp_smem(&sm.item_empty[n & 1]), ((n >> 1) - 1) & 1, waits))) break;
                int at = atomicAdd(&A.head->ticket, 1);
                if (at >= total) at = -1;
                const AttendTile t = at < 0 ? AttendTile() : AttendTile(A.items, A.start, A.T, at / A.Hq, 128);
                sm.item[n & 1][0] = at; sm.item[n & 1][1] = (int)t.base; sm.item[n & 1][2] = t.len; sm.item[n & 1][3] = t.row0;
                bar_arrive(rp_smem(&sm.item_full[n & 1]));
                if (at < 0) break;
                taken = n + 1;
                const AttendSteps w(WINDOW ? t.row0 : 0, WINDOW ? A.window : 1, WINDOW ? A.sinks : 0);
                const int hk = at % A.Hq / A.share, seen = rp_attend_tiles(t, 0, A.causal), nk = WINDOW ? w.steps(seen) : seen;
                for (int j = -1; j < nk; ++j, ++fill) {             // (-1: the block's own q and do)
                    const int from = j < 0 ? (int)t.base + t.row0 : (int)t.base + (WINDOW ? w.tile(j) : j) * 128, head = j < 0 ? at % A.Hq : hk;
                    const u32 s = fill % STAGES, turn = fill / STAGES;
                    if (!(ok = bar_place(turn, rp_smem(&sm.kv_empty[s]), (turn - 1) & 1, waits))) break;
                    bar_expect(rp_smem(&sm.kv_full[s]), 2 * Smem::TILE);
                    waits->copied = fill + 1;
                    for (int p = 0; p < PANELS; ++p) {
                        tma_load3(rp_smem(sm.k[s]) + p * PANEL, j < 0 ? &map_q : &map_k, p * 64, head, from, rp_smem(&sm.kv_full[s]));
                        tma_load3(rp_smem(sm.v[s]) + p * PANEL, j < 0 ? &map_g : &map_v, p * 64, head, from, rp_smem(&sm.kv_full[s]));
                    }
                }
            }
            sm.taken = taken;
            // nobody may leave while copies are under way (whoever should have waited for them may have given up)
            for (u32 f = fill > (u32)STAGES ? fill - STAGES : 0; f < fill; ++f) rp_drain(rp_smem(&sm.kv_full[f % STAGES]), (f / STAGES) & 1);
        }
        if (warp == ATTEND_MMA_WARP) {
            const u32 shape_s = mma_shape<X>(128, false), shape_o = mma_shape<X>(D, true);
            const int groups = WINDOW ? (int)rp_uniform((A.sinks + 31) >> 5) : 0;         // first tokens by 32: as narrow is the step that they are from afar
            const u32 shape_first = mma_shape<X>(32 * groups, false);
            u32 base = 0, stage = 0;                    // tiles of the items before, and stages
            for (int n = 0;; ++n, ++stage) {
                bar_hold(rp_smem(&sm.item_full[n & 1]), (n >> 1) & 1, waits);
                const int at = rp_uniform(sm.item[n & 1][0]);
                if (at < 0 || rp_uniform(waits->gave_up)) break;
                const AttendTile t(sm.item[n & 1]);
                bar_arrive_warp(rp_smem(&sm.item_empty[n & 1]), lane);
                const AttendSteps w(WINDOW ? (int)rp_uniform(t.row0) : 0, WINDOW ? A.window : 1, WINDOW ? A.sinks : 0);
                const int len = rp_uniform(t.len), seen = rp_uniform(rp_attend_tiles(t, 0, A.causal)), nk = WINDOW ? w.steps(seen) : seen;
                // 128 queries (or gradients) against a tile's keys (or values)
                auto against = [&](u32 to, u32 rows, const unsigned char *tile, u32 shape_s, u32 bar) {
                    const u32 b = mma_operand(rp_smem(tile), true, 0);
                    if (rp_elect()) {
#pragma unroll
                        for (int x = 0; x < D / 16; ++x) mma_ts(to, rows + x * 8, b + (((x / 4) * PANEL + (x % 4) * 32) >> 4), shape_s, x > 0);
                        mma_commit(bar);
                    }
                    __syncwarp();
                };
                const u32 own = stage % STAGES;
                auto arrived = [&](int j) {             // a tile's keys and values
                    const u32 f = stage + 1 + j;
                    bar_hold(rp_smem(&sm.kv_full[f % STAGES]), (f / STAGES) & 1, waits);
                    // keys behind the sample's end are another sample's: the gradients of their scores are 0, and 0 times NaN would not be
                    const int behind = len - (WINDOW ? w.tile(j) : j) * 128;
                    if (behind < 128) rp_clear_rows<D>(sm.k[f % STAGES], behind, 128, lane);
                    if (WINDOW && j < w.ahead) rp_clear_rows<D>(sm.k[f % STAGES], A.sinks, 32 * groups, lane);           // (neither are those behind the first tokens seen)
                };
                arrived(0);
                // (who has handed over q and do has taken dq of the block before, and has read them in their stage)
                bar_hold(rp_smem(&sm.q_full), n & 1, waits);
                tmem_after();
                bar_arrive_warp(rp_smem(&sm.kv_empty[own]), lane);
                against(tm, tm + 384, sm.k[(stage + 1) % STAGES], w.ahead ? shape_first : shape_s, rp_smem(&sm.s_full));
                against(tm + 128, tm + 448, sm.v[(stage + 1) % STAGES], w.ahead ? shape_first : shape_s, rp_smem(&sm.dp_full));
                for (int j = 0; j < nk; ++j) {
                    const u32 f = base + j, s = (stage + 1 + j) % STAGES, s1 = (stage + 2 + j) % STAGES;
                    if (j + 1 < nk) {
                        arrived(j + 1);
                        bar_hold(rp_smem(&sm.s_empty), f & 1, waits);
                        tmem_after();
                        against(tm, tm + 384, sm.k[s1], shape_s, rp_smem(&sm.s_full));
                    }
                    bar_hold(rp_smem(&sm.ds_full), f & 1, waits);
                    tmem_after();
                    const u32 k = mma_operand(rp_smem(sm.k[s]), false, PANEL);
                    if (rp_elect()) {
                        if (WINDOW && j < w.ahead)
                            for (int x = 0; x < 2 * groups; ++x) mma_ts(tm + 256, tm + 128 + (x / 4) * 64 + (x % 4) * 8, k + x * (2048 >> 4), shape_o, x > 0);
                        else {
#pragma unroll
                            for (int x = 0; x < 8; ++x) mma_ts(tm + 256, tm + 128 + (x / 4) * 64 + (x % 4) * 8, k + x * (2048 >> 4), shape_o, j > 0 || x > 0);
                        }
                    }
                    __syncwarp();
                    mma_commit_warp(rp_smem(&sm.kv_empty[s]));
                    if (j + 1 < nk) against(tm + 128, tm + 448, sm.v[s1], shape_s, rp_smem(&sm.dp_full));
                    else mma_commit_warp(rp_smem(&sm.acc_full));
                }
                base += nk;
                stage += nk;
            }
            // nobody may leave while products are under way
            mma_commit_warp(rp_smem(&sm.done));
            if (lane == 0) rp_drain(rp_smem(&sm.done), 0);
        }
    } else {
        rp_many_registers();
        const int b = warp >> 2, row = threadIdx.x & 127;
        const u32 lanes = (u32)(warp & 3) << 21, ts = tm + lanes + b * 64, td = tm + lanes + 128 + b * 64;
        const f2 sl2 = rp_f2(A.scale * RP_LOG2E, A.scale * RP_LOG2E);
        u32 f = 0;                                      // tiles so far
        u32 w[64];                                      // a row of q (first group) or of do (second): two elements a word
        int at = 0;                                     // the item
        AttendTile block;
        auto fetch = [&](int n) {
            at = -1;
            if (bar_wait_warp(rp_smem(&sm.item_full[n & 1]), (n >> 1) & 1, waits)) at = sm.item[n & 1][0];
            if (at < 0) return;
            const AttendTile t = block = AttendTile(sm.item[n & 1]);
            bar_arrive_warp(rp_smem(&sm.item_empty[n & 1]), lane);
            // its own row, from the stage ahead of its block's keys (tiles and blocks so far)
            const u32 g = f + n, s = g % STAGES;
            const bool come = bar_wait_warp(rp_smem(&sm.kv_full[s]), (g / STAGES) & 1, waits) && t.row0 + row < t.len;
            const unsigned char *p = (b ? sm.v[s] : sm.k[s]) + row * 128;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (come) v = *(const uint4 *)(p + (c >> 3) * PANEL + (((c & 7) ^ (row & 7)) << 4));
                w[4 * c] = v.x; w[4 * c + 1] = v.y; w[4 * c + 2] = v.z; w[4 * c + 3] = v.w;
            }
        };
        fetch(0);
        int n = 0;
        for (; at >= 0; ++n) {
            const AttendTile t = block;
            const AttendSteps steps(WINDOW ? t.row0 : 0, WINDOW ? A.window : 1, WINDOW ? A.sinks : 0);
            const int h = at % A.Hq, seen = rp_attend_tiles(t, 0, A.causal), nk = WINDOW ? steps.steps(seen) : seen, r = t.row0 + row;
#pragma unroll
            for (int c = 0; c < D / 2; c += 32) tmem_store32(tm + lanes + 384 + b * 64 + c, w + c);
            tmem_stored();
            tmem_before();
            bar_arrive_warp(rp_smem(&sm.q_full), lane);
            const float2 st = r < t.len ? A.stats[(i64)h * A.T + t.base + r] : make_float2(0.0f, 0.0f);
            float c1 = 1.0f;                            // float16: the factor of ds
            if constexpr (Narrow<X>::value) c1 = ds_scale(A.tops[A.items[at / A.Hq].x]);
            const f2 lse2 = rp_f2(-st.x, -st.x), delta2 = rp_f2(-st.y * c1, -st.y * c1), c2 = rp_f2(c1, c1);
            bool ok = true;
            for (int j = 0; j < nk; ++j, ++f) {
                if (!(ok = bar_wait_warp(rp_smem(&sm.s_full), f & 1, waits))) break;
                tmem_after();
                if (WINDOW && j < steps.ahead && b * 64 >= A.sinks) {
                    // first tokens from afar, of which there are none in this group's columns
                    bar_arrive_warp(rp_smem(&sm.s_empty), lane);
                    if (!(ok = bar_wait_warp(rp_smem(&sm.dp_full), f & 1, waits))) break;
                    bar_arrive_warp(rp_smem(&sm.ds_full), lane);
                    continue;
                }
                u32 s[64];
                f2 p[32];
                tmem_load32(ts, s);
                tmem_load32(ts + 32, s + 32);
                tmem_loaded();
                tmem_before();
                bar_arrive_warp(rp_smem(&sm.s_empty), lane);
#pragma unroll
                for (int c = 0; c < 32; ++c) p[c] = rp_exp2(rp_fma(rp_f2(__uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1])), sl2, lse2));
                const int k0 = (WINDOW ? steps.tile(j) : j) * 128 + b * 64, lim = (A.causal ? min(t.len, r + 1) : t.len) - k0;
                if (!(ok = bar_wait_warp(rp_smem(&sm.dp_full), f & 1, waits))) break;
                tmem_after();
                tmem_load32(td, s);
                tmem_load32(td + 32, s + 32);
                tmem_loaded();
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                    const f2 dp = rp_f2(__uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1]));
                    p[c] = rp_mul(p[c], Narrow<X>::value ? rp_fma(dp, c2, delta2) : rp_add(dp, delta2));
                }
                const bool behind = k0 + 64 > t.len || (A.causal && k0 + 63 > t.row0), before = WINDOW && k0 <= t.row0 + 127 - A.window;
                if (behind && !before) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) {
                        float x, y;
                        rp_parts(p[c], x, y);
                        s[c] = rp_pair(2 * c < lim ? x : 0.0f, 2 * c + 1 < lim ? y : 0.0f, X());
                    }
                } else if (before) {
                    // (the end of the window's reach and the row's own place are never both in 64 columns but with short windows)
                    const int from = r - A.window + 1 - k0, ahead = A.sinks - k0;
                    if (!behind && ahead <= 0) {
#pragma unroll
                        for (int c = 0; c < 32; ++c) {
                            float x, y;
                            rp_parts(p[c], x, y);
                            s[c] = rp_pair(2 * c >= from ? x : 0.0f, 2 * c + 1 >= from ? y : 0.0f, X());
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < 32; ++c) {
                            float x, y;
                            rp_parts(p[c], x, y);
                            s[c] = rp_pair(2 * c < lim && (2 * c >= from || 2 * c < ahead) ? x : 0.0f, 2 * c + 1 < lim && (2 * c + 1 >= from || 2 * c + 1 < ahead) ? y : 0.0f, X());
                        }
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 32; ++c) {
                        float x, y;
                        rp_parts(p[c], x, y);
                        s[c] = rp_pair(x, y, X());
                    }
                }
                tmem_store32(td, s);
                tmem_stored();
                tmem_before();
                bar_arrive_warp(rp_smem(&sm.ds_full), lane);
            }
            fetch(n + 1);                               // while dq is finished and handed over
            if (ok) ok = bar_wait_warp(rp_smem(&sm.acc_full), n & 1, waits) && !waits->gave_up;
            tmem_after();
            // each group hands over one half of the columns
            X *out = (X *)A.x[0] + (t.base + t.row0 + (row & ~31)) * A.token[0] + h * A.hd[0] + b * (D / 2);
            store_rows<X, D / 2>(tm + lanes + 256 + b * (D / 2), out, A.token[0], A.d - b * (D / 2), t.len - t.row0 - (row & ~31),
                                 !ok ? NAN : Narrow<X>::value ? A.scale / c1 : A.scale, sm.rows[warp], lane);
            tmem_before();
        }
        if (lane == 0) sm.handled[warp] = n;
    }
    __syncwarp();
    __syncthreads();
    if (warp < 8 && sm.waits.gave_up) {
        // A wait ran out: blocks that were taken and not handed over become NaN, and so does what nobody has taken.
        const int b = warp >> 2, row = threadIdx.x & 127;
        auto mark = [&](int at, int r0, int rows, int c0, int columns) {
            const AttendTile t(A.items, A.start, A.T, at / A.Hq, 128);
            for (int x = lane; x < rows * columns; x += 32) {
                const int r = t.row0 + r0 + x / columns, c = c0 + x % columns;
                if (r < t.len && c < A.d) ((X *)A.x[0])[(t.base + r) * A.token[0] + at % A.Hq * A.hd[0] + c] = rp_round<X>(NAN);
            }
        };
        for (int n = sm.handled[warp]; n < sm.taken; ++n) mark(sm.item[n & 1][0], row & ~31, 32, b * (D / 2), D / 2);
        for (;;) {
            int at = lane == 0 ? atomicAdd(&A.head->ticket, 1) : 0;
            at = __shfl_sync(0xffffffffu, at, 0);
            if (at >= total || at < 0) break;
            mark(at, 0, 128, 0, D);
        }
    }
    if (threadIdx.x == 0 && sm.waits.gave_up) *A.status = RP_ERR_TIMEOUT;
    rp_wait_for_launch_before();                     // this launch is not over before the keys' is
    if (warp == ATTEND_COPY_WARP) tmem_free(tm, 512);
}

// ---------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------
// Workspace: front and items of the keys' kernel, the same of the queries', statistics; for float16 norms of rows and the largest of each sample.
static i64 plan_bytes(i64 T, int N, i64 more) { return ((i64)sizeof(AttendHead) + 8 * (T / 128 + N + more) + 15) / 16 * 16; }

// With a window: room for the chunks of first blocks, and behind all else their sums.
static i64 more_items(i64 T, int window, int sinks) { return sinks ? T / (128 * rp_attend_chunk(window)) : 0; }
static i64 parts_at(const rp_attend_config *a, i64 T, int N, int window, int sinks)
{
    const i64 all = 2 * plan_bytes(T, N, more_items(T, window, sinks)) + 8 * T * a->q_heads + (a->type == RP_F16 ? 4 * (T * a->q_heads + N) : 0);
    return window ? (all + 15) / 16 * 16 : all;
}
static i64 grad_bytes(const rp_attend_config *a, i64 T, int N, int window, int sinks)
{
    const i64 more = more_items(T, window, sinks);
    return parts_at(a, T, N, window, sinks) + (more ? 2 * (more + 1) * a->kv_heads * 2 * sinks * a->head_dim * 4 : 0);
}
extern "C" int64_t rp_attend_grad_workspace(const rp_attend_config *a, int64_t n_tokens, int32_t n_samples)
{
    return rp_attend_check(a, n_tokens, n_samples) == RP_OK ? grad_bytes(a, n_tokens, n_samples, 0, 0) : 0;
}
extern "C" int64_t rp_attend_window_grad_workspace(const rp_attend_config *a, int32_t window, int32_t sinks, int64_t n_tokens, int32_t n_samples)
{
    return rp_attend_check_window(a, window, sinks, n_tokens, n_samples) == RP_OK ? grad_bytes(a, n_tokens, n_samples, rp_attend_window_of(window, n_tokens), sinks) : 0;
}

// Gradients of the first tokens that several chunks have parts of, in the order of the chunks.
template <typename X>
__global__ void __launch_bounds__(256) k_attend_sinks(const i64 *start, int N, i64 T, int window, int sinks, int Hk, int d, const float *parts, X *dv, X *dk, i64 v_token,
                                                      i64 v_head, i64 k_token, i64 k_head)
{
    const int tokens = rp_attend_chunk(window) * 128;
    for (i64 unit = blockIdx.x; unit < (i64)N * Hk * 2; unit += gridDim.x) {
        const int i = (int)(unit / (2 * Hk)), hk = (int)(unit % (2 * Hk)) >> 1, b = (int)(unit & 1);
        const i64 base = max(start[i], (i64)0);
        const i64 len = min(start[i + 1], T) - base;
        if (len <= tokens) continue;
        const int chunks = rp_attend_chunks((int)len, window);
        const float *const from = parts + ((part_place(base, 0, tokens) * Hk + hk) * 2 + b) * sinks * d;
        for (int x = threadIdx.x; x < sinks * d; x += 256) {
            float sum = 0.0f;
#pragma unroll 4
            for (int c = 0; c < chunks; ++c) sum += from[(i64)(2 * c + (c > 0)) * Hk * 2 * sinks * d + x];
            const int r = x / d, e = x % d;
            if (b) dk[(base + r) * k_token + hk * k_head + e] = rp_round<X>(sum);
            else dv[(base + r) * v_token + hk * v_head + e] = rp_round<X>(sum);
        }
    }
}

struct GradMaps { CUtensorMap q, k, v, g; };

template <typename X, int D, bool WINDOW>
static int launch(const GradMaps &M, GradArgs &keys, GradArgs &queries, i64 most_keys, i64 most, int sms, cudaStream_t stream)
{
    const size_t sk = sizeof(KeySmem<D>) + 1024, sq = sizeof(QuerySmem<D>) + 1024;
    RP_CUDA(cudaFuncSetAttribute(k_attend_keys<X, D, WINDOW>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sk));
    RP_CUDA(cudaFuncSetAttribute(k_attend_queries<X, D, WINDOW>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sq));
    cudaLaunchConfig_t how = {};                         // (both get their barriers, tensor memory and maps ready beside what runs before them)
    how.gridDim = dim3((unsigned)std::min((i64)sms, most_keys * keys.Hk));
    how.blockDim = dim3(ATTEND_THREADS);
    how.dynamicSmemBytes = sk;
    how.stream = stream;
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    how.attrs = &early; how.numAttrs = 1;
    RP_CUDA(cudaLaunchKernelEx(&how, k_attend_keys<X, D, WINDOW>, M.q, M.k, M.v, M.g, (const GradArgs)keys));
    RP_TRY(rp_op_launched());
    // (8192 tokens in three samples, 16 heads on 4, 128 wide: the keys' kernel, whose largest block of keys takes as long as 1.4 times its share of all work, 268 us, the
    // queries' 144; 346 us for the whole call, in which they overlap.  A block's query heads dealt out to several CTAs, whose sums meet behind them, make short lists of blocks faster - one
    // sample of 2048 tokens, 5 heads on 1: 193 -> 69 us - but a sample's gradients then depend on what else is in its row.)
    how.gridDim = dim3((unsigned)std::min((i64)sms, most * keys.Hq));
    how.dynamicSmemBytes = sq;
    RP_CUDA(cudaLaunchKernelEx(&how, k_attend_queries<X, D, WINDOW>, M.q, M.k, M.v, M.g, (const GradArgs)queries));
    return rp_op_launched();
}

static int attend_grad(const rp_attend_config *a, int window, int sinks, i64 n_tokens, const rp_view *q, const rp_view *k, const rp_view *v, const rp_view *out,
                       const rp_view *lse, const rp_view *out_grad, const int64_t *start, int n_samples, const rp_view *q_grad, const rp_view *k_grad,
                       const rp_view *v_grad, void *workspace, i64 workspace_bytes, void *cuda_stream)
{
    if (!start || !rp_aligned(start, 8) || !workspace || !rp_aligned(workspace, 16) || workspace_bytes < grad_bytes(a, n_tokens, n_samples, window, sinks)) return RP_ERR_ARG;
    if (!lse || !lse->x || !rp_aligned(lse->x, 4)) return RP_ERR_ARG;
    RpOpDevice dev;
    if (n_tokens == 0) {
        RP_TRY(rp_op_enter(dev, workspace));
        RP_CUDA(cudaMemsetAsync(workspace, 0, sizeof(AttendHead), (cudaStream_t)cuda_stream));
        return RP_OK;
    }
    const rp_view *const places[] = { q_grad, k_grad, v_grad, q, k, v, out, lse, out_grad };
    if (rp_attend_shared(places, 3, 6)) return RP_ERR_ARG;
    const rp_view *by_q[4] = { q, out, out_grad, q_grad }, *by_k[4] = { k, v, k_grad, v_grad };
    for (int i = 0; i < 4; ++i) {
        RP_TRY(rp_attend_view(by_q[i], n_tokens, a->q_heads, dev));
        RP_TRY(rp_attend_view(by_k[i], n_tokens, a->kv_heads, dev));
    }
    RP_TRY(rp_op_enter(dev, start, workspace, lse->x));
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    const i64 T = n_tokens, more = more_items(T, window, sinks), plan = plan_bytes(T, n_samples, more);
    AttendHead *head[2] = { (AttendHead *)workspace, (AttendHead *)((char *)workspace + plan) };
    float2 *stats = (float2 *)((char *)workspace + 2 * plan);
    const int d = a->head_dim, Hq = a->q_heads, Hk = a->kv_heads;
    GradMaps M;
    RP_TRY(rp_tensor_map(&M.q, a->type, q->x, T, Hq, d, q->token, q->head, 128));
    RP_TRY(rp_tensor_map(&M.k, a->type, k->x, T, Hk, d, k->token, k->head, 128));
    RP_TRY(rp_tensor_map(&M.v, a->type, v->x, T, Hk, d, v->token, v->head, 128));
    RP_TRY(rp_tensor_map(&M.g, a->type, out_grad->x, T, Hq, d, out_grad->token, out_grad->head, 128));
    AttendPlan P[2] = {};
    AttendClears C = {};
    C.x[C.n++] = { k_grad->x, k_grad->token, k_grad->head, Hk, d, 2 };
    C.x[C.n++] = { v_grad->x, v_grad->token, v_grad->head, Hk, d, 2 };
    C.x[C.n++] = { q_grad->x, q_grad->token, q_grad->head, Hq, d, 2 };
    GradArgs G[2];
    for (int w = 0; w < 2; ++w) {
        P[w].start = (const i64 *)start; P[w].T = T; P[w].N = n_samples; P[w].rows = 128; P[w].causal = a->causal; P[w].most = (int)(T / 128 + n_samples + (w ? 0 : more));
        P[w].window = window; P[w].sinks = sinks;
        P[w].by_key = w == 0; P[w].head = head[w]; P[w].items = (int2 *)(head[w] + 1);
        GradArgs &A = G[w];
        A = GradArgs();
        A.items = P[w].items; A.head = head[w]; A.start = (const i64 *)start; A.T = T; A.Hq = Hq; A.Hk = Hk; A.share = Hq / Hk; A.d = d; A.causal = a->causal;
        A.window = window; A.sinks = sinks; A.parts = (float *)((char *)workspace + parts_at(a, T, n_samples, window, sinks));
        A.scale = a->scale; A.stats = stats; A.status = &head[0]->status; A.wait_ns = (u64)g_attend_wait_ns;
    }
    G[0].x[0] = v_grad->x; G[0].token[0] = v_grad->token; G[0].hd[0] = v_grad->head;
    G[0].x[1] = k_grad->x; G[0].token[1] = k_grad->token; G[0].hd[1] = k_grad->head;
    G[1].x[0] = q_grad->x; G[1].token[0] = q_grad->token; G[1].hd[0] = q_grad->head;
    const int sms = rp_op_sms(dev.device);
    float *const norms = (float *)(stats + T * Hq);
    u32 *const tops = (u32 *)(norms + T * Hq);           // (float16)
    G[0].tops = G[1].tops = tops;
    // (where all tokens see few keys, nothing comes from the outputs; the window is cut to the row and 256, so a short one is as it was)
    const bool few = window && window + sinks <= FEW_KEYS;
    const StatsArgs S = { out->x, out_grad->x, (const float *)lse->x, out->token, out->head, out_grad->token, out_grad->head, lse->token, lse->head, few ? 0 : Hq, d, stats, norms,
                          tops };
    // (A CTA fills an SM's registers: one round of them.  Two rounds: 508 us for 503 with 16384 tokens, 51.6 for 43.6 with 3001.)
    const int ctas = 2 + (int)std::min((T * Hq + 63) / 64, std::max((i64)sms - 2, (i64)1));
    const bool half = a->type == RP_F16;
    if (half) k_attend_prepare<__half><<<ctas, 1024, 0, stream>>>(P[0], P[1], C, S);
    else k_attend_prepare<bf16><<<ctas, 1024, 0, stream>>>(P[0], P[1], C, S);
    RP_TRY(rp_op_launched());
    const unsigned blocks = (unsigned)((T + 255) / 256);
    if (window) {
        const int first = (int)std::min((i64)n_samples * Hq, (i64)sms * 8);
        const FirstArgs F = { (const i64 *)start, T, n_samples, Hq, Hq / Hk, d, window, sinks, a->scale, q->x, k->x, v->x, out_grad->x, q->token, q->head, k->token, k->head,
                              v->token, v->head, out_grad->token, out_grad->head, (const float *)lse->x, lse->token, lse->head, stats, norms, tops, first };
        cudaLaunchConfig_t how = {};                     // (while the statistics are worked out)
        how.gridDim = dim3(half ? first + blocks : first);
        how.blockDim = dim3(256);
        how.stream = stream;
        cudaLaunchAttribute early = {};
        early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        early.val.programmaticStreamSerializationAllowed = 1;
        how.attrs = &early; how.numAttrs = 1;
        if (few) {
            // a key head's query heads by one CTA, which reads the keys once, or by several where there are few blocks
            const i64 units = (i64)P[1].most * Hk, most = (i64)sms * 2;
            FewArgs E = { F, head[1], P[1].items, (int)std::min((i64)(Hq / Hk), (2 * most + units - 1) / units), (sinks + 7) / 8, (window + 6) / 8, 0 };
            E.tiles = E.ahead + E.before + 2;
            how.gridDim = dim3((unsigned)std::min(units * E.parts, most));
            if (half) RP_TRY((d <= 64 ? launch_few<__half, 64>(E, how) : launch_few<__half, 128>(E, how)));
            else RP_TRY((d <= 64 ? launch_few<bf16, 64>(E, how) : launch_few<bf16, 128>(E, how)));
        } else if (half) RP_CUDA(cudaLaunchKernelEx(&how, k_attend_first<__half>, F));
        else RP_CUDA(cudaLaunchKernelEx(&how, k_attend_first<bf16>, F));
        RP_TRY(rp_op_launched());
    } else if (half) {
        k_attend_tops<<<blocks, 256, 0, stream>>>((const i64 *)start, n_samples, T, Hq, norms, tops);
        RP_TRY(rp_op_launched());
    }
    const i64 mk = P[0].most, mq = P[1].most;
    if (!window) {
        if (half) return d <= 64 ? launch<__half, 64, false>(M, G[0], G[1], mk, mq, sms, stream) : launch<__half, 128, false>(M, G[0], G[1], mk, mq, sms, stream);
        return d <= 64 ? launch<bf16, 64, false>(M, G[0], G[1], mk, mq, sms, stream) : launch<bf16, 128, false>(M, G[0], G[1], mk, mq, sms, stream);
    }
    if (half) RP_TRY((d <= 64 ? launch<__half, 64, true>(M, G[0], G[1], mk, mq, sms, stream) : launch<__half, 128, true>(M, G[0], G[1], mk, mq, sms, stream)));
    else RP_TRY((d <= 64 ? launch<bf16, 64, true>(M, G[0], G[1], mk, mq, sms, stream) : launch<bf16, 128, true>(M, G[0], G[1], mk, mq, sms, stream)));
    if (!more) return RP_OK;
    const int grid = (int)std::min((i64)n_samples * Hk * 2, (i64)sms * 8);
    if (half)
        k_attend_sinks<<<grid, 256, 0, stream>>>((const i64 *)start, n_samples, T, window, sinks, Hk, d, G[0].parts, (__half *)v_grad->x, (__half *)k_grad->x, v_grad->token,
                                                 v_grad->head, k_grad->token, k_grad->head);
    else
        k_attend_sinks<<<grid, 256, 0, stream>>>((const i64 *)start, n_samples, T, window, sinks, Hk, d, G[0].parts, (bf16 *)v_grad->x, (bf16 *)k_grad->x, v_grad->token,
                                                 v_grad->head, k_grad->token, k_grad->head);
    return rp_op_launched();
}

extern "C" int rp_attend_grad(const rp_attend_config *a, int64_t n_tokens, const rp_view *q, const rp_view *k, const rp_view *v, const rp_view *out,
                              const rp_view *lse, const rp_view *out_grad, const int64_t *start, int32_t n_samples, const rp_view *q_grad,
                              const rp_view *k_grad, const rp_view *v_grad, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    RP_TRY(rp_attend_check(a, n_tokens, n_samples));
    return attend_grad(a, 0, 0, n_tokens, q, k, v, out, lse, out_grad, start, n_samples, q_grad, k_grad, v_grad, workspace, workspace_bytes, cuda_stream);
}

extern "C" int rp_attend_window_grad(const rp_attend_config *a, int32_t window, int32_t sinks, int64_t n_tokens, const rp_view *q, const rp_view *k, const rp_view *v,
                                     const rp_view *out, const rp_view *lse, const rp_view *out_grad, const int64_t *start, int32_t n_samples, const rp_view *q_grad,
                                     const rp_view *k_grad, const rp_view *v_grad, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    RP_TRY(rp_attend_check_window(a, window, sinks, n_tokens, n_samples));
    return attend_grad(a, rp_attend_window_of(window, n_tokens), sinks, n_tokens, q, k, v, out, lse, out_grad, start, n_samples, q_grad, k_grad, v_grad, workspace, workspace_bytes,
                       cuda_stream);
}
