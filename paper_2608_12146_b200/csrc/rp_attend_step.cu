// Attention of one new token of each sequence against the keys and values of those before it (decoding).
//
//   s = scale q k^T over the keys that the token sees, o = softmax(s) v, lse = log sum exp(s)
//
// Bound by HBM: each visible key and value is read once, 4 * head_dim bytes for 4 * share * head_dim operations (share: query heads to a key head).  The products go
// through the warps' matrix instruction, 16 query heads by 16 keys at a time, of which `share` rows are something: with a few rows to a tile there is nothing that
// fuller instructions could add.
// The keys that a sequence's token sees are cut into chunks of 128, or of a 128th of them where that is more; a chunk and a key head are a unit of one warp, which takes
// them 16 keys at a time through a ring of its own in shared memory.  Warps stay resident and take units in turn, and the ring runs on into the next unit; no warp waits
// for another.  The cut goes by the sequence alone, so that its bits do not depend on the others of the batch.  A second kernel adds up the chunks, in their order.
#include <algorithm>

#include "rp_attend.cuh"

#define STEP_WARPS 4
#define STEP_THREADS (32 * STEP_WARPS)
#define STEP_CHUNK 128                   // keys of a chunk at least
#define STEP_CHUNKS 128                  // chunks of a sequence at most
#define STEP_ROWS 16                     // query heads of a unit at most

struct StepHead { int count, pad[3]; };
// Keys x0 to x1 of those that a token sees: the first `ahead` of its sequence, then those from `first` on.
struct alignas(16) StepItem { i64 base; int sample, chunk, chunks, x0, x1, ahead, first, pad; };

struct StepPlan {
    const i64 *start, *length;
    i64 T;
    int N, window, sinks, most;
    StepHead *head;
    StepItem *items;
    int2 *where;                                        // [N] first item and number of items
};

// Lists the chunks, sequence after sequence.
__global__ void __launch_bounds__(1024) k_step_plan(StepPlan P)
{
    rp_let_next_launch_start();
    __shared__ int sums[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int total = 0;
    for (int i0 = 0; i0 < P.N; i0 += 1024) {
        const int i = i0 + threadIdx.x;
        i64 base = 0;
        int n = 0, seen = 0, ahead = 0, first = 0, size = STEP_CHUNK;
        if (i < P.N) {
            base = max(P.start[i], (i64)0);
            const i64 room = max(min(P.start[i + 1], P.T) - base, (i64)0);
            const int filled = (int)(P.length ? min(max(P.length[i], (i64)0), room) : room);
            first = P.window ? max(filled - P.window, 0) : 0;
            ahead = min(P.sinks, first);
            seen = ahead + filled - first;
            size = max(STEP_CHUNK, ((seen + STEP_CHUNKS - 1) / STEP_CHUNKS + 15) & ~15);
            n = max((seen + size - 1) / size, 1);       // (one without keys as well: it writes the outputs)
        }
        int x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) sums[warp] = x;
        __syncthreads();
        const int before = __reduce_add_sync(0xffffffffu, lane < warp ? sums[lane] : 0), all = __reduce_add_sync(0xffffffffu, sums[lane]);
        __syncthreads();
        const int at = total + before + x - n;
        if (i < P.N) P.where[i] = make_int2(at, at + n <= P.most ? n : 0);
        for (int c = 0; c < n && at + c < P.most; ++c) {
            StepItem it;
            it.base = base; it.sample = i; it.chunk = c; it.chunks = n; it.x0 = c * size; it.x1 = min((c + 1) * size, seen); it.ahead = ahead; it.first = first; it.pad = 0;
            P.items[at + c] = it;
        }
        total += all;
    }
    if (threadIdx.x == 0) P.head->count = min(total, P.most);
}

struct StepArgs {
    const StepHead *head;
    const StepItem *items;
    const int2 *where;
    int N, Hq, share, groups, d, units;        // groups: of 16 query heads to a key head
    float scale;
    const void *q, *k, *v;
    i64 q_token, q_head, k_token, k_head, v_token, v_head;
    void *out;
    i64 o_token, o_head;
    float *lse;
    i64 l_token, l_head;
    float2 *tops;                            // [item][Hq] maximum and sum of a chunk
    float *parts;                            // [item][Hq][d] its values
};

__device__ __forceinline__ void copy16(u32 to, const void *from, bool there)         // 16 bytes, or as many zeros
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void load_matrices(u32 at, u32 *r)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_matrices_across(u32 at, u32 *r)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void multiply(float *c, const u32 *a, const u32 *b, bf16)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ void multiply(float *c, const u32 *a, const u32 *b, __half)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
// Two weights as a pair of the type and a pair of what that leaves of them: as operands they keep 16 bits and more (bf16 alone keeps 8).
template <typename X> __device__ __forceinline__ void two_pairs(float a, float b, u32 &high, u32 &low)
{
    high = rp_pair(a, b, X());
    float x, y;
    if constexpr (std::is_same<X, bf16>::value) { x = __uint_as_float(high << 16); y = __uint_as_float(high & 0xffff0000u); }
    else {
        __half2 h;
        memcpy(&h, &high, 4);
        const float2 f = __half22float2(h);
        x = f.x; y = f.y;
    }
    low = rp_pair(a - x, b - y, X());
}

// The tiles that a warp copies: those of one of its units after the other.
struct StepCursor {
    int unit, x, x1, ahead, first;
    const char *k, *v;
    template <typename X> __device__ __forceinline__ void open(const StepArgs &A, int total)
    {
        for (; unit < total; unit += gridDim.x * STEP_WARPS) {
            const StepItem it = A.items[unit / A.units];
            x = it.x0; x1 = it.x1;
            if (x >= x1) continue;                      // a sequence without keys
            ahead = it.ahead; first = it.first;
            const int hk = unit % A.units / A.groups;
            k = (const char *)((const X *)A.k + it.base * A.k_token + hk * A.k_head);
            v = (const char *)((const X *)A.v + it.base * A.v_token + hk * A.v_head);
            return;
        }
    }
};

template <int D> struct StepSmem {
    static constexpr int TILE = 16 * D * 2, STAGES = 12288 / TILE;       // 96 KB of keys and values: two CTAs to an SM
    unsigned char ring[STEP_WARPS][STAGES][2][TILE];
};

template <typename X, int D>
__global__ void __launch_bounds__(STEP_THREADS, 2) k_attend_step(const StepArgs A)
{
    typedef StepSmem<D> Smem;
    constexpr int STAGES = Smem::STAGES, PIECES = D / 8, NT = D / 8, KS = D / 16;
    constexpr float LIFT = std::is_same<X, bf16>::value ? 1.0f : 32768.0f;            // float16: weights of 1 as 2^15, so that small ones stay something
    extern __shared__ __align__(128) unsigned char raw[];
    Smem &sm = *(Smem *)raw;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const u32 ring = rp_smem(sm.ring[warp]);
    rp_let_next_launch_start();
    rp_wait_for_launch_before();
    const int total = A.head->count * A.units;
    const float sl = A.scale * RP_LOG2E;

    StepCursor in;
    in.unit = blockIdx.x * STEP_WARPS + warp;
    in.open<X>(A, total);
    auto copy = [&](int stage) {                         // the next tile, if there is one
        if (in.unit < total) {
            const int p = lane % PIECES;
#pragma unroll
            for (int i = 0; i < 16 / (32 / PIECES); ++i) {
                const int r = lane / PIECES + i * (32 / PIECES), x = min(in.x + r, in.x1 - 1);
                const i64 row = x < in.ahead ? x : in.first + (x - in.ahead);
                const bool there = in.x + r < in.x1 && p * 8 < A.d;
                const u32 to = ring + stage * 2 * Smem::TILE + r * (D * 2) + ((p ^ (r & 7)) << 4);
                const int c = there ? p * 16 : 0;
                copy16(to, in.k + row * A.k_token * 2 + c, there);
                copy16(to + Smem::TILE, in.v + row * A.v_token * 2 + c, there);
            }
            in.x += 16;
            if (in.x >= in.x1) { in.unit += gridDim.x * STEP_WARPS; in.open<X>(A, total); }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int s = 0; s < STAGES; ++s) copy(s);
    int stage = 0;
    for (int unit = blockIdx.x * STEP_WARPS + warp; unit < total; unit += gridDim.x * STEP_WARPS) {
        const StepItem it = A.items[unit / A.units];
        const int hg = unit % A.units, hk = hg / A.groups, h0 = hk * A.share + hg % A.groups * STEP_ROWS, rows = min(A.share - hg % A.groups * STEP_ROWS, STEP_ROWS);
        u32 q[KS][4];
        const X *from = (const X *)A.q + it.sample * A.q_token;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = g + (i & 1) * 8, c = s * 16 + t * 2 + (i >> 1) * 8;
                q[s][i] = r < rows && c < A.d ? *(const u32 *)(from + (h0 + r) * A.q_head + c) : 0u;
            }
        float o[NT][4], m[2] = { -INFINITY, -INFINITY }, l[2] = { 0.0f, 0.0f };
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][i] = 0.0f;
        for (int x = it.x0; x < it.x1; x += 16) {
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
            __syncwarp();
            const u32 kt = ring + stage * 2 * Smem::TILE, vt = kt + Smem::TILE;
            float s[2][4] = { };
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                u32 b[4];
                const int r = (lane >> 4) * 8 + (lane & 7), p = 2 * ks + ((lane >> 3) & 1);
                load_matrices(kt + r * (D * 2) + ((p ^ (r & 7)) << 4), b);
                multiply(s[0], q[ks], b, X());
                multiply(s[1], q[ks], b + 2, X());
            }
            float top[2] = { m[0], m[1] };
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[n][i] = x + n * 8 + t * 2 + (i & 1) < it.x1 ? s[n][i] * sl : -INFINITY;
                    top[i >> 1] = fmaxf(top[i >> 1], s[n][i]);
                }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
            }
            if (__any_sync(0xffffffffu, top[0] > m[0] || top[1] > m[1])) {
                float f[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    f[i] = top[i] == m[i] ? 1.0f : rp_exp2(m[i] - top[i]);
                    l[i] *= f[i];
                    m[i] = top[i];
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[n][i] *= f[i >> 1];
            }
            u32 high[4], low[4];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float less = m[i] == -INFINITY ? 0.0f : m[i];
                    const float a = rp_exp2(s[n][2 * i] - less), b = rp_exp2(s[n][2 * i + 1] - less);
                    l[i] += a + b;
                    two_pairs<X>(a * LIFT, b * LIFT, high[2 * n + i], low[2 * n + i]);
                }
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                u32 b[4];
                const int r = ((lane >> 3) & 1) * 8 + (lane & 7), p = n + (lane >> 4);
                load_matrices_across(vt + r * (D * 2) + ((p ^ (r & 7)) << 4), b);
                multiply(o[n], high, b, X());
                multiply(o[n + 1], high, b + 2, X());
                multiply(o[n], low, b, X());
                multiply(o[n + 1], low, b + 2, X());
            }
            __syncwarp();
            copy(stage);
            stage = stage + 1 == STAGES ? 0 : stage + 1;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
        }
        const int item = unit / A.units;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = g + 8 * i, h = h0 + r;
            if (r >= rows) continue;
            if (it.chunks > 1) {
                float *part = A.parts + ((i64)item * A.Hq + h) * A.d;
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    if (n * 8 < A.d) *(float2 *)(part + n * 8 + t * 2) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
                if (t == 0) A.tops[(i64)item * A.Hq + h] = make_float2(m[i], l[i]);
                continue;
            }
            const bool none = it.x1 <= it.x0;            // no key at all: nothing, and the log of nothing
            const float f = none ? 0.0f : 1.0f / (l[i] * LIFT);
            X *out = (X *)A.out + it.sample * A.o_token + h * A.o_head;
#pragma unroll
            for (int n = 0; n < NT; ++n)
                if (n * 8 < A.d) *(u32 *)(out + n * 8 + t * 2) = rp_pair(o[n][2 * i] * f, o[n][2 * i + 1] * f, X());
            if (t == 0 && A.lse) A.lse[it.sample * A.l_token + h * A.l_head] = none ? -INFINITY : (m[i] + log2f(l[i])) * 0.6931471805599453f;
        }
        __syncwarp();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// Sequences of several chunks: a warp a query head, a lane four of its columns.
template <typename X>
__global__ void __launch_bounds__(STEP_THREADS) k_step_join(const StepArgs A)
{
    constexpr float LIFT = std::is_same<X, bf16>::value ? 1.0f : 32768.0f;
    constexpr int MINE = STEP_CHUNKS / 32, AHEAD = 8;
    const int lane = threadIdx.x & 31;
    rp_wait_for_launch_before();
    for (i64 unit = (i64)blockIdx.x * STEP_WARPS + (threadIdx.x >> 5); unit < (i64)A.N * A.Hq; unit += (i64)gridDim.x * STEP_WARPS) {
        const int sample = (int)(unit / A.Hq), h = (int)(unit % A.Hq);
        const int2 at = A.where[sample];
        if (at.y <= 1) continue;
        float2 y[MINE];
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int c = i * 32 + lane;
            y[i] = c < at.y ? A.tops[(i64)(at.x + c) * A.Hq + h] : make_float2(-INFINITY, 0.0f);
            top = fmaxf(top, y[i].x);
        }
#pragma unroll
        for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            y[i].x = y[i].x == top ? 1.0f : rp_exp2(y[i].x - top);
            sum = fmaf(y[i].y, y[i].x, sum);
        }
#pragma unroll
        for (int x = 16; x; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
        const int e = lane * 4;
        const float *part = A.parts + ((i64)at.x * A.Hq + h) * A.d + (e < A.d ? e : 0);
        float o[4] = { };
#pragma unroll
        for (int i = 0; i < MINE; ++i)
            for (int c0 = i * 32; c0 < min(at.y, i * 32 + 32); c0 += AHEAD) {
                float4 z[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) z[u] = c0 + u < at.y ? *(const float4 *)(part + (i64)(c0 + u) * A.Hq * A.d) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const float f = __shfl_sync(0xffffffffu, y[i].x, (c0 + u) & 31);
                    if (c0 + u >= at.y) continue;
                    o[0] = fmaf(z[u].x, f, o[0]); o[1] = fmaf(z[u].y, f, o[1]); o[2] = fmaf(z[u].z, f, o[2]); o[3] = fmaf(z[u].w, f, o[3]);
                }
            }
        const float f = 1.0f / (sum * LIFT);
        if (e < A.d) *(uint2 *)((X *)A.out + sample * A.o_token + h * A.o_head + e) = make_uint2(rp_pair(o[0] * f, o[1] * f, X()), rp_pair(o[2] * f, o[3] * f, X()));
        if (lane == 0 && A.lse) A.lse[sample * A.l_token + h * A.l_head] = (top + log2f(sum)) * 0.6931471805599453f;
    }
}

// ---------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------
struct StepSpace { i64 items, where, tops, parts, all; };
static int step_units(const rp_attend_config *a) { return a->kv_heads * ((a->q_heads / a->kv_heads + STEP_ROWS - 1) / STEP_ROWS); }
static i64 step_most(i64 T, int N, int window, int sinks)
{
    i64 each = STEP_CHUNKS;
    if (window) each = std::min(each, ((i64)window + sinks) / STEP_CHUNK + 1);
    return std::min(T / STEP_CHUNK + N, N * each);
}
static StepSpace step_space(const rp_attend_config *a, i64 T, int N, int window, int sinks)
{
    const i64 most = step_most(T, N, window, sinks);
    const auto up = [](i64 x) { return (x + 15) / 16 * 16; };
    StepSpace s;
    s.items = sizeof(StepHead);
    s.where = s.items + most * (i64)sizeof(StepItem);
    s.tops = up(s.where + 8ll * N);
    s.parts = up(s.tops + most * a->q_heads * 8);
    s.all = s.parts + most * a->q_heads * a->head_dim * 4;
    return s;
}
static int check_step(const rp_attend_config *a, int window, int sinks, i64 T, int N)
{
    RP_TRY(rp_attend_check(a, T, N));
    return window < 0 || sinks < 0 ? RP_ERR_ARG : RP_OK;
}

extern "C" int64_t rp_attend_step_workspace(const rp_attend_config *a, int32_t window, int32_t sinks, int64_t n_tokens, int32_t n_samples)
{
    return check_step(a, window, sinks, n_tokens, n_samples) == RP_OK ? step_space(a, n_tokens, n_samples, window, sinks).all : 0;
}

template <typename X, int D>
static int launch(const StepArgs &A, i64 units, bool several, int sms, cudaStream_t stream)
{
    const size_t smem = sizeof(StepSmem<D>);
    RP_CUDA(cudaFuncSetAttribute(k_attend_step<X, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t how = {};
    how.gridDim = dim3((unsigned)std::min((i64)sms * 2, (units + STEP_WARPS - 1) / STEP_WARPS));
    how.blockDim = dim3(STEP_THREADS);
    how.dynamicSmemBytes = smem;
    how.stream = stream;
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    how.attrs = &early; how.numAttrs = 1;
    RP_CUDA(cudaLaunchKernelEx(&how, k_attend_step<X, D>, A));
    RP_TRY(rp_op_launched());
    if (!several) return RP_OK;
    how.gridDim = dim3((unsigned)std::min((i64)sms * 8, ((i64)A.N * A.Hq + STEP_WARPS - 1) / STEP_WARPS));
    how.dynamicSmemBytes = 0;
    RP_CUDA(cudaLaunchKernelEx(&how, k_step_join<X>, A));
    return rp_op_launched();
}

extern "C" int rp_attend_step(const rp_attend_config *a, int32_t window, int32_t sinks, int64_t n_tokens, const rp_view *q, const rp_view *k, const rp_view *v,
                              const int64_t *start, int32_t n_samples, const int64_t *length, const rp_view *out, const rp_view *lse, void *workspace,
                              int64_t workspace_bytes, void *cuda_stream)
{
    RP_TRY(check_step(a, window, sinks, n_tokens, n_samples));
    const int N = n_samples;
    const StepSpace space = step_space(a, n_tokens, N, window, sinks);
    if (!start || !rp_aligned(start, 8) || !rp_aligned(length, 8) || !workspace || !rp_aligned(workspace, 16) || workspace_bytes < space.all) return RP_ERR_ARG;
    RpOpDevice dev;
    const rp_view *const places[] = { out, lse, q, k, v };
    if (rp_attend_shared(places, 2, 3)) return RP_ERR_ARG;
    RP_TRY(rp_attend_view(q, N, a->q_heads, dev));
    RP_TRY(rp_attend_view(out, N, a->q_heads, dev));
    if (n_tokens) {                                      // (an empty cache has no address)
        RP_TRY(rp_attend_view(k, n_tokens, a->kv_heads, dev));
        RP_TRY(rp_attend_view(v, n_tokens, a->kv_heads, dev));
    }
    if (lse && lse->x && !rp_aligned(lse->x, 4)) return RP_ERR_ARG;
    RP_TRY(rp_op_enter(dev, start, length, workspace, lse ? lse->x : nullptr));
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    char *const w = (char *)workspace;
    StepPlan P = {};
    P.start = (const i64 *)start; P.length = (const i64 *)length; P.T = n_tokens; P.N = N; P.window = window; P.sinks = sinks;
    P.most = (int)step_most(n_tokens, N, window, sinks); P.head = (StepHead *)w; P.items = (StepItem *)(w + space.items); P.where = (int2 *)(w + space.where);
    k_step_plan<<<1, 1024, 0, stream>>>(P);
    RP_TRY(rp_op_launched());
    StepArgs A = {};
    A.head = P.head; A.items = P.items; A.where = P.where; A.N = N; A.Hq = a->q_heads; A.share = a->q_heads / a->kv_heads; A.units = step_units(a);
    A.groups = A.units / a->kv_heads; A.d = a->head_dim; A.scale = a->scale; A.q = q->x; A.q_token = q->token; A.q_head = q->head; A.out = out->x; A.o_token = out->token; A.o_head = out->head;
    if (n_tokens) { A.k = k->x; A.k_token = k->token; A.k_head = k->head; A.v = v->x; A.v_token = v->token; A.v_head = v->head; }
    if (lse && lse->x) { A.lse = (float *)lse->x; A.l_token = lse->token; A.l_head = lse->head; }
    A.tops = (float2 *)(w + space.tops); A.parts = (float *)(w + space.parts);
    const int sms = rp_op_sms(dev.device);
    const i64 units = (i64)P.most * A.units;
    const bool several = n_tokens > STEP_CHUNK && (!window || (i64)window + sinks > STEP_CHUNK);
    if (a->type == RP_F16) return a->head_dim <= 64 ? launch<__half, 64>(A, units, several, sms, stream) : launch<__half, 128>(A, units, several, sms, stream);
    return a->head_dim <= 64 ? launch<bf16, 64>(A, units, several, sms, stream) : launch<bf16, 128>(A, units, several, sms, stream);
}
