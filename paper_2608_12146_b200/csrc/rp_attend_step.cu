// Attention of one new token of each sequence against the keys and values of those before it (decoding).
//
//   s = scale q k^T over the keys that the token sees, o = softmax(s) v, lse = log sum exp(s)
//
// Bound by HBM: each visible key and value is read once, 4 * head_dim bytes for 4 * share * head_dim operations (share: query heads to a key head).  The products go
// through the warps' matrix instruction, 16 query heads by 16 keys at a time, of which `share` rows are something: with a few rows to a tile there is nothing that
// fuller instructions could add.
// The keys that a sequence's token sees are cut into chunks of 256, or of a 64th of them where that is more; a chunk and a key head are a unit, and CTAs stay resident
// and take units in turn.  The cut goes by the sequence alone, so that its bits do not depend on the others of the batch.  A warp takes every fourth tile of 16 keys through
// a ring of its own in shared memory, which runs on into the next unit; the four meet at the unit's end.  The last CTA to be done with a sequence's head adds up its
// chunks, in their order.
#include <algorithm>

#include "rp_attend.cuh"

#define STEP_WARPS 4
#define STEP_THREADS (32 * STEP_WARPS)
#define STEP_CHUNK 256                   // keys of a chunk at least
#define STEP_CHUNKS 64                   // chunks of a sequence at most
#define STEP_ROWS 16                     // query heads of a unit at most

struct StepHead { int count, pad[3]; };
// Keys x0 to x1 of those that a token sees: the first `ahead` of its sequence, then those from `first` on.
struct alignas(16) StepItem { i64 base; int sample, chunk, chunks, x0, x1, ahead, first, pad; };

struct StepPlan {
    const i64 *start, *length;
    i64 T;
    int N, window, sinks, most, units;                  // units: of a chunk (key heads, in groups of 16 query heads)
    StepHead *head;
    StepItem *items;
    int *done;                                          // [N][units] chunks that are worked out
};

// CTA 0 lists the chunks, sequence after sequence; the others set the counters to 0.
__global__ void __launch_bounds__(1024) k_step_plan(StepPlan P)
{
    rp_let_next_launch_start();
    if (blockIdx.x) {
        for (i64 i = (i64)(blockIdx.x - 1) * 1024 + threadIdx.x; i < (i64)P.N * P.units; i += (i64)(gridDim.x - 1) * 1024) P.done[i] = 0;
        return;
    }
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
    int *done;
    int Hq, share, groups, d, units;        // groups: of 16 query heads to a key head
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

// The tiles that a warp copies: its own of one unit after the other.
struct StepCursor {
    int unit, x, x1, ahead, first;
    const char *k, *v;
    template <typename X> __device__ __forceinline__ void open(const StepArgs &A, int total, int warp)
    {
        for (; unit < total; unit += gridDim.x) {
            const StepItem it = A.items[unit / A.units];
            x = it.x0 + 16 * warp; x1 = it.x1;
            if (x >= x1) continue;
            ahead = it.ahead; first = it.first;
            const int hk = unit % A.units / A.groups;
            k = (const char *)((const X *)A.k + it.base * A.k_token + hk * A.k_head);
            v = (const char *)((const X *)A.v + it.base * A.v_token + hk * A.v_head);
            return;
        }
    }
};

template <int D> struct StepSmem {
    static constexpr int TILE = 16 * D * 2, STAGES = 12288 / TILE;       // 96 KB of keys and values, 113 KB in all: two CTAs to an SM
    unsigned char ring[STEP_WARPS][STAGES][2][TILE];
    union {
        float o[STEP_WARPS][8][D + 4];                   // the warps' sums
        float f[STEP_ROWS][STEP_CHUNKS];                 // the chunks' factors
    };
    float2 top[STEP_WARPS][8];
    float inv[STEP_ROWS];
    int last;
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
    rp_wait_for_launch_before();
    const int total = A.head->count * A.units;
    const float sl = A.scale * RP_LOG2E;

    StepCursor in;
    in.unit = blockIdx.x;
    in.open<X>(A, total, warp);
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
            in.x += 16 * STEP_WARPS;
            if (in.x >= in.x1) { in.unit += gridDim.x; in.open<X>(A, total, warp); }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int s = 0; s < STAGES; ++s) copy(s);
    int stage = 0;
    for (int unit = blockIdx.x; unit < total; unit += gridDim.x) {
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
        for (int x = it.x0 + 16 * warp; x < it.x1; x += 16 * STEP_WARPS) {
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
        // The warps meet, eight heads at a time.
        const bool whole = it.chunks == 1;
        const int item = unit / A.units;
        for (int half = 0; half < (rows > 8 ? 2 : 1); ++half) {
#pragma unroll
            for (int n = 0; n < NT; ++n) *(float2 *)&sm.o[warp][g][n * 8 + t * 2] = half ? make_float2(o[n][2], o[n][3]) : make_float2(o[n][0], o[n][1]);
            if (t == 0) sm.top[warp][g] = half ? make_float2(m[1], l[1]) : make_float2(m[0], l[0]);
            __syncthreads();
            for (int e = threadIdx.x * 2; e < 8 * D; e += STEP_THREADS * 2) {
                const int r = e / D, c = e % D, h = h0 + half * 8 + r;
                if (half * 8 + r >= rows || c >= A.d) continue;
                float top = -INFINITY, sum = 0.0f, a = 0.0f, b = 0.0f;
#pragma unroll
                for (int w = 0; w < STEP_WARPS; ++w) top = fmaxf(top, sm.top[w][r].x);
#pragma unroll
                for (int w = 0; w < STEP_WARPS; ++w) {
                    const float2 y = sm.top[w][r], z = *(const float2 *)&sm.o[w][r][c];
                    const float f = y.x == top ? 1.0f : rp_exp2(y.x - top);
                    sum = fmaf(y.y, f, sum);
                    a = fmaf(z.x, f, a); b = fmaf(z.y, f, b);
                }
                if (!whole) {
                    *(float2 *)(A.parts + ((i64)item * A.Hq + h) * A.d + c) = make_float2(a, b);
                    if (c == 0) A.tops[(i64)item * A.Hq + h] = make_float2(top, sum);
                } else {
                    const bool none = it.x1 <= it.x0;    // no key at all: nothing, and the log of nothing
                    const float f = none ? 0.0f : 1.0f / (sum * LIFT);
                    *(u32 *)((X *)A.out + it.sample * A.o_token + h * A.o_head + c) = rp_pair(a * f, b * f, X());
                    if (c == 0 && A.lse) A.lse[it.sample * A.l_token + h * A.l_head] = none ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
                }
            }
            __syncthreads();
        }
        if (whole) continue;
        // (what this CTA's threads have written is there for the others before the count goes up)
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) sm.last = atomicAdd(A.done + (i64)it.sample * A.units + hg, 1) == it.chunks - 1;
        __syncthreads();
        if (!sm.last) continue;
        __threadfence();
        const i64 item0 = item - it.chunk;
        for (int r = warp; r < rows; r += STEP_WARPS) {
            float2 y[STEP_CHUNKS / 32];
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < STEP_CHUNKS / 32; ++i) {
                const int c = i * 32 + lane;
                y[i] = c < it.chunks ? __ldcg(A.tops + (item0 + c) * A.Hq + h0 + r) : make_float2(-INFINITY, 0.0f);
                top = fmaxf(top, y[i].x);
            }
#pragma unroll
            for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
#pragma unroll
            for (int i = 0; i < STEP_CHUNKS / 32; ++i) {
                const float f = y[i].x == top ? 1.0f : rp_exp2(y[i].x - top);
                sum = fmaf(y[i].y, f, sum);
                sm.f[r][i * 32 + lane] = f;
            }
#pragma unroll
            for (int x = 16; x; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
            if (lane == 0) {
                sm.inv[r] = 1.0f / (sum * LIFT);
                if (A.lse) A.lse[it.sample * A.l_token + (h0 + r) * A.l_head] = (top + log2f(sum)) * 0.6931471805599453f;
            }
        }
        __syncthreads();
        for (int e = threadIdx.x * 2; e < rows * A.d; e += STEP_THREADS * 2) {
            const int r = e / A.d, c = e % A.d, h = h0 + r;
            const float *p = A.parts + (item0 * A.Hq + h) * A.d + c;
            float a = 0.0f, b = 0.0f;
#pragma unroll 8
            for (int i = 0; i < it.chunks; ++i) {
                const float2 z = __ldcg((const float2 *)(p + (i64)i * A.Hq * A.d));
                a = fmaf(z.x, sm.f[r][i], a); b = fmaf(z.y, sm.f[r][i], b);
            }
            *(u32 *)((X *)A.out + it.sample * A.o_token + h * A.o_head + c) = rp_pair(a * sm.inv[r], b * sm.inv[r], X());
        }
        __syncthreads();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// ---------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------
struct StepSpace { i64 items, done, tops, parts, all; };
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
    s.done = s.items + most * (i64)sizeof(StepItem);
    s.tops = up(s.done + 4ll * N * step_units(a));
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
static int launch(const StepArgs &A, i64 units, int sms, cudaStream_t stream)
{
    const size_t smem = sizeof(StepSmem<D>);
    RP_CUDA(cudaFuncSetAttribute(k_attend_step<X, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t how = {};
    how.gridDim = dim3((unsigned)std::min((i64)sms * 2, units));
    how.blockDim = dim3(STEP_THREADS);
    how.dynamicSmemBytes = smem;
    how.stream = stream;
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    how.attrs = &early; how.numAttrs = 1;
    RP_CUDA(cudaLaunchKernelEx(&how, k_attend_step<X, D>, A));
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
    P.most = (int)step_most(n_tokens, N, window, sinks); P.units = step_units(a); P.head = (StepHead *)w; P.items = (StepItem *)(w + space.items);
    P.done = (int *)(w + space.done);
    k_step_plan<<<1 + (int)std::min(((i64)N * P.units + 1023) / 1024, (i64)32), 1024, 0, stream>>>(P);
    RP_TRY(rp_op_launched());
    StepArgs A = {};
    A.head = P.head; A.items = P.items; A.done = P.done; A.Hq = a->q_heads; A.share = a->q_heads / a->kv_heads; A.groups = P.units / a->kv_heads; A.d = a->head_dim;
    A.units = P.units; A.scale = a->scale; A.q = q->x; A.q_token = q->token; A.q_head = q->head; A.out = out->x; A.o_token = out->token; A.o_head = out->head;
    if (n_tokens) { A.k = k->x; A.k_token = k->token; A.k_head = k->head; A.v = v->x; A.v_token = v->token; A.v_head = v->head; }
    if (lse && lse->x) { A.lse = (float *)lse->x; A.l_token = lse->token; A.l_head = lse->head; }
    A.tops = (float2 *)(w + space.tops); A.parts = (float *)(w + space.parts);
    const int sms = rp_op_sms(dev.device);
    const i64 units = (i64)P.most * P.units;
    if (a->type == RP_F16) return a->head_dim <= 64 ? launch<__half, 64>(A, units, sms, stream) : launch<__half, 128>(A, units, sms, stream);
    return a->head_dim <= 64 ? launch<bf16, 64>(A, units, sms, stream) : launch<bf16, 128>(A, units, sms, stream);
}
