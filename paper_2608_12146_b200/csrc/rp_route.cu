// Router of one MoE layer with its balance loss, and its gradient.
//
//   s = softmax(x) or sigmoid(x) over the E experts, p = s / sum s
//   gates: scale * s at the k chosen or replayed experts (over their sum)
//   loss = coef / G * sum_g E / (k T_g^2) * sum_e counts[g][e] * sum_{t in g} p[t][e]
//
// One pass over the logits each way: T * E elements read (and written by the gradient), T * k routes and gates beside them.
// A token belongs to SUB neighbouring lanes of a warp, VPL experts to a lane, so that its row is read with one or two 16-byte loads a lane and all
// sums over experts are shuffles.  Every such group of lanes owns a run of neighbouring tokens and carries the sums of p of the run's
// present group of tokens in registers, its counts in shared memory; what a CTA's last runs hold meets in shared memory before it goes out.
// Sums of p leave a CTA in fixed point (2^-36): additions of whole numbers, so their order does not matter.
// Bound by instructions: 131072 tokens of 256 experts, k = 8, take 80 us where their bytes take 12: 427 warp instructions a token (scores of 8 experts a lane, their keys,
// k rounds of the largest), 73 % of the issue slots, the integer units 58 %.  The gradient, 344 a token, 64 us (its bytes 22): it waits for shuffles and shared memory.
#include <limits.h>

#include <algorithm>

#include "rp_ops.cuh"

#define ROUTE_WARPS 8
#define ROUTE_THREADS (32 * ROUTE_WARPS)
#define ROUTE_MAX_K 32
#define ROUTE_FIX 68719476736.0f            // 2^36: up to 2^26 tokens of p <= 1 add up to less than 2^63
#define ROUTE_LOSS_CTAS 128

struct RouteSpace {                         // workspace of rp_route; sums [G][E] behind it
    u32 ticket, loss_ticket, odd, pad;      // odd: some p was not a number
    double part[ROUTE_LOSS_CTAS];
};

struct RouteArgs {
    const void *x;
    i64 row, T, run;                        // run: tokens of a group of lanes
    int E, k, score, normalise, replay, G;
    float scale, coef;
    const float *bias;
    const i64 *start;
    void *routes;
    int route_bytes;
    i64 route_row;
    float *gates;
    int *counts;
    u64 *sums;
    RouteSpace *space;
    float *loss;
    int wide;                               // rows can be read (and written) 16 bytes at a time
    int finish;                             // 0: one CTA does it all, 1: the last CTA works out the loss, 2: another launch does
    // gradient
    const float *gates_grad, *loss_grad;
    const int *counts_in;
    void *dx;
    i64 dx_row;
};

template <int SUB> __device__ __forceinline__ float sub_sum(float v)
{
#pragma unroll
    for (int o = 1; o < SUB; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int SUB> __device__ __forceinline__ u32 sub_max(u32 v);
__device__ __forceinline__ u32 order_of(float x);
template <int SUB> __device__ __forceinline__ float sub_max(float v)      // of numbers; NaN loses against any
{
    if constexpr (SUB == 32) {                              // by one instruction of the whole warp, on numbers in the floats' order (fmaxf has taken NaN out, or all are)
        const u32 m = sub_max<SUB>(v == v ? order_of(v) : 0u);
        return m == 0 ? NAN : __uint_as_float((m >> 31) ? m ^ 0x80000000u : ~m);
    } else {
#pragma unroll
        for (int o = 1; o < SUB; o <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
        return v;
    }
}
template <int SUB> __device__ __forceinline__ u32 sub_max(u32 v)
{
    if constexpr (SUB == 32) return __reduce_max_sync(0xffffffffu, v);
    else {
#pragma unroll
        for (int o = 1; o < SUB; o <<= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
        return v;
    }
}

// A row's VPL elements of a lane, as they lie in memory: read 16 bytes at a time (then a lane's eight all exist or none does), or one by one where rows are not on such
// boundaries.  Experts from E on have a logit of -inf: they come behind all others and have a score of 0.
template <typename X, int VPL> struct Row {
    Pack8<X> p[VPL / 8];
    __device__ __forceinline__ Row()
    {
#pragma unroll
        for (int c = 0; c < VPL / 8; ++c)
#pragma unroll
            for (int i = 0; i < (int)sizeof(X) / 2; ++i) {
                const u32 w = sizeof(X) == 4 ? 0xff800000u : std::is_same<X, bf16>::value ? 0xff80ff80u : 0xfc00fc00u;
                p[c].w[i] = make_uint4(w, w, w, w);
            }
    }
};
template <typename X, int VPL>
__device__ __forceinline__ void load_row(const RouteArgs &A, const X *row, int e0, Row<X, VPL> &r)      // row: of the lane's first expert
{
#pragma unroll
    for (int c = 0; c < VPL; c += 8) {
        if (A.wide) {
            if (e0 + c < A.E) r.p[c / 8] = rp_load8(row + c);
        } else {
            X x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = e0 + c + i < A.E ? row[c + i] : rp_round<X>(-INFINITY);
            memcpy(&r.p[c / 8], x, sizeof(x));
        }
    }
}
template <typename X, int VPL> __device__ __forceinline__ void open_row(const Row<X, VPL> &r, float *x)
{
#pragma unroll
    for (int c = 0; c < VPL; c += 8) rp_open8(r.p[c / 8], x + c);
}

__device__ __forceinline__ float reciprocal(float x)        // by the special function unit: 1 ulp
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sigmoid(float x) { return reciprocal(1.0f + rp_exp2(-x * RP_LOG2E)); }

__device__ __forceinline__ float min_or_nan(float x, float y)
{
    float z;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}

// Scores of one token from its logits: softmax: e^(x - max) and 1 / their sum; sigmoid: s, and 1 / their sum.
// `top` is what the largest logit is taken for: 0 where it is -inf (all scores are 0 then, and so is the inverse).
// SHARED: two sigmoids share a reciprocal, 1 / (1 + a) = (1 + b) / ((1 + a)(1 + b)), where a score of less than 2^-63 counts as 2^-63; rows whose scores add up to
// less than 2^-28 are worked out one by one (1024 such experts are 2^-25 of that).  So are all rows whose experts are chosen by score and bias: a score may not
// depend on its neighbour's logit there (equal logits are ties, and a NaN stays where it is).
template <int VPL, int SUB, bool SHARED>
__device__ __forceinline__ void scores(const RouteArgs &A, const float *x, float *s, float &top, float &inv)
{
    float sum = 0.0f;
    top = 0.0f;
    if (A.score == RP_SCORE_SOFTMAX) {
        float m = x[0];
#pragma unroll
        for (int i = 1; i < VPL; ++i) m = fmaxf(m, x[i]);
        m = sub_max<SUB>(m);
        top = m == -INFINITY ? 0.0f : m;
        // (the difference first: a maximum beyond 2^30, such as a row of nothing but the type's lowest value, would shift all exponents by an error of its own)
        f2 both = rp_f2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < VPL; i += 2) {
            const f2 v = rp_exp2(rp_mul(rp_add(rp_f2(x[i], x[i + 1]), rp_f2(-top, -top)), rp_f2(RP_LOG2E, RP_LOG2E)));
            both = rp_add(both, v);
            rp_parts(v, s[i], s[i + 1]);
        }
        float other;
        rp_parts(both, sum, other);
        sum += other;
        sum = sub_sum<SUB>(sum);
    } else {
        if (SHARED && !A.bias) {
            f2 both = rp_f2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < VPL; i += 2) {
                float a, b;
                rp_parts(rp_mul(rp_f2(x[i], x[i + 1]), rp_f2(-RP_LOG2E, -RP_LOG2E)), a, b);
                rp_parts(rp_add(rp_f2(rp_exp2(min_or_nan(a, 63.0f)), rp_exp2(min_or_nan(b, 63.0f))), rp_f2(1.0f, 1.0f)), a, b);
                const float r = reciprocal(a * b);
                const f2 v = rp_mul(rp_f2(b, a), rp_f2(r, r));
                both = rp_add(both, v);
                rp_parts(v, s[i], s[i + 1]);
            }
            float other;
            rp_parts(both, sum, other);
            sum = sub_sum<SUB>(sum + other);
        }
        if constexpr (!SHARED) {
#pragma unroll
            for (int i = 0; i < VPL; ++i) { s[i] = sigmoid(x[i]); sum += s[i]; }
            sum = sub_sum<SUB>(sum);
        } else if (const bool alone = A.bias || sum < 4.0e-9f; __any_sync(0xffffffffu, alone)) {
            float s1[VPL], sum1 = 0.0f;                      // (the warp's other tokens keep theirs)
#pragma unroll
            for (int i = 0; i < VPL; ++i) { s1[i] = sigmoid(x[i]); sum1 += s1[i]; }
            sum1 = sub_sum<SUB>(sum1);
            if (alone) {
                sum = sum1;
#pragma unroll
                for (int i = 0; i < VPL; ++i) s[i] = s1[i];
            }
        }
    }
    inv = sum < 1.2e-38f ? 0.0f : reciprocal(sum);
}
// Score of one expert as the gates use it.
__device__ __forceinline__ float score_of(const RouteArgs &A, float x, float top, float inv)
{
    if (A.score != RP_SCORE_SOFTMAX) return sigmoid(x);
    return rp_exp2((x - top) * RP_LOG2E) * inv;
}

// Shares of a token's choices in their sum, over the lanes that have them, from the logits alone: for sums under SHARES_FROM, where scores leave the numbers' range while
// their shares do not.  (A sigmoid of less than that is e^x.)  No choice with a score: 0.
#define SHARES_FROM 1.0e-30f
__device__ __forceinline__ float shares(bool valid, float x, int k_lanes)
{
    float m = valid ? x : -INFINITY;
    for (int o = 1; o < k_lanes; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float v = valid && m > -INFINITY ? rp_exp2((x - m) * RP_LOG2E) : 0.0f;
    float total = v;
    for (int o = 1; o < k_lanes; o <<= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    return total > 0.0f ? v * reciprocal(total) : 0.0f;
}

// Floats as unsigned numbers in the same order; -0 as 0, NaN above all.
__device__ __forceinline__ u32 order_of(float x)
{
    const int b = __float_as_int(x + 0.0f);                  // (any NaN becomes 0x7fffffff)
    return (u32)b ^ ((u32)(b >> 31) | 0x80000000u);
}

// Two 16-bit numbers as unsigned ones in the same order; -0 as 0, NaN above all.
__device__ __forceinline__ u32 signs_of_pair(u32 w) { u32 m; asm("prmt.b32 %0, %1, 0, 0xbb99;" : "=r"(m) : "r"(w)); return m; }      // 0xffff where the sign is set
__device__ __forceinline__ u32 order_of_pair(u32 w, bf16) { asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(w) : "r"(0u)); return w ^ (signs_of_pair(w) | 0x80008000u); }
__device__ __forceinline__ u32 order_of_pair(u32 w, __half) { asm("add.rn.f16x2 %0, %0, %1;" : "+r"(w) : "r"(0u)); return w ^ (signs_of_pair(w) | 0x80008000u); }
__device__ __forceinline__ float of_16(u32 w, bf16) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float of_16(u32 w, __half) { return __half2float(__ushort_as_half((unsigned short)w)); }

// The k experts with the largest logits, in falling order, ties to the lower one: lane j of the token's gets the j-th, and its logit.
// 16-bit logits leave half a word for the expert's number: keys that are all different and tell it all.  The largest of all goes round by
// round; a lane has only its two largest at hand.  Where one that has had both turns out to hold a third of the k (one token in 25 of independent logits,
// 256 experts and k = 8), the token is done again by lanes that look for their next key each time.
template <typename X, int VPL, int SUB>
__device__ __forceinline__ void choose_by_keys(const RouteArgs &A, const Row<X, VPL> &row, int e0, int sl, i64 &e, float &xe)
{
    u32 key[VPL], first = 0, second = 0;
    const u32 code = (u32)(1023 - e0) | 0x400u;
#pragma unroll
    for (int i = 0; i < VPL; i += 2) {
        const uint4 &q = row.p[i / 8].w[0];
        const u32 w = order_of_pair(i % 8 == 0 ? q.x : i % 8 == 2 ? q.y : i % 8 == 4 ? q.z : q.w, X()), codes = (code - i) | (code - i - 1) << 16;
        key[i] = __byte_perm(codes, w, 0x5410);
        key[i + 1] = __byte_perm(codes, w, 0x7632);
        first = max(max(first, key[i]), key[i + 1]);
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) second = max(second, key[i] - first);      // (those below it wrap around to the largest numbers, in their order)
    second += first;
    u32 mine = 0, best = 0;
#pragma unroll 4
    for (int j = 0; j < A.k; ++j) {
        best = sub_max<SUB>(first);
        if (sl == j) mine = best;
        if (first == best) { first = second; second = 0; }
    }
    const bool both = first == 0;
    if (__any_sync(0xffffffffu, both)) {
        int more = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i) more += key[i] >= best;
        if (__any_sync(0xffffffffu, both && more > 2)) {
            u32 limit = 0;
            for (int j = 0; j < A.k; ++j) {
                u32 f = 0;
#pragma unroll
                for (int i = 0; i < VPL; ++i) f = max(f, key[i] - limit);
                best = sub_max<SUB>(f) + limit;
                if (sl == j) mine = best;
                limit = best;
            }
        }
    }
    e = 1023 - (int)(mine & 0x3ffu);
    const u32 b = mine >> 16;
    xe = of_16(b & 0x8000u ? b ^ 0x8000u : b ^ 0xffffu, X());
}
// The same by any number, round by round: the largest, the lowest lane that has it, and its lowest expert.
template <int VPL, int SUB>
__device__ __forceinline__ void choose_by_numbers(const RouteArgs &A, const float *number, int e0, int sl, i64 &e)
{
    const int first_lane = (threadIdx.x & 31) - sl;
    u32 key[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) key[i] = e0 + i < A.E ? max(order_of(number[i]), 1u) : 0u;
    for (int j = 0; j < A.k; ++j) {
        u32 top = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i) top = max(top, key[i]);
        const u32 best = sub_max<SUB>(top);
        u32 who = __ballot_sync(0xffffffffu, top == best) >> first_lane;
        if (SUB < 32) who &= (1u << (SUB & 31)) - 1u;
        const int owner = __ffs((int)who) - 1;
        int at = 0;
#pragma unroll
        for (int i = VPL - 1; i >= 0; --i) at = key[i] == best ? i : at;
#pragma unroll
        for (int i = 0; i < VPL; ++i) key[i] = sl == owner && i == at ? 0u : key[i];
        const int found = __shfl_sync(0xffffffffu, e0 + at, first_lane + owner);
        if (sl == j) e = found;
    }
}

// Counts, sums of p and the front of the workspace before several CTAs add to them.
__global__ void __launch_bounds__(ROUTE_THREADS) k_route_clear(RouteArgs A)
{
    rp_let_next_launch_start();
    const i64 cells = (i64)A.G * A.E, step = (i64)gridDim.x * ROUTE_THREADS, first = (i64)blockIdx.x * ROUTE_THREADS + threadIdx.x;
    for (i64 x = first; x < cells; x += step) {
        A.counts[x] = 0;
        if (A.loss) A.sums[x] = 0;
    }
    if (A.loss && first == 0) { A.space->ticket = 0; A.space->loss_ticket = 0; A.space->odd = 0; }
}

// One group's part of the loss, by one warp.
__device__ double group_loss(const RouteArgs &A, int g, int lane)
{
    i64 lo = A.start[g], hi = A.start[g + 1];
    lo = lo < 0 ? 0 : lo; hi = hi > A.T ? A.T : hi;
    if (hi <= lo) return 0.0;
    double sum = 0.0;
    for (int e = lane; e < A.E; e += 32)
        sum += (double)__ldcg(A.counts + (i64)g * A.E + e) * ((double)__ldcg(A.sums + (i64)g * A.E + e) * (1.0 / 68719476736.0));
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const double n = (double)(hi - lo);
    return sum * ((double)A.coef / A.G * A.E / A.k / (n * n));
}
// The groups first, first + step, ... of each warp, added up in a fixed order by all threads of a CTA.
__device__ double groups_loss(const RouteArgs &A, int first, int step, double *part)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double sum = 0.0;
    for (i64 g = first + warp; g < A.G; g += step) sum += group_loss(A, (int)g, lane);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < ROUTE_WARPS; ++w) sum += part[w];
    return sum;
}

template <int VPL>
__device__ __forceinline__ void add_sums(const RouteArgs &A, int g, int e0, const float *acc)
{
    bool odd = false;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        if (e0 + i >= A.E) continue;
        if (!(acc[i] >= 0.0f && acc[i] < 1.0e8f)) { odd = true; continue; }
        const u64 v = __float2ull_rn(acc[i] * ROUTE_FIX);
        if (v) atomicAdd(&A.sums[(i64)g * A.E + e0 + i], v);
    }
    if (odd) atomicExch(&A.space->odd, 1u);
}

// Adds up over a CTA's runs what each has of the group that it ends in, expert by expert: PARTS neighbouring lanes an expert, each with as many runs; where those
// all end in one group, as they mostly do, the lanes' sums meet before they go out.  (A thread an expert: 2048 tokens of 16 experts 26.8 us, of 64 20.2 us.)
template <int NSUB, int EP, typename Get, typename Put>
__device__ __forceinline__ void meet(const RouteArgs &A, const int *last, Get get, Put put)
{
    constexpr int PARTS = EP < ROUTE_THREADS ? ROUTE_THREADS / EP : 1, RUNS = NSUB / PARTS;
    const int lane = threadIdx.x & 31, part = threadIdx.x % PARTS;
    for (int e0 = 0; e0 < A.E; e0 += ROUTE_THREADS / PARTS) {            // (all threads go round as often)
        const int e = e0 + threadIdx.x / PARTS;
        const bool there = e < A.E;
        int u = part * RUNS, g = last[u];
        auto sum = there ? get(u, e) : decltype(get(0, 0))(0);
        for (int end = u + RUNS; ++u < end;) {
            const int gu = last[u];
            if (gu != g) {
                if (there && g >= 0) put(g, e, sum);
                g = gu;
                sum = 0;
            }
            if (there) sum += get(u, e);
        }
        if constexpr (PARTS > 1) {
            const int g0 = __shfl_sync(0xffffffffu, g, lane & ~(PARTS - 1));
            if (__all_sync(0xffffffffu, g == g0)) {
#pragma unroll
                for (int o = 1; o < PARTS; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (part) continue;
            }
        }
        if (there && g >= 0) put(g, e, sum);
    }
}

template <typename X, int VPL, int SUB>
__global__ void __launch_bounds__(ROUTE_THREADS, VPL == 8 ? 4 : 1) k_route(RouteArgs A)
{
    constexpr int NSUB = ROUTE_THREADS / SUB, EP = VPL * SUB;             // groups of lanes, experts they hold
    __shared__ int cnt[NSUB][EP];
    __shared__ int last[NSUB];                                           // group of tokens that a run ends in
    __shared__ double part[ROUTE_WARPS];
    __shared__ u32 turn;
    const int sub = threadIdx.x / SUB, sl = threadIdx.x % SUB, e0 = sl * VPL;
    const bool want_loss = A.loss != nullptr, want_counts = A.counts != nullptr;
    if (A.finish == 0 && want_counts) {
        // the only CTA: nobody has cleared its sums
        for (i64 x = threadIdx.x; x < (i64)A.G * A.E; x += ROUTE_THREADS) { A.counts[x] = 0; if (want_loss) A.sums[x] = 0; }
        if (want_loss && threadIdx.x == 0) A.space->odd = 0;
        __threadfence();
    }
    for (int x = threadIdx.x; x < NSUB * EP; x += ROUTE_THREADS) (&cnt[0][0])[x] = 0;
    __syncthreads();

    // the run's tokens are counted from 0; `next`: where the next group begins
    const i64 t0 = ((i64)blockIdx.x * NSUB + sub) * A.run;
    const int run = (int)A.run, n = (int)max(min(A.T - t0, A.run), (i64)0);
    int g = rp_sample_of(A.start, A.G, t0);
    int next = g < A.G ? (int)min(A.start[g + 1] - t0, (i64)INT_MAX) : INT_MAX;
    float acc[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) acc[i] = 0.0f;
    const X *x_at = (const X *)A.x + t0 * A.row;
    float *gate_at = A.gates + t0 * A.k + sl;
    char *route_at = (char *)A.routes + (t0 * A.route_row + sl) * A.route_bytes;
    const i64 route_step = A.route_row * A.route_bytes;
    Row<X, VPL> row;
    i64 e_next = -1;
    if (n > 0) {
        load_row<X, VPL>(A, x_at + e0, e0, row);
        if (A.replay && sl < A.k) e_next = rp_load_route(route_at, A.route_bytes, 0);
    }
    rp_wait_for_launch_before();                                          // the clearing of counts and sums
    int k_lanes = 1;                                                      // lanes that the sum over the chosen goes over
    while (k_lanes < A.k) k_lanes <<= 1;
    for (int step = 0; step < run; ++step, x_at += A.row, gate_at += A.k, route_at += route_step) {
        const bool there = step < n;
        float x[VPL], s[VPL], top = 0.0f, inv = 0.0f, xe = 0.0f;
        const Row<X, VPL> here = row;
        // lane j of the token's has its j-th choice (there are at least k of them)
        i64 e = e_next;
        if (step + 1 < n) {
            load_row<X, VPL>(A, x_at + A.row + e0, e0, row);
            if (A.replay && sl < A.k) e_next = rp_load_route(route_at + route_step, A.route_bytes, 0);
        }
        if constexpr (sizeof(X) == 2)
            if (!A.replay && !A.bias) choose_by_keys<X, VPL, SUB>(A, here, e0, sl, e, xe);
        open_row<X, VPL>(here, x);
        if (want_loss || A.score == RP_SCORE_SOFTMAX || A.bias) scores<VPL, SUB, true>(A, x, s, top, inv);
        if (!A.replay) {
            if (sizeof(X) == 4 || A.bias) {
                float number[VPL];
#pragma unroll
                for (int i = 0; i < VPL; ++i)
                    number[i] = !A.bias ? x[i] : (A.score == RP_SCORE_SOFTMAX ? s[i] * inv : s[i]) + (e0 + i < A.E ? A.bias[e0 + i] : 0.0f);
                choose_by_numbers<VPL, SUB>(A, number, e0, sl, e);
            }
        }
        const bool valid = there && sl < A.k && e >= 0 && e < A.E;
        if (valid && (A.replay || sizeof(X) == 4 || A.bias)) xe = rp_float(x_at[e]);
        const float v = valid ? score_of(A, xe, top, inv) : 0.0f;
        float gate = v * A.scale;
        if (A.normalise) {
            float total = v;
            for (int o = 1; o < k_lanes; o <<= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
            const bool tiny = valid && total < SHARES_FROM;
            gate = total < SHARES_FROM ? 0.0f : gate * reciprocal(total);
            if (__any_sync(0xffffffffu, tiny)) {
                const float y = shares(valid, xe, k_lanes);
                if (tiny) gate = y * A.scale;
            }
        }
        if (there && step >= next) {
            // another group: what the run has of the one before goes out
            if (g >= 0 && g < A.G) {
                if (want_loss) add_sums<VPL>(A, g, e0, acc);
                if (want_counts)
                    for (int i = 0; i < VPL; ++i) {
                        const int c = cnt[sub][e0 + i];
                        if (c) { atomicAdd(&A.counts[(i64)g * A.E + e0 + i], c); cnt[sub][e0 + i] = 0; }
                    }
#pragma unroll
                for (int i = 0; i < VPL; ++i) acc[i] = 0.0f;
            }
            g = rp_sample_of(A.start, A.G, t0 + step);
            next = g < A.G ? (int)min(A.start[g + 1] - t0, (i64)INT_MAX) : INT_MAX;
        }
        __syncwarp();
        const bool held = there && g >= 0 && g < A.G;
        if (want_loss && held) {
#pragma unroll
            for (int i = 0; i < VPL; i += 2) rp_parts(rp_fma(rp_f2(s[i], s[i + 1]), rp_f2(inv, inv), rp_f2(acc[i], acc[i + 1])), acc[i], acc[i + 1]);
        }
        if (valid && held && want_counts) atomicAdd(&cnt[sub][(int)e], 1);
        if (there && sl < A.k) {
            *gate_at = held ? gate : 0.0f;
            if (!A.replay) rp_store_route(route_at, A.route_bytes, 0, held ? (int)e : -1);
        }
        __syncwarp();
    }
    // Runs that end in the same group meet here: their counts, then in the same place their sums of p.
    if (!want_counts) return;
    if (sl == 0) last[sub] = g >= 0 && g < A.G ? g : -1;
    __syncthreads();
    meet<NSUB, EP>(A, last, [&](int u, int e) { return cnt[u][e]; }, [&](int gu, int e, int c) { if (c) atomicAdd(&A.counts[(i64)gu * A.E + e], c); });
    if (!want_loss) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VPL; ++i) cnt[sub][e0 + i] = __float_as_int(acc[i]);
    __syncthreads();
    meet<NSUB, EP>(A, last, [&](int u, int e) { return __int_as_float(cnt[u][e]); }, [&](int gu, int e, float f) { add_sums<1>(A, gu, e, &f); });
    if (A.finish == 2) return;
    __threadfence();
    __syncthreads();
    if (A.finish == 1) {
        if (threadIdx.x == 0) turn = atomicAdd(&A.space->ticket, 1u);
        __syncthreads();
        if (turn != gridDim.x - 1) return;
        __threadfence();
    }
    const double loss = groups_loss(A, 0, ROUTE_WARPS, part);
    if (threadIdx.x == 0) *A.loss = __ldcg(&A.space->odd) ? NAN : (float)loss;
}

// The loss where there are many groups: CTAs add up groups of their own, the last one adds up the CTAs.
__global__ void __launch_bounds__(ROUTE_THREADS) k_route_loss(RouteArgs A)
{
    __shared__ double part[ROUTE_WARPS];
    const double mine = groups_loss(A, blockIdx.x * ROUTE_WARPS, gridDim.x * ROUTE_WARPS, part);
    if (threadIdx.x) return;
    A.space->part[blockIdx.x] = mine;
    __threadfence();
    if (atomicAdd(&A.space->loss_ticket, 1u) != gridDim.x - 1) return;
    __threadfence();
    double sum = 0.0;
    for (int b = 0; b < (int)gridDim.x; ++b) sum += __ldcg(&A.space->part[b]);
    *A.loss = __ldcg(&A.space->odd) ? NAN : (float)sum;
}

// Gradient for the logits.  With b[e] = loss_grad * coef / G * E * counts[g][e] / (k T_g^2), a_j = scale * gates_grad_j and y_j = s_j / sum of the chosen:
//   softmax: dx = p (b - sum p b) + at the chosen: y_j (a_j - sum y a), or, not normalised, p (b - sum p b - sum_j p_j a_j) + p_j a_j
//   sigmoid: ds = (b - sum p b) / sum s + at the chosen: (a_j - sum y a) / sum of the chosen, or a_j;  dx = s (1 - s) ds
// The token's row is put together in shared memory, where the lanes that have its chosen experts each add their part; an expert that a token has twice gets its
// parts one after the other.
template <typename X, int VPL, int SUB>
__global__ void __launch_bounds__(ROUTE_THREADS, VPL == 8 ? 4 : 1) k_route_grad(RouteArgs A)
{
    constexpr int NSUB = ROUTE_THREADS / SUB, EP = VPL * SUB;
    __shared__ __align__(16) float rows[NSUB][EP];
    __shared__ unsigned char tags[NSUB][EP];
    const int sub = threadIdx.x / SUB, sl = threadIdx.x % SUB, e0 = sl * VPL, first_lane = (threadIdx.x & 31) - sl;
    const bool soft = A.score == RP_SCORE_SOFTMAX, gates = A.gates_grad != nullptr;
    const float loss_grad = A.loss_grad ? *A.loss_grad : 0.0f;
    const i64 t0 = ((i64)blockIdx.x * NSUB + sub) * A.run;
    const int run = (int)A.run, n = (int)max(min(A.T - t0, A.run), (i64)0);
    int g = -2, k_lanes = 1, next = INT_MIN;               // (tokens of the run are counted from 0)
    while (k_lanes < A.k) k_lanes <<= 1;
    float b[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) b[i] = 0.0f;
    const X *x_at = (const X *)A.x + t0 * A.row;
    X *out = (X *)A.dx + t0 * A.dx_row;
    const char *route_at = (const char *)A.routes + (t0 * A.route_row + sl) * A.route_bytes;
    const float *gate_at = A.gates_grad + t0 * A.k + sl;
    const i64 route_step = A.route_row * A.route_bytes;
    Row<X, VPL> row;
    // lane j of the token's has its j-th choice
    i64 e_next = -1;
    float a_next = 0.0f;
    auto fetch = [&](const X *x) {
        load_row<X, VPL>(A, x + e0, e0, row);
        if (gates && sl < A.k) { e_next = rp_load_route(route_at, A.route_bytes, 0); a_next = *gate_at; }
        route_at += route_step;
        gate_at += A.k;
    };
    if (n > 0) fetch(x_at);
    for (int step = 0; step < run; ++step, x_at += A.row, out += A.dx_row) {
        const bool there = step < n;
        if (there && step >= next) {
            g = rp_sample_of(A.start, A.G, t0 + step);
            next = g < A.G ? (int)min(A.start[g + 1] - t0, (i64)INT_MAX) : INT_MAX;
            if (A.loss_grad && g >= 0 && g < A.G) {
                const i64 lo = max(A.start[g], (i64)0), hi = min(A.start[g + 1], A.T);
                const float m = (float)(hi - lo), f = loss_grad * (A.coef / A.G) * A.E / A.k / m / m;
#pragma unroll
                for (int i = 0; i < VPL; ++i) b[i] = e0 + i < A.E ? f * (float)A.counts_in[(i64)g * A.E + e0 + i] : 0.0f;
            }
        }
        const bool held = there && g >= 0 && g < A.G;
        float x[VPL], s[VPL], top, inv;
        open_row<X, VPL>(row, x);
        const bool valid = gates && held && sl < A.k && e_next >= 0 && e_next < A.E;
        const int e = valid ? (int)e_next : -1;
        const float a = A.scale * a_next, xe = valid ? rp_float(x_at[e]) : 0.0f;
        if (step + 1 < n) fetch(x_at + A.row);
        scores<VPL, SUB, false>(A, x, s, top, inv);
        float pb = 0.0f;
        if (A.loss_grad) {
#pragma unroll
            for (int i = 0; i < VPL; ++i) pb = fmaf(s[i], b[i], pb);
            pb = sub_sum<SUB>(pb) * inv;
        }
        float add = 0.0f;
        bool tiny = false;
        if (gates) {
            const float v = valid ? score_of(A, xe, top, inv) : 0.0f;
            float z = v, za = valid ? v * a : 0.0f;
            for (int o = 1; o < k_lanes; o <<= 1) { z += __shfl_xor_sync(0xffffffffu, z, o); za += __shfl_xor_sync(0xffffffffu, za, o); }
            // (lanes behind the choices have their own sums: what all lanes need is the first's)
            const float zi = z < SHARES_FROM ? 0.0f : reciprocal(z), ds = soft ? v : v * (1.0f - v);
            add = A.normalise ? (a - za * zi) * (zi * ds) : a * ds;       // (zi may be large: the score is multiplied with it first)
            tiny = A.normalise && z < SHARES_FROM;
            if (soft && !A.normalise) pb += __shfl_sync(0xffffffffu, za, first_lane);
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const float p = s[i] * inv;
            s[i] = (b[i] - pb) * (soft ? p : p * (1.0f - s[i]));
        }
#pragma unroll
        for (int i = 0; i < VPL; i += 4) *(float4 *)&rows[sub][e0 + i] = make_float4(s[i], s[i + 1], s[i + 2], s[i + 3]);
        __syncwarp();
        if (gates) {
            // (does an expert come twice? its tag is then another lane's)
            if (valid) tags[sub][e] = (unsigned char)sl;
            __syncwarp();
            if (!__any_sync(0xffffffffu, valid && (tiny || tags[sub][e] != sl))) {
                if (valid) rows[sub][e] += add;
            } else {
                const float y = shares(valid, xe, k_lanes);
                float ya = valid ? y * a : 0.0f;
                for (int o = 1; o < k_lanes; o <<= 1) ya += __shfl_xor_sync(0xffffffffu, ya, o);
                if (tiny) add = (a - ya) * y;
                for (int j = 0; j < A.k; ++j) {
                    if (sl == j && valid) rows[sub][e] += add;
                    __syncwarp();
                }
            }
            __syncwarp();
        }
        if (there) {
#pragma unroll
            for (int c = 0; c < VPL; c += 8) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const float4 v = *(const float4 *)&rows[sub][e0 + c + i];
                    f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
                }
                if (!held) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = 0.0f;
                }
                if (A.wide) {
                    if (e0 + c < A.E) rp_store8(out + e0 + c, rp_close8<X>(f));
                } else
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (e0 + c + i < A.E) out[e0 + c + i] = rp_round<X>(f[i]);
            }
        }
        __syncwarp();
    }
}

// ---------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------
// A lane holds 8 experts (more where a row of E needs more than a warp), so SUB lanes a token; never fewer lanes than choices.  One CTA alone, which clears its own
// counts: 16 tokens of 256 experts 8.6 us (two launches: 11.6), 64 tokens of 64 experts 9.0 (12.5); from 8 tokens a group of lanes on it is slower.
template <typename X, int VPL, int SUB>
static int launch(RouteArgs &A, bool grad, int sms, cudaStream_t stream)
{
    constexpr int NSUB = ROUTE_THREADS / SUB;
    if (grad) {
        const i64 subs = std::min((A.T + 1) / 2, (i64)sms * 4 * NSUB);
        A.run = (A.T + subs - 1) / subs;
        k_route_grad<X, VPL, SUB><<<(unsigned)((A.T + A.run * NSUB - 1) / (A.run * NSUB)), ROUTE_THREADS, 0, stream>>>(A);
        return rp_op_launched();
    }
    const i64 cells = (i64)A.G * A.E;
    if (A.T <= (i64)NSUB * 4 && cells <= 4096) {         // up to four tokens a group of lanes: one CTA, one launch
        A.finish = 0;
        A.run = (A.T + NSUB - 1) / NSUB;
    } else {
        const i64 subs = std::min((A.T + 3) / 4, (i64)sms * 4 * NSUB);
        A.finish = A.G <= 16 ? 1 : 2;                    // (a warp of the last CTA takes 2 us a group; the launch costs 2 us)
        A.run = (A.T + subs - 1) / subs;
        if (A.counts) {
            k_route_clear<<<(unsigned)std::min((cells + 2 * ROUTE_THREADS - 1) / (2 * ROUTE_THREADS), (i64)sms * 4), ROUTE_THREADS, 0, stream>>>(A);
            RP_TRY(rp_op_launched());
        }
    }
    cudaLaunchConfig_t how = {};                         // (starts beside the clearing)
    how.gridDim = dim3((unsigned)((A.T + A.run * NSUB - 1) / (A.run * NSUB)));
    how.blockDim = dim3(ROUTE_THREADS);
    how.stream = stream;
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    how.attrs = &early; how.numAttrs = A.finish && A.counts ? 1 : 0;
    RP_CUDA(cudaLaunchKernelEx(&how, k_route<X, VPL, SUB>, (RouteArgs)A));
    RP_TRY(rp_op_launched());
    if (A.loss && A.finish == 2) {
        k_route_loss<<<std::min(ROUTE_LOSS_CTAS, (A.G + ROUTE_WARPS - 1) / ROUTE_WARPS), ROUTE_THREADS, 0, stream>>>(A);
        RP_TRY(rp_op_launched());
    }
    return RP_OK;
}
template <typename X>
static int launch_for(RouteArgs &A, bool grad, int sms, cudaStream_t stream)
{
    const int lanes = std::max((A.E + 7) / 8, A.k);
    if (lanes <= 2) return launch<X, 8, 2>(A, grad, sms, stream);
    if (lanes <= 4) return launch<X, 8, 4>(A, grad, sms, stream);
    if (lanes <= 8) return launch<X, 8, 8>(A, grad, sms, stream);
    if (lanes <= 16) return launch<X, 8, 16>(A, grad, sms, stream);
    if (lanes <= 32) return launch<X, 8, 32>(A, grad, sms, stream);
    if (A.E <= 512) return launch<X, 16, 32>(A, grad, sms, stream);
    return launch<X, 32, 32>(A, grad, sms, stream);
}

static int check_router(const rp_router *r, const void *logits, i64 T, const void *start, int G, int route_bytes)
{
    if (!r || !logits || !start || T < 0 || G < 1) return RP_ERR_ARG;
    if (r->n_experts < 1 || r->top_k < 1 || r->top_k > r->n_experts || r->type < RP_F32 || r->type > RP_BF16 ||
        r->score < RP_SCORE_SOFTMAX || r->score > RP_SCORE_SIGMOID || r->normalise < 0 || r->normalise > 1)
        return RP_ERR_ARG;
    if (route_bytes != 1 && route_bytes != 2 && route_bytes != 4 && route_bytes != 8) return RP_ERR_ARG;
    if (r->n_experts > 1024 || r->top_k > ROUTE_MAX_K || T > (1ll << 26) || T * r->top_k >= (1ll << 31) || (i64)G * r->n_experts >= (1ll << 31))
        return RP_ERR_RANGE;
    if (!rp_aligned(logits, rp_type_bytes(r->type)) || !rp_aligned(start, 8)) return RP_ERR_ARG;
    return RP_OK;
}
static bool wide_rows(const void *p, i64 row, int E, int bytes) { return E % 8 == 0 && rp_aligned(p, 16) && row * bytes % 16 == 0; }

extern "C" int64_t rp_route_workspace(const rp_router *r, int32_t n_groups)
{
    if (!r || r->n_experts < 1 || n_groups < 1) return 0;
    return (int64_t)sizeof(RouteSpace) + (int64_t)sizeof(u64) * n_groups * r->n_experts;
}

static RouteArgs router_args(const rp_router *r, const void *logits, i64 row, i64 T, const int64_t *start, int G, const void *routes, int bytes, i64 route_row)
{
    RouteArgs A = {};
    A.x = logits; A.row = row; A.T = T; A.E = r->n_experts; A.k = r->top_k; A.score = r->score; A.normalise = r->normalise;
    A.G = G; A.scale = r->scale; A.coef = r->loss_coef; A.start = (const i64 *)start;
    A.routes = (void *)routes; A.route_bytes = bytes; A.route_row = route_row;
    A.wide = wide_rows(logits, row, r->n_experts, rp_type_bytes(r->type));
    return A;
}

extern "C" int rp_route(const rp_router *r, const void *logits, int64_t row_stride, int64_t n_tokens, const float *choice_bias,
                        const int64_t *start, int32_t n_groups, int32_t replay, void *routes, int32_t route_bytes, int64_t route_stride,
                        float *gates, int32_t *counts, float *loss, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    RP_TRY(check_router(r, logits, n_tokens, start, n_groups, route_bytes));
    if (!routes || !gates || (loss && (!counts || !workspace)) || replay < 0 || replay > 1) return RP_ERR_ARG;
    if (loss && (workspace_bytes < rp_route_workspace(r, n_groups) || !rp_aligned(workspace, 16))) return RP_ERR_ARG;
    if (!rp_aligned(routes, route_bytes) || !rp_aligned(gates, 4) || !rp_aligned(counts, 4) || !rp_aligned(loss, 4) || !rp_aligned(choice_bias, 4))
        return RP_ERR_ARG;
    if (!replay && route_stride < r->top_k && n_tokens > 1) return RP_ERR_ARG;         // rows would write over one another
    if (!replay && route_bytes == 1 && r->n_experts > 256) return RP_ERR_RANGE;
    RpOpDevice dev;
    RP_TRY(rp_op_enter(dev, logits, choice_bias, start, routes, gates, counts, loss, workspace));
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    RouteArgs A = router_args(r, logits, row_stride, n_tokens, start, n_groups, routes, route_bytes, route_stride);
    A.replay = replay; A.bias = choice_bias; A.gates = gates; A.counts = counts;
    A.space = (RouteSpace *)workspace; A.sums = loss ? (u64 *)(A.space + 1) : nullptr; A.loss = loss;
    if (n_tokens == 0) {
        if (counts) RP_CUDA(cudaMemsetAsync(counts, 0, sizeof(int) * (size_t)n_groups * r->n_experts, stream));
        if (loss) RP_CUDA(cudaMemsetAsync(loss, 0, sizeof(float), stream));
        return RP_OK;
    }
    int st = RP_OK;
    RP_FOR_TYPE(r->type, st = launch_for<X>(A, false, rp_op_sms(dev.device), stream));
    return st;
}

extern "C" int rp_route_grad(const rp_router *r, const void *logits, int64_t row_stride, int64_t n_tokens, const void *routes, int32_t route_bytes,
                             int64_t route_stride, const float *gates_grad, const float *loss_grad, const int64_t *start, int32_t n_groups,
                             const int32_t *counts, void *logits_grad, int64_t grad_stride, void *cuda_stream)
{
    RP_TRY(check_router(r, logits, n_tokens, start, n_groups, route_bytes));
    if (!logits_grad || (gates_grad && !routes) || (loss_grad && !counts) || logits_grad == logits) return RP_ERR_ARG;
    if (!rp_aligned(routes, route_bytes) || !rp_aligned(gates_grad, 4) || !rp_aligned(loss_grad, 4) || !rp_aligned(counts, 4) ||
        !rp_aligned(logits_grad, rp_type_bytes(r->type)))
        return RP_ERR_ARG;
    if (grad_stride < r->n_experts && n_tokens > 1) return RP_ERR_ARG;
    RpOpDevice dev;
    RP_TRY(rp_op_enter(dev, logits, routes, gates_grad, loss_grad, start, counts, logits_grad));
    if (n_tokens == 0) return RP_OK;
    RouteArgs A = router_args(r, logits, row_stride, n_tokens, start, n_groups, routes, route_bytes, route_stride);
    A.gates_grad = gates_grad; A.loss_grad = loss_grad; A.counts_in = counts; A.dx = logits_grad; A.dx_row = grad_stride;
    A.wide = A.wide && wide_rows(logits_grad, grad_stride, r->n_experts, rp_type_bytes(r->type));
    int st = RP_OK;
    RP_FOR_TYPE(r->type, st = launch_for<X>(A, true, rp_op_sms(dev.device), (cudaStream_t)cuda_stream));
    return st;
}
