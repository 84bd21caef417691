// Norm of every head and rotation by position for the queries and keys of packed rows, and the gradient.
//
//   y = turn(x * rsqrt(mean x^2 + eps) * w, angle = position * inv_freq)
//   gradient: u = turn back(dy), dw = sum u xhat, dx = r (w u - xhat mean(w u xhat)), xhat = x r
//
// Bound by HBM bandwidth: T * heads * head_dim elements read and written once (two reads in the gradient).  Positions are counted from the start of a
// token's sample; the angle is reduced to a part of a turn in 64 bits (a place of 10^6 in the context leaves 32 bits an error of 0.06) and its sine
// and cosine are worked out once a token, for all heads of queries and keys.
#include <algorithm>

#include "rp_ops.cuh"

#define ROT_WARPS 8
#define ROT_THREADS (32 * ROT_WARPS)
#define ROT_MAX_DIM 1024

struct RotTensor {
    const void *x;
    i64 x_token, x_head;
    void *y;
    i64 y_token, y_head;
    const void *w;
    const void *dy;
    i64 g_token, g_head;
    float *dw;
    int heads;
};
struct RotArgs {
    RotTensor h[2];         // queries, keys
    int d, r, half, w32;    // head_dim, rotary_dim, half layout, weights in 32 bits
    float eps, mscale, inv_d;               // inv_d: 1 / head_dim
    i64 T, run;             // run: tokens of a warp (k_rotate_any)
    int parts;              // a token's heads are dealt out to this many warps
    const double *freq;
    const i64 *start, *first;
    int N;
    float *part;            // gradient: [CTAs][2][d] partial sums of the weights' gradients
};

// Cosine and sine (times mscale) of one pair at a position.
__device__ __forceinline__ float2 turn_of(const RotArgs &A, i64 position, int pair)
{
    const double turns = (double)position * (__ldg(A.freq + pair) * 0.15915494309189533577);      // / 2 pi
    float sn, cs;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
    return make_float2(cs * A.mscale, sn * A.mscale);
}

// Where a run of tokens is: its sample's end, and what a token's index lacks to its position.
struct Place {
    i64 next, base;
    bool held;
    __device__ __forceinline__ void find(const RotArgs &A, i64 t)
    {
        const int i = rp_sample_of(A.start, A.N, t);
        held = i >= 0 && i < A.N;
        next = i < A.N ? __ldg(A.start + i + 1) : INT64_MAX;
        base = held ? (A.first ? __ldg(A.first + i) : 0) - __ldg(A.start + i) : 0;
    }
};

template <typename X> __device__ __forceinline__ float weight_at(const RotArgs &A, const void *w, int i)
{
    return A.w32 ? ((const float *)w)[i] : rp_float(((const X *)w)[i]);
}

// Any head size and alignment: a warp takes one head after the other, a lane the pairs lane, lane + 32, .. and then the elements behind them.  Elements are read one by one,
// once for the norm and again for each pass behind it, and one head at a time is on its way: 16384 tokens of 32 + 8 heads of 72 take 310 us (gradient 511), of 128 in
// pieces 71 (122).
// GRAD: y receives the gradient of x.
template <typename X, bool GRAD>
__global__ void __launch_bounds__(ROT_THREADS) k_rotate_any(RotArgs A)
{
    extern __shared__ float2 table[];                    // [warps][r / 2], then (GRAD) the CTA's weight gradients [warps][2][d]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pairs = A.r / 2, rest = A.d - A.r;
    float2 *cs = table + warp * pairs;
    float *dw = (float *)(table + ROT_WARPS * pairs) + warp * 2 * A.d;
    if (GRAD && A.part)
        for (int i = lane; i < 2 * A.d; i += 32) dw[i] = 0.0f;
    __syncwarp();
    const i64 unit = (i64)blockIdx.x * ROT_WARPS + warp;
    const i64 t0 = unit / A.parts * A.run;
    const int share = (int)(unit % A.parts), all = A.h[0].heads + A.h[1].heads;
    Place at;
    at.next = INT64_MIN;
    for (i64 t = t0; t < min(A.T, t0 + A.run); ++t) {
        if (t >= at.next) at.find(A, t);
        __syncwarp();
        for (int p = lane; p < pairs; p += 32) cs[p] = turn_of(A, t + at.base, p);
        __syncwarp();
        for (int hd = share; hd < all; hd += A.parts) {
            const int which = hd >= A.h[0].heads;
            const RotTensor &H = A.h[which];
            const int head = which ? hd - A.h[0].heads : hd;
            const X *x = (const X *)H.x + t * H.x_token + head * H.x_head;
            X *y = (X *)H.y + t * H.y_token + head * H.y_head;
            if (!at.held) {
                for (int i = lane; i < A.d; i += 32) y[i] = rp_round<X>(0.0f);
                continue;
            }
            float r = 1.0f;
            if (H.w) {
                float sum = 0.0f;
                for (int i = lane; i < A.d; i += 32) { const float v = rp_float(x[i]); sum = fmaf(v, v, sum); }
#pragma unroll
                for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                r = 1.0f / sqrtf(sum / A.d + A.eps);
            }
            if (!GRAD) {
                for (int p = lane; p < pairs + rest; p += 32) {
                    const bool turned = p < pairs;
                    const int i = !turned ? A.r + p - pairs : A.half ? p : 2 * p, i2 = A.half ? p + pairs : 2 * p + 1;
                    float a = rp_float(x[i]), b = turned ? rp_float(x[i2]) : 0.0f;
                    if (H.w) { a *= r * weight_at<X>(A, H.w, i); if (turned) b *= r * weight_at<X>(A, H.w, i2); }
                    if (turned) {
                        y[i] = rp_round<X>(a * cs[p].x - b * cs[p].y);
                        y[i2] = rp_round<X>(a * cs[p].y + b * cs[p].x);
                    } else
                        y[i] = rp_round<X>(a);
                }
            } else {
                const X *g = (const X *)H.dy + t * H.g_token + head * H.g_head;
                float dot = 0.0f;
                if (H.w) {
                    for (int p = lane; p < pairs + rest; p += 32) {
                        const bool turned = p < pairs;
                        const int i = !turned ? A.r + p - pairs : A.half ? p : 2 * p, i2 = A.half ? p + pairs : 2 * p + 1;
                        const float ga = rp_float(g[i]), gb = turned ? rp_float(g[i2]) : 0.0f;
                        const float u = turned ? ga * cs[p].x + gb * cs[p].y : ga;
                        const float xa = rp_float(x[i]) * r;
                        dot = fmaf(u * weight_at<X>(A, H.w, i), xa, dot);
                        if (A.part) dw[which * A.d + i] += u * xa;
                        if (turned) {
                            const float u2 = gb * cs[p].x - ga * cs[p].y, xb = rp_float(x[i2]) * r;
                            dot = fmaf(u2 * weight_at<X>(A, H.w, i2), xb, dot);
                            if (A.part) dw[which * A.d + i2] += u2 * xb;
                        }
                    }
#pragma unroll
                    for (int o = 16; o; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
                    dot /= A.d;
                }
                for (int p = lane; p < pairs + rest; p += 32) {
                    const bool turned = p < pairs;
                    const int i = !turned ? A.r + p - pairs : A.half ? p : 2 * p, i2 = A.half ? p + pairs : 2 * p + 1;
                    const float ga = rp_float(g[i]), gb = turned ? rp_float(g[i2]) : 0.0f;
                    float u = turned ? ga * cs[p].x + gb * cs[p].y : ga, u2 = turned ? gb * cs[p].x - ga * cs[p].y : 0.0f;
                    if (H.w) {
                        u = r * (u * weight_at<X>(A, H.w, i) - rp_float(x[i]) * r * dot);
                        if (turned) u2 = r * (u2 * weight_at<X>(A, H.w, i2) - rp_float(x[i2]) * r * dot);
                    }
                    y[i] = rp_round<X>(u);
                    if (turned) y[i2] = rp_round<X>(u2);
                }
            }
        }
    }
    if (GRAD && A.part) {
        __syncthreads();
        const float *from = (const float *)(table + ROT_WARPS * pairs);
        for (int i = threadIdx.x; i < 2 * A.d; i += ROT_THREADS) {
            float sum = 0.0f;
            for (int w = 0; w < ROT_WARPS; ++w) sum += from[w * 2 * A.d + i];
            A.part[(i64)blockIdx.x * 2 * A.d + i] = sum;
        }
    }
}

// Heads of whole 16-byte pieces.  A head belongs to TPH neighbouring lanes of a warp with two pieces of eight elements each: those that are turned into one another
// (half layout) or neighbours, so that a lane has all pairs that it needs and the mean of squares is a few shuffles.  A warp takes ROT_CHUNK tokens at a time:
// their sines and cosines go to shared memory once, for all heads; then it goes through the heads of the queries, then of the keys, with a token's factors (and the
// sums for the weights' gradients) in registers.  The loads of two steps are issued before either is worked on.
// 32768 tokens of 32 + 8 heads of 128 in bf16 129 us, 81 % of the measured copy rate; the gradient of 16411 with half of each head turned 114 us, 69 % (128 registers,
// 16 warps an SM): it waits for memory.  All forms keep some registers in local memory: 12 to 60 bytes a thread forward in 16 bits (52 for these rows), 28 to 124
// backward, 76 to 128 in 32 bits.  Tried: a third step in flight (more of that, 300 us for 131), rows through shared memory by asynchronous copies (136 to 150), rows
// asked into L2 ahead (147).
// Element i of a lane's 16 in the order of its registers: the first of each pair (0 to 7), then the second.
template <bool INTERLEAVED> __device__ __forceinline__ int place(int pa, int pb, int i)
{
    if (!INTERLEAVED) return i < 8 ? pa + i : pb + i - 8;
    const int pair = i & 7;
    return (pair < 4 ? pa + 2 * pair : pb + 2 * pair - 8) + (i >> 3);
}
template <typename X, bool INTERLEAVED> __device__ __forceinline__ void open_pairs(const Pack8<X> &p, const Pack8<X> &q, f2 *a, f2 *b)
{
    float x[8], y[8];
    rp_open8(p, x); rp_open8(q, y);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (!INTERLEAVED) { a[i] = rp_f2(x[2 * i], x[2 * i + 1]); b[i] = rp_f2(y[2 * i], y[2 * i + 1]); }
        else {
            const float *z = i < 2 ? x + 4 * i : y + 4 * i - 8;
            a[i] = rp_f2(z[0], z[2]); b[i] = rp_f2(z[1], z[3]);
        }
    }
}
template <typename X, bool INTERLEAVED> __device__ __forceinline__ void close_pairs(const f2 *a, const f2 *b, Pack8<X> &p, Pack8<X> &q)
{
    float x[8], y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (!INTERLEAVED) { rp_parts(a[i], x[2 * i], x[2 * i + 1]); rp_parts(b[i], y[2 * i], y[2 * i + 1]); }
        else {
            float *z = i < 2 ? x + 4 * i : y + 4 * i - 8;
            rp_parts(a[i], z[0], z[2]); rp_parts(b[i], z[1], z[3]);
        }
    }
    p = rp_close8<X>(x); q = rp_close8<X>(y);
}
// Turns pairs, or turns them back: the lane's first two of each piece where that piece is turned at all (0 times what an element behind rotary_dim holds may be NaN).
template <bool BACK> __device__ __forceinline__ void turn_piece(f2 *a, f2 *b, const f2 *c, const f2 *s)
{
    const f2 minus = rp_f2(-1.0f, -1.0f);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const f2 x = a[p], n = rp_mul(s[p], minus);
        a[p] = rp_fma(x, c[p], rp_mul(b[p], BACK ? s[p] : n));
        b[p] = rp_fma(b[p], c[p], rp_mul(x, BACK ? n : s[p]));
    }
}
template <bool BACK> __device__ __forceinline__ void turn(f2 *a, f2 *b, const f2 *c, const f2 *s, bool first, bool second)
{
    if (first) turn_piece<BACK>(a, b, c, s);
    if (second) turn_piece<BACK>(a + 2, b + 2, c + 2, s + 2);
}
// Sum over the lanes of a head.
template <int TPH> __device__ __forceinline__ float head_sum(f2 v)
{
    float x, y;
    rp_parts(v, x, y);
    x += y;
#pragma unroll
    for (int o = 1; o < TPH; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
#define ROT_CHUNK 4
#define ROT_CTAS(GRAD) ((GRAD) ? 2 : 3)                  // resident on an SM
template <typename X, int TPH, bool INTERLEAVED, bool GRAD>
__global__ void __launch_bounds__(ROT_THREADS, ROT_CTAS(GRAD)) k_rotate_rows(RotArgs A)
{
    constexpr int NG = 32 / TPH, STEPS = 2;              // heads of a warp at a time; how many of them in flight
    constexpr int ROW = 8 * TPH;                         // pairs of a token in the table; those that are not turned have an angle of 0
    extern __shared__ __align__(16) float2 table[];      // [warps][ROT_CHUNK][ROW], weights [2][16 TPH] in 32 bits, (GRAD) their gradients [warps][2][d]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pairs = A.r / 2, j = lane % TPH, group = lane / TPH;
    float2 *cs = table + warp * ROT_CHUNK * ROW;
    float *weights = (float *)(table + ROT_WARPS * ROT_CHUNK * ROW), *dw = weights + 2 * 16 * TPH + warp * 2 * A.d;
    const bool mine = 16 * j < A.d;
    const int turned = A.r / 16;                         // half layout: pieces of a half
    const int pa = INTERLEAVED ? 16 * j : j < turned ? 8 * j : A.r + 16 * (j - turned);          // first elements of the lane's pieces
    const int pb = INTERLEAVED || j >= turned ? pa + 8 : pa + A.r / 2;
    const bool turns_a = INTERLEAVED ? 16 * j < A.r : j < turned, turns_b = INTERLEAVED ? 16 * j + 8 < A.r : j < turned;
    if (GRAD && A.part)
        for (int i = lane; i < 2 * A.d; i += 32) dw[i] = 0.0f;
    if (warp < 2 && group == 0) {
        const RotTensor &H = A.h[warp];                  // two of each lane side by side, lane after lane
        for (int i = 0; i < 16; ++i)
            weights[warp * 16 * TPH + (i >> 1) * 2 * TPH + 2 * j + (i & 1)] = H.w && mine ? weight_at<X>(A, H.w, place<INTERLEAVED>(pa, pb, i)) : 1.0f;
    }
    __syncthreads();
    const int unit = blockIdx.x * ROT_WARPS + warp, lanes = gridDim.x * ROT_WARPS / A.parts, share = unit % A.parts;
    // tokens unit / parts, + lanes, + 2 lanes ..: at any time the warps read neighbouring tokens
    Place at;
    at.next = INT64_MIN;
    for (i64 c0 = unit / A.parts; c0 < (unit / A.parts < lanes ? A.T : 0); c0 += (i64)ROT_CHUNK * lanes) {
        const int n = (int)min((i64)ROT_CHUNK, (A.T - c0 + lanes - 1) / lanes);
        u32 held = 0;
        __syncwarp();
        for (int i = 0; i < n; ++i) {
            const i64 t = c0 + (i64)i * lanes;
            if (t >= at.next) at.find(A, t);
            held |= (at.held ? 1u : 0u) << i;
            for (int p = lane; p < ROW; p += 32) {
                // two cosines and two sines of a lane side by side, lane after lane: no two of a load's lanes in one bank
                const float2 v = p < pairs ? turn_of(A, t + at.base, p) : make_float2(1.0f, 0.0f);
                float *to = (float *)(cs + i * ROW + ((p & 7) >> 1) * 2 * TPH + (p >> 3) * 2) + (p & 1);
                to[0] = v.x; to[2] = v.y;
            }
        }
        __syncwarp();
        int before = 0;                                  // steps of the tensor before
        for (int which = 0; which < 2; ++which) {
            const RotTensor &H = A.h[which];
            const int steps = (H.heads + NG - 1) / NG;
            // a step's warp goes by its number in both tensors
            const int first = A.parts == 1 ? 0 : ((share - before) % A.parts + A.parts) % A.parts;
            before += steps;
            if (first >= steps) continue;
            const bool norm = H.w != nullptr;
            const int head0 = first * NG + group, head_step = A.parts * NG;
            const i64 x_step = head_step * H.x_head, g_step = GRAD ? head_step * H.g_head : 0, y_step = head_step * H.y_head;
            const f2 *w = (const f2 *)(weights + which * 16 * TPH) + j;
            f2 da[4], db[4];
            if (GRAD) {
#pragma unroll
                for (int p = 0; p < 4; ++p) { da[p] = rp_f2(0.0f, 0.0f); db[p] = da[p]; }
            }
            for (int i = 0; i < n; ++i) {
                const i64 t = c0 + (i64)i * lanes;
                f2 c[4], s[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const ulonglong2 v = *(const ulonglong2 *)(cs + i * ROW + p * 2 * TPH + 2 * j);
                    c[p].v = v.x; s[p].v = v.y;
                }
                const bool there = held >> i & 1;
                const X *x = (const X *)H.x + t * H.x_token + head0 * H.x_head, *g = GRAD ? (const X *)H.dy + t * H.g_token + head0 * H.g_head : nullptr;
                X *y = (X *)H.y + t * H.y_token + head0 * H.y_head;
                for (int st = first, head = head0; st < steps; st += A.parts * STEPS) {
                    Pack8<X> xa[STEPS], xb[STEPS], ga[STEPS], gb[STEPS];
                    bool ok[STEPS];
#pragma unroll
                    for (int u = 0; u < STEPS; ++u) {
                        ok[u] = mine && head < H.heads;
                        xa[u] = Pack8<X>(); xb[u] = Pack8<X>(); ga[u] = Pack8<X>(); gb[u] = Pack8<X>();
                        if (ok[u] && there) {
                            if (!GRAD || norm) { xa[u] = rp_load8(x + pa); xb[u] = rp_load8(x + pb); }
                            if (GRAD) { ga[u] = rp_load8(g + pa); gb[u] = rp_load8(g + pb); }
                        }
                        head += head_step;
                        x += x_step;
                        if (GRAD) g += g_step;
                    }
#pragma unroll
                    for (int u = 0; u < STEPS; ++u) {
                        f2 a[4], b[4];
                        open_pairs<X, INTERLEAVED>(xa[u], xb[u], a, b);
                        f2 r = rp_f2(1.0f, 1.0f);
                        if (norm) {
                            f2 sum2 = rp_f2(0.0f, 0.0f);
#pragma unroll
                            for (int p = 0; p < 4; ++p) sum2 = rp_fma(a[p], a[p], rp_fma(b[p], b[p], sum2));
                            const float sum = head_sum<TPH>(sum2), q = ok[u] && there ? rsqrtf(fmaf(sum, A.inv_d, A.eps)) : 0.0f;       // (eps may be 0)
                            r = rp_f2(q, q);
                        }
                        if (!GRAD) {
                            if (norm)
#pragma unroll
                                for (int p = 0; p < 4; ++p) { a[p] = rp_mul(a[p], rp_mul(r, w[p * TPH])); b[p] = rp_mul(b[p], rp_mul(r, w[(p + 4) * TPH])); }
                            turn<false>(a, b, c, s, turns_a, turns_b);
                        } else {
                            f2 g2[4], h2[4];
                            open_pairs<X, INTERLEAVED>(ga[u], gb[u], g2, h2);
                            turn<true>(g2, h2, c, s, turns_a, turns_b);
                            if (norm) {
                                f2 dot2 = rp_f2(0.0f, 0.0f);
#pragma unroll
                                for (int p = 0; p < 4; ++p) {
                                    a[p] = rp_mul(a[p], r); b[p] = rp_mul(b[p], r);
                                    da[p] = rp_fma(g2[p], a[p], da[p]); db[p] = rp_fma(h2[p], b[p], db[p]);
                                    g2[p] = rp_mul(g2[p], w[p * TPH]); h2[p] = rp_mul(h2[p], w[(p + 4) * TPH]);
                                    dot2 = rp_fma(g2[p], a[p], rp_fma(h2[p], b[p], dot2));
                                }
                                const float dot = -head_sum<TPH>(dot2) * A.inv_d;
                                const f2 d2 = rp_f2(dot, dot);
#pragma unroll
                                for (int p = 0; p < 4; ++p) { g2[p] = rp_mul(r, rp_fma(a[p], d2, g2[p])); h2[p] = rp_mul(r, rp_fma(b[p], d2, h2[p])); }
                            }
#pragma unroll
                            for (int p = 0; p < 4; ++p) { a[p] = g2[p]; b[p] = h2[p]; }
                        }
                        if (!there) {
#pragma unroll
                            for (int p = 0; p < 4; ++p) { a[p] = rp_f2(0.0f, 0.0f); b[p] = a[p]; }
                        }
                        if (ok[u]) {
                            Pack8<X> oa, ob;
                            close_pairs<X, INTERLEAVED>(a, b, oa, ob);
                            rp_store8(y + pa, oa);
                            rp_store8(y + pb, ob);
                        }
                        y += y_step;
                    }
                }
            }
            if (GRAD && norm && A.part) {
#pragma unroll
                for (int p = 0; p < 4; ++p)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        float v[2];
                        rp_parts(q ? db[p] : da[p], v[0], v[1]);
#pragma unroll
                        for (int o = TPH; o < 32; o <<= 1) { v[0] += __shfl_xor_sync(0xffffffffu, v[0], o); v[1] += __shfl_xor_sync(0xffffffffu, v[1], o); }
                        const int e0 = place<INTERLEAVED>(pa, pb, 8 * q + 2 * p), e1 = place<INTERLEAVED>(pa, pb, 8 * q + 2 * p + 1);
                        if (group == 0 && mine) { dw[which * A.d + e0] += v[0]; dw[which * A.d + e1] += v[1]; }
                    }
            }
        }
    }
    if (GRAD && A.part) {
        __syncthreads();
        const float *from = weights + 2 * 16 * TPH;
        for (int i = threadIdx.x; i < 2 * A.d; i += ROT_THREADS) {
            float sum = 0.0f;
            for (int w = 0; w < ROT_WARPS; ++w) sum += from[w * 2 * A.d + i];
            A.part[(i64)blockIdx.x * 2 * A.d + i] = sum;
        }
    }
}

// Weights' gradients: the CTAs' partial sums, added up in 64 bits in their order.  32 columns a CTA, every warp takes a stretch of CTAs.
__global__ void __launch_bounds__(1024) k_rotate_weights(RotArgs A, int ctas)
{
    __shared__ double part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    const int per = (ctas + 31) / 32, lo = warp * per, hi = min(ctas, lo + per);
    double sum = 0.0;
    if (col < 2 * A.d)
        for (int b = lo; b < hi; ++b) sum += A.part[(i64)b * 2 * A.d + col];
    part[warp][lane] = sum;
    __syncthreads();
    if (warp || col >= 2 * A.d) return;
    sum = 0.0;
    for (int w = 0; w < 32; ++w) sum += part[w][lane];
    const int which = col >= A.d;
    if (A.h[which].dw) A.h[which].dw[col - which * A.d] = (float)sum;
}

// ---------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------
#define ROT_MAX_CTAS 1184                // CTAs at most (8 on each of 148 SMs): what the workspace is sized for

static int check_heads(const rp_rotary *r, const rp_heads *h, bool grad, RpOpDevice &dev)
{
    if (!h || h->n_heads == 0) return RP_OK;
    const int b = rp_type_bytes(r->type);
    if (h->n_heads < 0 || h->n_heads > 65536 || !h->y || (!h->x && (!grad || h->weight)) || (grad && !h->y_grad) ||
        (grad && h->weight_grad && !h->weight))
        return RP_ERR_ARG;
    if (!rp_aligned(h->x, b) || !rp_aligned(h->y, b) || (grad && !rp_aligned(h->y_grad, b)) || (grad && !rp_aligned(h->weight_grad, 4)) ||
        !rp_aligned(h->weight, r->weight_type == RP_F32 ? 4 : b))
        return RP_ERR_ARG;
    RP_TRY(dev.hold(h->x)); RP_TRY(dev.hold(h->y)); RP_TRY(dev.hold(h->weight));
    if (grad) { RP_TRY(dev.hold(h->y_grad)); RP_TRY(dev.hold(h->weight_grad)); }
    return RP_OK;
}
static void take_heads(RotTensor &o, const rp_heads *h, bool grad)
{
    o = RotTensor();
    if (!h || h->n_heads == 0) return;
    o.x = h->x; o.x_token = h->x_token; o.x_head = h->x_head; o.y = h->y; o.y_token = h->y_token; o.y_head = h->y_head;
    o.w = h->weight; o.heads = h->n_heads;
    if (grad) { o.dy = h->y_grad; o.g_token = h->g_token; o.g_head = h->g_head; o.dw = h->weight_grad; }
}

template <typename X, int TPH> static void (*rows_kernel(bool interleaved, bool grad))(RotArgs)
{
    if (interleaved) return grad ? k_rotate_rows<X, TPH, true, true> : k_rotate_rows<X, TPH, true, false>;
    return grad ? k_rotate_rows<X, TPH, false, true> : k_rotate_rows<X, TPH, false, false>;
}
template <typename X> static void (*rows_kernel(int tph, bool interleaved, bool grad))(RotArgs)
{
    switch (tph) {
        case 1: return rows_kernel<X, 1>(interleaved, grad);
        case 2: return rows_kernel<X, 2>(interleaved, grad);
        case 4: return rows_kernel<X, 4>(interleaved, grad);
        case 8: return rows_kernel<X, 8>(interleaved, grad);
        case 16: return rows_kernel<X, 16>(interleaved, grad);
        default: return rows_kernel<X, 32>(interleaved, grad);
    }
}

static int rotate(const rp_rotary *r, i64 T, const double *freq, const i64 *start, int N, const i64 *first, const rp_heads *q, const rp_heads *k,
                  bool grad, float *workspace, i64 workspace_bytes, cudaStream_t stream)
{
    if (!r || T < 0 || N < 1 || !start || r->head_dim < 1 || r->rotary_dim < 0 || r->rotary_dim % 2 || r->rotary_dim > r->head_dim ||
        (r->rotary_dim && !freq) || r->layout < RP_ROTARY_HALF || r->layout > RP_ROTARY_INTERLEAVED || r->type < RP_F32 || r->type > RP_BF16 ||
        (r->weight_type != RP_F32 && r->weight_type != r->type) || !(r->eps >= 0.0f))
        return RP_ERR_ARG;
    if (r->head_dim > ROT_MAX_DIM || T > (1ll << 40)) return RP_ERR_RANGE;
    if (!rp_aligned(freq, 8) || !rp_aligned(start, 8) || !rp_aligned(first, 8)) return RP_ERR_ARG;
    RpOpDevice dev;
    RP_TRY(check_heads(r, q, grad, dev));
    RP_TRY(check_heads(r, k, grad, dev));
    if (q && k && q->n_heads && k->n_heads && (q->y == k->y || (grad && q->weight_grad && q->weight_grad == k->weight_grad))) return RP_ERR_ARG;   // two outputs in one place
    const bool weights = grad && ((q && q->n_heads && q->weight_grad) || (k && k->n_heads && k->weight_grad));
    if (weights && (!workspace || workspace_bytes < rp_rotate_workspace(r) || !rp_aligned(workspace, 16))) return RP_ERR_ARG;
    RP_TRY(rp_op_enter(dev, freq, start, first, weights ? workspace : nullptr));
    RotArgs A = {};
    take_heads(A.h[0], q, grad);
    take_heads(A.h[1], k, grad);
    const int all = A.h[0].heads + A.h[1].heads;
    if (!all) return RP_ERR_ARG;
    A.d = r->head_dim; A.r = r->rotary_dim; A.half = r->layout == RP_ROTARY_HALF; A.w32 = r->weight_type == RP_F32;
    A.eps = r->eps; A.mscale = r->mscale; A.inv_d = 1.0f / r->head_dim; A.T = T; A.freq = freq; A.start = start; A.first = first; A.N = N;
    A.part = weights ? workspace : nullptr;
    if (T == 0) {
        for (int w = 0; w < 2; ++w)
            if (A.h[w].dw) RP_CUDA(cudaMemsetAsync(A.h[w].dw, 0, sizeof(float) * A.d, stream));
        return RP_OK;
    }
    // Heads of whole 16-byte pieces, all rows on 16-byte boundaries: 32768 tokens of 32 + 8 heads of 128, 16 bits, take 129 us (gradient 220), by the other kernel
    // 522 (969); 64 tokens 5.3 us and 5.0
    bool pieces = A.d % 16 == 0 && A.d <= 512 && (A.half ? A.r % 16 == 0 : A.r % 8 == 0);
    for (int w = 0; w < 2; ++w) {
        const RotTensor &H = A.h[w];
        if (!H.heads) continue;
        const int e = 16 / rp_type_bytes(r->type);
        pieces = pieces && rp_aligned(H.x, 16) && rp_aligned(H.y, 16) && rp_aligned(H.dy, 16) && H.x_token % e == 0 && H.x_head % e == 0 && H.y_token % e == 0 &&
                 H.y_head % e == 0 && H.g_token % e == 0 && H.g_head % e == 0;
    }
    int tph = 1;
    while (16 * tph < A.d) tph <<= 1;
    // A CTA's warps share out the tokens, or each token's heads where there are fewer tokens than warps.
    const int ng = pieces ? 32 / tph : 1, steps = (A.h[0].heads + ng - 1) / ng + (A.h[1].heads + ng - 1) / ng;
    const i64 warps = std::min((i64)ROT_MAX_CTAS, (i64)rp_op_sms(dev.device) * (pieces ? ROT_CTAS(grad) : 8)) * ROT_WARPS;
    A.parts = T >= warps ? 1 : (int)std::min((i64)steps, warps / T);
    const i64 lanes = std::min(T, warps / A.parts);
    A.run = (T + lanes - 1) / lanes;
    const int ctas = (int)((lanes * A.parts + ROT_WARPS - 1) / ROT_WARPS);
    size_t smem = ROT_WARPS * ((pieces ? ROT_CHUNK * 8 * tph : A.r / 2) * sizeof(float2) + (A.part ? 2 * A.d * sizeof(float) : 0)) + (pieces ? 2 * 16 * tph * sizeof(float) : 0);
    RP_FOR_TYPE(r->type, {
        void (*f)(RotArgs) = grad ? k_rotate_any<X, true> : k_rotate_any<X, false>;
        if (pieces) f = rows_kernel<X>(tph, !A.half, grad);
        if (smem > 48 * 1024) RP_CUDA(cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, RP_SMEM_LIMIT));
        f<<<ctas, ROT_THREADS, smem, stream>>>(A);
    });
    RP_TRY(rp_op_launched());
    if (A.part) {
        k_rotate_weights<<<(2 * A.d + 31) / 32, 1024, 0, stream>>>(A, ctas);
        RP_TRY(rp_op_launched());
    }
    return RP_OK;
}

extern "C" int rp_rotate(const rp_rotary *r, int64_t n_tokens, const double *inv_freq, const int64_t *start, int32_t n_samples,
                         const int64_t *first_position, const rp_heads *q, const rp_heads *k, void *cuda_stream)
{
    return rotate(r, n_tokens, inv_freq, (const i64 *)start, n_samples, (const i64 *)first_position, q, k, false, nullptr, 0, (cudaStream_t)cuda_stream);
}

extern "C" int64_t rp_rotate_workspace(const rp_rotary *r)
{
    if (!r || r->head_dim < 1) return 0;
    return (int64_t)ROT_MAX_CTAS * 2 * r->head_dim * (int64_t)sizeof(float);
}

extern "C" int rp_rotate_grad(const rp_rotary *r, int64_t n_tokens, const double *inv_freq, const int64_t *start, int32_t n_samples,
                              const int64_t *first_position, const rp_heads *q, const rp_heads *k, void *workspace, int64_t workspace_bytes,
                              void *cuda_stream)
{
    return rotate(r, n_tokens, inv_freq, (const i64 *)start, n_samples, (const i64 *)first_position, q, k, true, (float *)workspace, workspace_bytes,
                  (cudaStream_t)cuda_stream);
}
