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
    float eps, mscale;
    i64 T, run;             // run: tokens of a warp
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

// Any head size and alignment: a warp takes one head after the other, a lane the pairs lane, lane + 32, .. and then the elements behind them.
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
#define ROT_MAX_CTAS 1184                // CTAs of the gradient, at most (8 on each of 148 SMs): what the workspace is sized for

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
    const bool weights = grad && ((q && q->n_heads && q->weight_grad) || (k && k->n_heads && k->weight_grad));
    if (weights && (!workspace || workspace_bytes < rp_rotate_workspace(r) || !rp_aligned(workspace, 16))) return RP_ERR_ARG;
    RP_TRY(rp_op_enter(dev, freq, start, first, weights ? workspace : nullptr));
    RotArgs A = {};
    take_heads(A.h[0], q, grad);
    take_heads(A.h[1], k, grad);
    const int all = A.h[0].heads + A.h[1].heads;
    if (!all) return RP_ERR_ARG;
    A.d = r->head_dim; A.r = r->rotary_dim; A.half = r->layout == RP_ROTARY_HALF; A.w32 = r->weight_type == RP_F32;
    A.eps = r->eps; A.mscale = r->mscale; A.T = T; A.freq = freq; A.start = start; A.first = first; A.N = N;
    A.part = weights ? workspace : nullptr;
    if (T == 0) {
        for (int w = 0; w < 2; ++w)
            if (A.h[w].dw) RP_CUDA(cudaMemsetAsync(A.h[w].dw, 0, sizeof(float) * A.d, stream));
        return RP_OK;
    }
    const i64 warps = std::min((i64)ROT_MAX_CTAS, (i64)rp_op_sms(dev.device) * 8) * ROT_WARPS;
    A.parts = T >= warps ? 1 : (int)std::min((i64)all, warps / T);
    const i64 lanes = warps / A.parts;
    A.run = (T + lanes - 1) / lanes;
    const i64 units = (T + A.run - 1) / A.run * A.parts;
    const int ctas = (int)((units + ROT_WARPS - 1) / ROT_WARPS);
    const size_t smem = ROT_WARPS * (A.r / 2 * sizeof(float2) + (A.part ? 2 * A.d * sizeof(float) : 0));
    if (grad) {
        RP_FOR_TYPE(r->type, {
            if (smem > 48 * 1024) RP_CUDA(cudaFuncSetAttribute(k_rotate_any<X, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, RP_SMEM_LIMIT));
            k_rotate_any<X, true><<<ctas, ROT_THREADS, smem, stream>>>(A);
        });
    } else
        RP_FOR_TYPE(r->type, (k_rotate_any<X, false><<<ctas, ROT_THREADS, smem, stream>>>(A)));
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
