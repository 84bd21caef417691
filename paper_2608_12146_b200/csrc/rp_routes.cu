// Per-expert counts of recorded routes: demand[i][l][e] = #{(t, j): token t in sample i, routes[t][l][j] = e}, the demand tensor of the
// planner from what a serving engine or a trainer recorded.
//
// Reads n_tokens * L * k route values once and writes N * L * E counts.
#include <algorithm>

#include "rp_ops.cuh"

int rp_op_sms(int device)
{
    static int sms[64];                                  // the same value from every thread that fills it in
    if (device < 0 || device >= 64) return 148;
    if (!sms[device] && cudaDeviceGetAttribute(&sms[device], cudaDevAttrMultiProcessorCount, device) != cudaSuccess) { cudaGetLastError(); return 148; }
    return sms[device];
}

struct CountArgs {
    const void *routes;
    i64 T, ts, ls;
    int L, k, E, N;
    const i64 *start;
    int *demand;
    int layers;             // layers of a CTA
    i64 tile;               // tokens of a CTA
};

#define COUNT_THREADS 256
// A CTA owns a tile of tokens and a range of layers, whatever samples they belong to: it counts one sample after the other in shared memory and
// adds what it found to the output (whole numbers: the order does not matter).
template <typename R>
__global__ void __launch_bounds__(COUNT_THREADS) k_count_routes(CountArgs A)
{
    extern __shared__ int hist[];                        // [layers][E]
    const i64 t0 = (i64)blockIdx.x * A.tile, t1 = min(A.T, t0 + A.tile);
    const int l0 = blockIdx.y * A.layers, nl = min(A.L - l0, A.layers);
    const R *routes = (const R *)A.routes;
    for (int x = threadIdx.x; x < nl * A.E; x += COUNT_THREADS) hist[x] = 0;
    __syncthreads();
    for (i64 t = t0; t < t1;) {
        const int i = rp_sample_of(A.start, A.N, t);
        i64 end = t1;
        if (i < A.N) end = min(end, __ldg(A.start + i + 1));
        if (end <= t) end = t + 1;                       // starts that decrease: every step makes headway all the same
        if (i >= 0 && i < A.N) {
            const i64 items = (end - t) * nl;
            for (i64 x = threadIdx.x; x < items; x += COUNT_THREADS) {
                const i64 tok = A.ls < A.ts ? x / nl : x % (end - t);
                const int l = (int)(A.ls < A.ts ? x % nl : x / (end - t));
                const R *at = routes + (t + tok) * A.ts + (l0 + l) * A.ls;
                for (int j = 0; j < A.k; ++j) {
                    const i64 e = (i64)at[j];
                    if (e >= 0 && e < A.E) atomicAdd(&hist[l * A.E + (int)e], 1);
                }
            }
            __syncthreads();
            int *out = A.demand + ((i64)i * A.L + l0) * A.E;
            for (int x = threadIdx.x; x < nl * A.E; x += COUNT_THREADS) {
                const int c = hist[x];
                if (c) { atomicAdd(out + x, c); hist[x] = 0; }
            }
            __syncthreads();
        }
        t = end;
    }
}

// Queues the count on a stream of the current device; `demand` is written whole.
int rp_launch_count(int device, const void *routes, int bytes, i64 T, int L, int k, int E, i64 ts, i64 ls, const i64 *start, int N, int *demand,
                    cudaStream_t stream)
{
    RP_CUDA(cudaMemsetAsync(demand, 0, sizeof(int) * (size_t)N * L * E, stream));
    if (T < 1) return RP_OK;
    CountArgs A = { routes, T, ts, ls, L, k, E, N, start, demand, 0, 0 };
    A.layers = std::max(1, std::min(L, 32 * 1024 / 4 / E));
    const int groups = (L + A.layers - 1) / A.layers;
    const i64 want = std::max((i64)1, (i64)rp_op_sms(device) * 8 / groups);
    A.tile = std::max((T + want - 1) / want, (i64)16);
    const dim3 grid((unsigned)((T + A.tile - 1) / A.tile), groups);
    const size_t smem = sizeof(int) * (size_t)A.layers * E;
    switch (bytes) {
        case 1: k_count_routes<unsigned char><<<grid, COUNT_THREADS, smem, stream>>>(A); break;
        case 2: k_count_routes<short><<<grid, COUNT_THREADS, smem, stream>>>(A); break;
        case 4: k_count_routes<int><<<grid, COUNT_THREADS, smem, stream>>>(A); break;
        default: k_count_routes<i64><<<grid, COUNT_THREADS, smem, stream>>>(A); break;
    }
    return rp_op_launched();
}

// start[i] = lengths[0] + .. + lengths[i-1], by one CTA (N <= 2^20).
__global__ void __launch_bounds__(1024) k_starts(const int *__restrict__ lengths, int N, i64 *__restrict__ start)
{
    __shared__ i64 part[32];
    __shared__ i64 carry;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) { carry = 0; start[0] = 0; }
    __syncthreads();
    for (int base = 0; base < N; base += 1024) {
        const int i = base + threadIdx.x;
        i64 sum = i < N ? lengths[i] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const i64 x = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += x;
        }
        if (lane == 31) part[warp] = sum;
        __syncthreads();
        i64 before = carry;
        for (int w = 0; w < warp; ++w) before += part[w];
        if (i < N) start[i + 1] = before + sum;
        __syncthreads();
        if (threadIdx.x == 1023) carry = before + sum;
        __syncthreads();
    }
}
int rp_launch_starts(const int *lengths, int N, i64 *start, cudaStream_t stream)
{
    k_starts<<<1, 1024, 0, stream>>>(lengths, N, start);
    return rp_op_launched();
}

int rp_count_args(const void *routes, int bytes, i64 T, int L, int k, int E)
{
    if (!routes || T < 0 || L < 1 || k < 1 || E < 1 || (bytes != 1 && bytes != 2 && bytes != 4 && bytes != 8)) return RP_ERR_ARG;
    if (!rp_aligned(routes, bytes)) return RP_ERR_ARG;
    if (E > 1024 || k > 1024 || (i64)L * E >= (1ll << 31) || T > (1ll << 40)) return RP_ERR_RANGE;
    return RP_OK;
}

extern "C" int rp_count_routes(const void *routes, int32_t route_bytes, int64_t n_tokens, int32_t n_layers, int32_t top_k, int32_t n_experts,
                               int64_t token_stride, int64_t layer_stride, const int64_t *start, int32_t n_samples, int32_t *demand,
                               void *cuda_stream)
{
    if (!start || !demand || n_samples < 1 || !rp_aligned(start, 8) || !rp_aligned(demand, 4)) return RP_ERR_ARG;
    RP_TRY(rp_count_args(routes, route_bytes, n_tokens, n_layers, top_k, n_experts));
    RpOpDevice dev;
    RP_TRY(rp_op_enter(dev, routes, start, demand));
    return rp_launch_count(dev.device, routes, route_bytes, n_tokens, n_layers, top_k, n_experts, token_stride, layer_stride, (const i64 *)start,
                           n_samples, demand, (cudaStream_t)cuda_stream);
}
