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
    int lanes;              // lanes of a warp that share a token: 4 where a token's layers lie side by side, 1 where a layer's tokens do
    int rows;               // experts of the counters in shared memory
};

#define COUNT_THREADS 512
// A lane's counters lie in a bank of its own (counter of expert e at e * 32 + lane), so that the 32 additions of a warp go in one go whatever they count; with one
// counter for all lanes, skewed choices put 3 to 4 of them in one bank (900001 tokens of 32 layers, 8 of 128 experts in bytes: 207 us for what takes 91).
__device__ __forceinline__ void count_one(u32 at, u32 e)
{
    u32 to;
    asm("mad.lo.u32 %0, %1, 128, %2;" : "=r"(to) : "r"(e), "r"(at));
    asm volatile("red.shared.add.u32 [%0], 1;" ::"r"(to) : "memory");
}
template <int ENTRY> __device__ __forceinline__ void count_word(u32 at, u32 w, u32 hi, int E)
{
    if constexpr (ENTRY == 1) {
        // 256 rows of counters: any byte has one
#pragma unroll
        for (int b = 0; b < 4; ++b) count_one(at, __byte_perm(w, 0, 0x4440 | b));
    } else if constexpr (ENTRY == 2) {
        if ((w & 0xffffu) < (u32)E) count_one(at, w & 0xffffu);
        if ((w >> 16) < (u32)E) count_one(at, w >> 16);
    } else {
        if (w < (u32)E && hi == 0) count_one(at, w);
    }
}
// Where tile b of n begins: a sample's end costs as much as COUNT_END tokens (two meetings of the CTA, and adding up its counters), and the tiles are of one cost.
#define COUNT_END 160
__device__ __forceinline__ i64 tile_start(const CountArgs &A, int b, int n)
{
    if (b <= 0) return 0;
    if (b >= n) return A.T;
    const i64 cost = A.T + (i64)COUNT_END * A.N, want = cost / n * b + cost % n * b / n;
    u32 lo = 0, hi = (u32)A.N + 1;                       // first i with start[i] + COUNT_END * i above it
    while (lo < hi) {
        const u32 mid = (lo + hi) >> 1;
        if (__ldg(A.start + mid) + (i64)COUNT_END * mid <= want) lo = mid + 1; else hi = mid;
    }
    i64 t = want - (i64)COUNT_END * max((i64)lo - 1, (i64)0);
    if (lo <= (u32)A.N) t = min(t, __ldg(A.start + lo));
    return min(max(t, (i64)0), A.T);
}
// Bound by the additions: 230 million of them for those 230 MB, 58 % of what shared memory takes (52 us), 2.7 TB/s from memory of 6.5.
// A CTA owns a tile of tokens and lanes * LAYERS layers, whatever samples the tokens belong to: it counts one sample after the other in shared memory and adds what
// it found to the output (whole numbers: the order does not matter).  WORDS: 32-bit words of a token's choices in LAYERS layers, copied as such into a ring of the
// lane's own, DEPTH tokens ahead, across the samples' ends; 0: any number of choices, read one by one (450001 tokens of 32 layers, 2 or 6 of 128 experts in bytes: 79 and
// 120 us, where 8, copied, take 54).
template <int WORDS> struct CountRing { static constexpr int DEPTH = WORDS <= 4 ? 4 : WORDS == 8 ? 3 : 2, BYTES = WORDS ? DEPTH * WORDS * 4 * COUNT_THREADS : 0; };
template <typename R, int WORDS, int LAYERS>
__global__ void __launch_bounds__(COUNT_THREADS, 2) k_count_routes(CountArgs A)
{
    constexpr int DEPTH = CountRing<WORDS>::DEPTH, COPY = WORDS >= 4 ? 16 : 4 * WORDS;       // bytes of a copy
    extern __shared__ __align__(16) u32 hist[];          // [LAYERS][rows][32], ring
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // (no tile is as long as 2^30 tokens where the starts do not decrease)
    const i64 t0 = tile_start(A, blockIdx.x, gridDim.x), t1 = min(max(t0, tile_start(A, blockIdx.x + 1, gridDim.x)), t0 + (1ll << 30));
    const int l0 = blockIdx.y * A.lanes * LAYERS, layer = l0 + lane % A.lanes * LAYERS;      // first of the CTA, first of the lane
    const int per = 32 / A.lanes, step = COUNT_THREADS / 32 * per;                          // tokens of a warp, of the CTA at a time
    const R *routes = (const R *)A.routes;
    const u32 base = (u32)__cvta_generic_to_shared(hist) + lane * 4;
    // the lane's tokens, from the tile's first: x, x + step, ..; fetched so far: up to `far`
    const int len = (int)(t1 - t0);
    int x = layer < A.L ? warp * per + lane / A.lanes : len, far = x;
    const i64 inc = step * A.ts * (i64)sizeof(R);
    const char *from = (const char *)(routes + (layer < A.L ? layer * A.ls + (t0 + x) * A.ts : 0));
    const char *ring = (const char *)(hist + LAYERS * A.rows * 32) + threadIdx.x * (COPY ? COPY : 4);
    const u32 ring_at = (u32)__cvta_generic_to_shared(ring);
    auto fetch = [&](int slot) {
        if constexpr (WORDS > 0) {
            if (far < len) {
                const u32 to = ring_at + slot * (WORDS * 4 * COUNT_THREADS);
                if constexpr (COPY == 16) {
#pragma unroll
                    for (int v = 0; v < WORDS / 4; ++v)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + v * 16 * COUNT_THREADS), "l"(from + 16 * v) : "memory");
                } else
                    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(COPY ? COPY : 4) : "memory");
                from += inc;
                far += step;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    int slot = 0;
#pragma unroll
    for (int u = 0; u < DEPTH; ++u) fetch(u);
    for (int y = threadIdx.x; y < LAYERS * A.rows * 8; y += COUNT_THREADS) ((uint4 *)hist)[y] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    for (i64 t = t0; t < t1;) {
        const int i = rp_sample_of(A.start, A.N, t);
        i64 end = t1;
        if (i < A.N) end = min(end, __ldg(A.start + i + 1));
        if (end <= t) end = t + 1;                       // starts that decrease: every step makes headway all the same
        const bool held = i >= 0 && i < A.N;
        const int stop = (int)(end - t0);
        if constexpr (WORDS > 0) {
            for (; x < stop; x += step) {
                asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
                u32 w[WORDS];
                const char *p = ring + slot * (WORDS * 4 * COUNT_THREADS);
                if constexpr (COPY == 16) {
#pragma unroll
                    for (int v = 0; v < WORDS; v += 4) {
                        const uint4 q = *(const uint4 *)(p + v * 4 * COUNT_THREADS);
                        w[v] = q.x; w[v + 1] = q.y; w[v + 2] = q.z; w[v + 3] = q.w;
                    }
                } else {
#pragma unroll
                    for (int v = 0; v < WORDS; ++v) w[v] = ((const u32 *)p)[v];
                }
                fetch(slot);
                slot = slot + 1 == DEPTH ? 0 : slot + 1;
                if (held)
#pragma unroll
                    for (int v = 0; v < WORDS; ++v) {
                        const u32 to = base + v / (WORDS / LAYERS) * A.rows * 128;
                        if constexpr (sizeof(R) < 8) count_word<sizeof(R)>(to, w[v], 0, A.E);
                        else if (v % 2 == 0) count_word<8>(to, w[v], w[v + 1], A.E);
                    }
            }
        } else {
            for (; x < stop; x += step)
                for (int j = 0; held && j < A.k; ++j) {
                    const i64 e = (i64)routes[(t0 + x) * A.ts + layer * A.ls + j];
                    if (e >= 0 && e < A.E) count_one(base, (u32)e);
                }
        }
        if (held) {
            int *out = A.demand + ((i64)i * A.L + l0) * A.E;
            const int layers = min(A.L - l0, A.lanes * LAYERS), experts = min(A.E, A.rows);        // (a byte has no choice above 255)
            __syncthreads();
            // Eight lanes add up an expert's 32 counters; those of lanes that share a token are layers of their own: at the end lane q of the eight has the sum of the
            // counters q mod 4 of four lanes, and its neighbour four lanes on that of the others.
#pragma unroll
            for (int sub = 0; sub < LAYERS; ++sub)
                for (int first = warp * 4; first < experts; first += COUNT_THREADS / 8) {    // (the whole warp goes round as often)
                    const int e = first + (lane >> 3), q = lane & 3, l = q * LAYERS + sub;
                    uint4 *p = (uint4 *)(hist + (sub * A.rows + e) * 32) + (lane & 7), c = make_uint4(0, 0, 0, 0);
                    if (e < experts) { c = *p; *p = make_uint4(0, 0, 0, 0); }
                    const bool odd = lane & 1, high = lane & 2;
                    // the pair's even lane goes on with x and z, the odd one with y and w; of two pairs the lower with the first of those
                    const u32 k0 = (odd ? c.y : c.x) + __shfl_xor_sync(0xffffffffu, odd ? c.x : c.y, 1);
                    const u32 k1 = (odd ? c.w : c.z) + __shfl_xor_sync(0xffffffffu, odd ? c.z : c.w, 1);
                    u32 v = (high ? k1 : k0) + __shfl_xor_sync(0xffffffffu, high ? k0 : k1, 2);
                    v += __shfl_xor_sync(0xffffffffu, v, 4);
                    if (A.lanes == 1) { v += __shfl_xor_sync(0xffffffffu, v, 1); v += __shfl_xor_sync(0xffffffffu, v, 2); }
                    if ((lane & 7) < A.lanes && v && e < experts && l < layers) atomicAdd(out + l * A.E + e, (int)v);
                }
            __syncthreads();
        }
        t = end;
    }
}

template <typename R>
static int launch_count(CountArgs &A, int sms, cudaStream_t stream)
{
    const int bytes = A.k * (int)sizeof(R);
    const auto words = [&](int n) {                      // can a token's choices be read as n bytes at a time?
        const int w = n >= 16 ? 16 : n;
        return rp_aligned(A.routes, w) && A.ts * (i64)sizeof(R) % w == 0 && (A.lanes == 1 && A.L == 1 ? true : A.ls * (i64)sizeof(R) % w == 0);
    };
    // Bytes of eight choices: two layers of a lane's in 16 bytes (one layer in 8 leaves half of every 64 bytes from memory to another CTA)
    const bool two = sizeof(R) == 1 && bytes == 8 && A.lanes == 4 && A.ls == A.k && A.L % 2 == 0 && A.L >= 8 && rp_aligned(A.routes, 16) && A.ts % 16 == 0;
    void (*f)(CountArgs) = k_count_routes<R, 0, 1>;
    const int layers = two ? 2 : 1;
    size_t ring = 0;
    const auto pick = [&](void (*g)(CountArgs), int bytes_ahead) { f = g; ring = bytes_ahead; };
    if (two) { if constexpr (sizeof(R) == 1) pick(k_count_routes<R, 4, 2>, CountRing<4>::BYTES); }
    else if (bytes == 4 && words(4)) { if constexpr (sizeof(R) <= 4) pick(k_count_routes<R, 1, 1>, CountRing<1>::BYTES); }
    else if (bytes == 8 && words(8)) pick(k_count_routes<R, 2, 1>, CountRing<2>::BYTES);
    else if (bytes == 16 && words(16)) pick(k_count_routes<R, 4, 1>, CountRing<4>::BYTES);
    else if (bytes == 32 && words(16)) pick(k_count_routes<R, 8, 1>, CountRing<8>::BYTES);
    else if (bytes == 64 && words(16)) pick(k_count_routes<R, 16, 1>, CountRing<16>::BYTES);
    A.rows = sizeof(R) == 1 ? 256 : A.E;
    const size_t smem = (size_t)layers * A.rows * 128 + ring;
    if (smem > 48 * 1024) RP_CUDA(cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, RP_SMEM_LIMIT));
    // as many CTAs as stay resident; a tile is not so short that setting its counters to zero and adding them up costs more than counting
    const int groups = (A.L + A.lanes * layers - 1) / (A.lanes * layers);
    const i64 resident = (i64)sms * std::min((size_t)2, (size_t)(224 * 1024) / (smem + 1024));
    const i64 most = std::max((i64)1, resident / groups), cost = A.T + (i64)COUNT_END * A.N;
    const i64 tiles = std::max(std::min(most, (cost + 511) / 512), (cost >> 30) + 1);            // (a tile's tokens are counted in 32 bits)
    f<<<dim3((unsigned)tiles, groups), COUNT_THREADS, smem, stream>>>(A);
    return rp_op_launched();
}

// Queues the count on a stream of the current device; `demand` is written whole.
int rp_launch_count(int device, const void *routes, int bytes, i64 T, int L, int k, int E, i64 ts, i64 ls, const i64 *start, int N, int *demand,
                    cudaStream_t stream)
{
    RP_CUDA(cudaMemsetAsync(demand, 0, sizeof(int) * (size_t)N * L * E, stream));
    if (T < 1) return RP_OK;
    CountArgs A = { routes, T, ts, ls, L, k, E, N, start, demand, ls < ts && L > 1 ? 4 : 1, 0 };
    const int sms = rp_op_sms(device);
    switch (bytes) {
        case 1: return launch_count<unsigned char>(A, sms, stream);
        case 2: return launch_count<short>(A, sms, stream);
        case 4: return launch_count<int>(A, sms, stream);
        default: return launch_count<i64>(A, sms, stream);
    }
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
    if (E > 1024 || k > 1024 || L > 65535 || (i64)L * E >= (1ll << 31) || T > (1ll << 36)) return RP_ERR_RANGE;
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
