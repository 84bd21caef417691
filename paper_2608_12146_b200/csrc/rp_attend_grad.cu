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
// those of the softmax: at 4096 tokens the tensor cores are busy for 21 % (keys, which also wait for the largest block) and 41 % (queries) of the time.
#include <algorithm>

#include "rp_attend.cuh"

struct GradArgs {
    const int2 *items;
    AttendHead *head;
    const i64 *start;
    i64 T;
    int Hq, Hk, share, d, causal;
    float scale;
    const float2 *stats;                     // [Hq][T]: lse / ln 2, delta
    const u32 *tops;                         // float16: [samples] square of the norm of the largest row of do, as bits
    void *x[2];                              // dv, dk, or dq
    i64 token[2], hd[2];
    int *status;
    u64 wait_ns;
    const void *rows[2];                     // queries' kernel: q, do
    i64 r_token[2], r_head[2];
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
    if (blockIdx.x == 0) { rp_attend_plan(keys); return; }
    if (blockIdx.x == 1) { rp_attend_plan(queries); return; }
    const int b = blockIdx.x - 2, n = gridDim.x - 2, lane = threadIdx.x & 15;
    rp_attend_clear(C, keys.start, keys.N, keys.T, b, n);
    if constexpr (Narrow<X>::value)
        for (int i = b * 1024 + threadIdx.x; i < keys.N; i += n * 1024) A.tops[i] = 0;
    // 64 rows of a CTA: heads of a token, tokens; four steps on their way at a time (all lanes go round as often)
    constexpr int AHEAD = 4;
    const i64 T = keys.T;
    const int heads = min(A.H, 64), tokens = 64 / heads, row = threadIdx.x >> 4, dt = row / heads;
    for (int h0 = 0; h0 < A.H; h0 += heads) {
        const int h = h0 + row % heads;
        const bool mine = dt < tokens && h < A.H;
        const X *o = (const X *)A.o + h * A.o_head + lane * 8, *g = (const X *)A.g + h * A.g_head + lane * 8;
        for (i64 t0 = (i64)b * tokens; t0 < T; t0 += (i64)AHEAD * n * tokens) {
            Pack8<X> p[AHEAD], q[AHEAD];
            float l[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const i64 t = t0 + (i64)u * n * tokens + dt;
                p[u] = Pack8<X>(); q[u] = Pack8<X>(); l[u] = 0.0f;
                if (mine && t < T && lane * 8 < A.d) { p[u] = rp_load8(o + t * A.o_token); q[u] = rp_load8(g + t * A.g_token); }
                if (mine && t < T && lane == 0) l[u] = A.lse[t * A.l_token + h * A.l_head];
            }
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
        }
    }
}

// The largest of a sample's rows of do, for float16 (infinities and NaN, which no factor mends, do not count): a thread a token.
__global__ void __launch_bounds__(256) k_attend_tops(const i64 *start, int N, i64 T, int H, const float *norms, u32 *tops)
{
    const i64 t = (i64)blockIdx.x * 256 + threadIdx.x;
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

// ---------------------------------------------------------------------------------------
// keys: dk and dv
// ---------------------------------------------------------------------------------------
// Tiles of 128 queries: scores, do v^T and the two sums fill the tensor memory (2 * 128 + 2 * head_dim columns).  Both groups of four warps work on a tile, 64 columns
// each.  The products come in the order dv(j), s(j + 1), dk(j), do v^T(j + 1): while the weights of a tile are worked out, the tensor cores add up dk of the one
// before and multiply do v^T of this one; while the gradients of its scores are, dv of this and scores of the next.  Weights and gradients lie as operands where the
// scores and the products of their group were.  (Tiles of 64 queries, two of them at a time, one for each group: 435 us
// for what takes 249; see the launch.)
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

template <typename X, int D>
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
    rp_let_next_launch_start();              // the queries' kernel takes the SMs that run out of work here
    if (warp == ATTEND_COPY_WARP) tmem_alloc(rp_smem(&sm.tmem), 512);
    tmem_before();
    __syncthreads();
    tmem_after();
    const u32 tm = rp_uniform(sm.tmem);
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
                const AttendTile t(A.items, A.start, A.T, at / A.Hk, 128);
                const int hk = at % A.Hk, first = A.causal ? t.row0 >> 7 : 0, per = ((t.len + 127) >> 7) - first;
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
            const u32 one = lane == 0;
            u32 base = 0;                               // tiles of the items before
            for (int n = 0;; ++n) {
                const int at = rp_attend_item(n, total);
                if (at < 0 || rp_uniform(waits->gave_up)) break;
                const AttendTile t(A.items, A.start, A.T, at / A.Hk, 128);
                const int len = rp_uniform(t.len), first = A.causal ? (int)rp_uniform(t.row0 >> 7) : 0, per = ((len + 127) >> 7) - first, nt = per * A.share;
                int tile = first;                       // of queries: the next to arrive
                // 128 keys against a tile's queries, or their values against the gradients
                auto against = [&](u32 to, const unsigned char *keys, const unsigned char *queries, u32 bar) {
                    const u32 a = mma_operand(rp_smem(keys), true, 0), b = mma_operand(rp_smem(queries), true, 0);
#pragma unroll
                    for (int x = 0; x < D / 16; ++x) {
                        const u32 off = ((x / 4) * PANEL + (x % 4) * 32) >> 4;
                        mma_ss(one, to, a + off, b + off, shape_s, x > 0);
                    }
                    mma_commit(one, bar);
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
#pragma unroll
                    for (int x = 0; x < 8; ++x) mma_ts(one, to, weights + (x / 4) * 64 + (x % 4) * 8, b + x * (2048 >> 4), shape_o, more || x > 0);
                };
                bar_hold(rp_smem(&sm.kv_full), n & 1, waits);
                arrived(base);
                against(tm, sm.k, sm.q[base % STAGES], rp_smem(&sm.s_full));
                against(tm + 128, sm.v, sm.g[base % STAGES], rp_smem(&sm.dp_full));
                if (nt == 1) mma_commit(one, rp_smem(&sm.kv_empty));
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
                    mma_commit(one, rp_smem(&sm.q_empty[s]));
                    if (j + 1 < nt) {
                        against(tm + 128, sm.v, sm.g[s1], rp_smem(&sm.dp_full));
                        if (j + 2 == nt) mma_commit(one, rp_smem(&sm.kv_empty));
                    } else
                        mma_commit(one, rp_smem(&sm.acc_full));
                }
                base += nt;
            }
            // nobody may leave while products are under way
            mma_commit(one, rp_smem(&sm.done));
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
            const AttendTile t(A.items, A.start, A.T, at / A.Hk, 128);
            const int hk = at % A.Hk, first = A.causal ? t.row0 >> 7 : 0, per = ((t.len + 127) >> 7) - first, nt = per * A.share, r = t.row0 + row;
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
                if (q0 + 64 > t.len || (A.causal && q0 < t.row0 + 128)) {
                    const int lo = A.causal ? r - q0 : 0, hi = t.len - q0;
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
            store_row<X, D>(tm + lanes + 256 + b * D, out, A.d, r < t.len, !ok ? NAN : b ? f1 : f0);
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
// takes 166).  Scores are multiplied while the weights of the tile before are worked out (as soon as those have been read), dq of a
// tile and do v^T of the next while the weights of the next are.  Columns: scores 128, do v^T 128 (and in its place ds as operand), dq, q and do 64 each.
template <int D> struct QuerySmem {
    static constexpr int TILE = 128 * D * 2, STAGES = 3;
    alignas(1024) unsigned char k[STAGES][TILE];
    alignas(1024) unsigned char v[STAGES][TILE];
    u64 q_full, kv_full[STAGES], kv_empty[STAGES], s_full, s_empty, dp_full, ds_full, acc_full, item_full[2], item_empty[2], done;
    u32 tmem;
    volatile int item[2];
    int taken, handled[8];                   // when a wait has run out: blocks that the CTA took, blocks that each warp of the softmax handed over
    Waits waits;
};

template <typename X, int D>
__global__ void __launch_bounds__(ATTEND_THREADS, 1)
k_attend_queries(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const GradArgs A)
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
            tma_prefetch(&map_k); tma_prefetch(&map_v);
            u32 fill = 0;
            int taken = 0;
            bool ok = true;
            for (int n = 0; ok; ++n) {
                // the next of the list for whoever is free: CTAs start as the keys' kernel leaves them an SM
                if (!(ok = bar_place(n > 1, rp_smem(&sm.item_empty[n & 1]), ((n >> 1) - 1) & 1, waits))) break;
                int at = atomicAdd(&A.head->ticket, 1);
                if (at >= total) at = -1;
                sm.item[n & 1] = at;
                bar_arrive(rp_smem(&sm.item_full[n & 1]));
                if (at < 0) break;
                taken = n + 1;
                const AttendTile t(A.items, A.start, A.T, at / A.Hq, 128);
                const int hk = at % A.Hq / A.share, nk = rp_attend_tiles(t, 0, A.causal);
                for (int j = 0; j < nk; ++j, ++fill) {
                    const u32 s = fill % STAGES, turn = fill / STAGES;
                    if (!(ok = bar_place(turn, rp_smem(&sm.kv_empty[s]), (turn - 1) & 1, waits))) break;
                    bar_expect(rp_smem(&sm.kv_full[s]), 2 * Smem::TILE);
                    waits->copied = fill + 1;
                    for (int p = 0; p < PANELS; ++p) {
                        tma_load3(rp_smem(sm.k[s]) + p * PANEL, &map_k, p * 64, hk, (int)t.base + j * 128, rp_smem(&sm.kv_full[s]));
                        tma_load3(rp_smem(sm.v[s]) + p * PANEL, &map_v, p * 64, hk, (int)t.base + j * 128, rp_smem(&sm.kv_full[s]));
                    }
                }
            }
            sm.taken = taken;
            // nobody may leave while copies are under way (whoever should have waited for them may have given up)
            for (u32 f = fill > (u32)STAGES ? fill - STAGES : 0; f < fill; ++f) rp_drain(rp_smem(&sm.kv_full[f % STAGES]), (f / STAGES) & 1);
        }
        if (warp == ATTEND_MMA_WARP) {
            const u32 shape_s = mma_shape<X>(128, false), shape_o = mma_shape<X>(D, true);
            const u32 one = lane == 0;
            u32 base = 0;                               // tiles of the items before
            for (int n = 0;; ++n) {
                bar_hold(rp_smem(&sm.item_full[n & 1]), (n >> 1) & 1, waits);
                const int at = rp_uniform(sm.item[n & 1]);
                if (at < 0 || rp_uniform(waits->gave_up)) break;
                bar_arrive_warp(rp_smem(&sm.item_empty[n & 1]), lane);
                const AttendTile t(A.items, A.start, A.T, at / A.Hq, 128);
                const int len = rp_uniform(t.len), nk = rp_uniform(rp_attend_tiles(t, 0, A.causal));
                // 128 queries (or gradients) against a tile's keys (or values)
                auto against = [&](u32 to, u32 rows, const unsigned char *tile, u32 bar) {
                    const u32 b = mma_operand(rp_smem(tile), true, 0);
#pragma unroll
                    for (int x = 0; x < D / 16; ++x) mma_ts(one, to, rows + x * 8, b + (((x / 4) * PANEL + (x % 4) * 32) >> 4), shape_s, x > 0);
                    mma_commit(one, bar);
                };
                auto arrived = [&](int j) {             // a tile's keys and values
                    const u32 f = base + j;
                    bar_hold(rp_smem(&sm.kv_full[f % STAGES]), (f / STAGES) & 1, waits);
                    // keys behind the sample's end are another sample's: the gradients of their scores are 0, and 0 times NaN would not be
                    if (len - j * 128 < 128) rp_clear_rows<D>(sm.k[f % STAGES], len - j * 128, 128, lane);
                };
                arrived(0);
                // (who has handed over q and do has taken dq of the block before)
                bar_hold(rp_smem(&sm.q_full), n & 1, waits);
                tmem_after();
                against(tm, tm + 384, sm.k[base % STAGES], rp_smem(&sm.s_full));
                against(tm + 128, tm + 448, sm.v[base % STAGES], rp_smem(&sm.dp_full));
                for (int j = 0; j < nk; ++j) {
                    const u32 f = base + j, s = f % STAGES, s1 = (f + 1) % STAGES;
                    if (j + 1 < nk) {
                        arrived(j + 1);
                        bar_hold(rp_smem(&sm.s_empty), f & 1, waits);
                        tmem_after();
                        against(tm, tm + 384, sm.k[s1], rp_smem(&sm.s_full));
                    }
                    bar_hold(rp_smem(&sm.ds_full), f & 1, waits);
                    tmem_after();
                    const u32 k = mma_operand(rp_smem(sm.k[s]), false, PANEL);
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        mma_ts(one, tm + 256, tm + 128 + (x / 4) * 64 + (x % 4) * 8, k + x * (2048 >> 4), shape_o, j > 0 || x > 0);
                    mma_commit(one, rp_smem(&sm.kv_empty[s]));
                    if (j + 1 < nk) against(tm + 128, tm + 448, sm.v[s1], rp_smem(&sm.dp_full));
                    else mma_commit(one, rp_smem(&sm.acc_full));
                }
                base += nk;
            }
            // nobody may leave while products are under way
            mma_commit(one, rp_smem(&sm.done));
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
        auto fetch = [&](int n) {
            at = -1;
            if (bar_wait_warp(rp_smem(&sm.item_full[n & 1]), (n >> 1) & 1, waits)) at = sm.item[n & 1];
            if (at < 0) return;
            bar_arrive_warp(rp_smem(&sm.item_empty[n & 1]), lane);
            const AttendTile t(A.items, A.start, A.T, at / A.Hq, 128);
            const int r = t.row0 + row;
            const X *p = (b ? (const X *)A.rows[1] + (t.base + r) * A.r_token[1] + at % A.Hq * A.r_head[1] : (const X *)A.rows[0] + (t.base + r) * A.r_token[0] + at % A.Hq * A.r_head[0]);
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (r < t.len && c * 8 < A.d) v = *(const uint4 *)(p + c * 8);
                w[4 * c] = v.x; w[4 * c + 1] = v.y; w[4 * c + 2] = v.z; w[4 * c + 3] = v.w;
            }
        };
        fetch(0);
        int n = 0;
        for (; at >= 0; ++n) {
            const AttendTile t(A.items, A.start, A.T, at / A.Hq, 128);
            const int h = at % A.Hq, nk = rp_attend_tiles(t, 0, A.causal), r = t.row0 + row;
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
                u32 s[64];
                f2 p[32];
                tmem_load32(ts, s);
                tmem_load32(ts + 32, s + 32);
                tmem_loaded();
                tmem_before();
                bar_arrive_warp(rp_smem(&sm.s_empty), lane);
#pragma unroll
                for (int c = 0; c < 32; ++c) p[c] = rp_exp2(rp_fma(rp_f2(__uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1])), sl2, lse2));
                const int k0 = j * 128 + b * 64, lim = (A.causal ? min(t.len, r + 1) : t.len) - k0;
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
                if (k0 + 64 > t.len || (A.causal && k0 + 63 > t.row0)) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) {
                        float x, y;
                        rp_parts(p[c], x, y);
                        s[c] = rp_pair(2 * c < lim ? x : 0.0f, 2 * c + 1 < lim ? y : 0.0f, X());
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
            X *out = (X *)A.x[0] + (t.base + r) * A.token[0] + h * A.hd[0] + b * (D / 2);
            store_row<X, D / 2>(tm + lanes + 256 + b * (D / 2), out, A.d - b * (D / 2), r < t.len, !ok ? NAN : Narrow<X>::value ? A.scale / c1 : A.scale);
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
        for (int n = sm.handled[warp]; n < sm.taken; ++n) mark(sm.item[n & 1], row & ~31, 32, b * (D / 2), D / 2);
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
static i64 plan_bytes(i64 T, int N) { return ((i64)sizeof(AttendHead) + 8 * (T / 128 + N) + 15) / 16 * 16; }

extern "C" int64_t rp_attend_grad_workspace(const rp_attend_config *a, int64_t n_tokens, int32_t n_samples)
{
    if (rp_attend_check(a, n_tokens, n_samples) != RP_OK) return 0;
    return 2 * plan_bytes(n_tokens, n_samples) + 8 * n_tokens * a->q_heads + (a->type == RP_F16 ? 4 * (n_tokens * a->q_heads + n_samples) : 0);
}

struct GradMaps { CUtensorMap q, k, v, g; };

template <typename X, int D>
static int launch(const GradMaps &M, GradArgs &keys, GradArgs &queries, i64 most, int sms, cudaStream_t stream)
{
    const size_t sk = sizeof(KeySmem<D>) + 1024, sq = sizeof(QuerySmem<D>) + 1024;
    RP_CUDA(cudaFuncSetAttribute(k_attend_keys<X, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sk));
    RP_CUDA(cudaFuncSetAttribute(k_attend_queries<X, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sq));
    k_attend_keys<X, D><<<(int)std::min((i64)sms, most * keys.Hk), ATTEND_THREADS, sk, stream>>>(M.q, M.k, M.v, M.g, keys);
    RP_TRY(rp_op_launched());
    // (8192 tokens in three samples, 16 heads on 4, 128 wide: the keys' kernel, whose largest block of keys takes as long as 1.4 times its share of all work, 249 us, the
    // queries' 166; 398 us for the whole call.  A block's query heads dealt out to several CTAs, whose sums meet behind them, make short lists of blocks faster - one
    // sample of 2048 tokens, 5 heads on 1: 193 -> 69 us - but a sample's gradients then depend on what else is in its row.)
    cudaLaunchConfig_t how = {};
    how.gridDim = dim3((unsigned)std::min((i64)sms, most * keys.Hq));
    how.blockDim = dim3(ATTEND_THREADS);
    how.dynamicSmemBytes = sq;
    how.stream = stream;
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    how.attrs = &early; how.numAttrs = 1;
    RP_CUDA(cudaLaunchKernelEx(&how, k_attend_queries<X, D>, M.k, M.v, (const GradArgs)queries));
    return rp_op_launched();
}

extern "C" int rp_attend_grad(const rp_attend_config *a, int64_t n_tokens, const rp_view *q, const rp_view *k, const rp_view *v, const rp_view *out,
                              const rp_view *lse, const rp_view *out_grad, const int64_t *start, int32_t n_samples, const rp_view *q_grad,
                              const rp_view *k_grad, const rp_view *v_grad, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    RP_TRY(rp_attend_check(a, n_tokens, n_samples));
    if (!start || !rp_aligned(start, 8) || !workspace || !rp_aligned(workspace, 16) || workspace_bytes < rp_attend_grad_workspace(a, n_tokens, n_samples)) return RP_ERR_ARG;
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
    const i64 T = n_tokens, plan = plan_bytes(T, n_samples);
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
        P[w].start = (const i64 *)start; P[w].T = T; P[w].N = n_samples; P[w].rows = 128; P[w].causal = a->causal; P[w].most = (int)(T / 128 + n_samples);
        P[w].by_key = w == 0; P[w].head = head[w]; P[w].items = (int2 *)(head[w] + 1);
        GradArgs &A = G[w];
        A = GradArgs();
        A.items = P[w].items; A.head = head[w]; A.start = (const i64 *)start; A.T = T; A.Hq = Hq; A.Hk = Hk; A.share = Hq / Hk; A.d = d; A.causal = a->causal;
        A.scale = a->scale; A.stats = stats; A.status = &head[0]->status; A.wait_ns = (u64)g_attend_wait_ns;
    }
    G[0].x[0] = v_grad->x; G[0].token[0] = v_grad->token; G[0].hd[0] = v_grad->head;
    G[0].x[1] = k_grad->x; G[0].token[1] = k_grad->token; G[0].hd[1] = k_grad->head;
    G[1].rows[0] = q->x; G[1].r_token[0] = q->token; G[1].r_head[0] = q->head;
    G[1].rows[1] = out_grad->x; G[1].r_token[1] = out_grad->token; G[1].r_head[1] = out_grad->head;
    G[1].x[0] = q_grad->x; G[1].token[0] = q_grad->token; G[1].hd[0] = q_grad->head;
    const int sms = rp_op_sms(dev.device);
    float *const norms = (float *)(stats + T * Hq);
    u32 *const tops = (u32 *)(norms + T * Hq);           // (float16)
    G[0].tops = G[1].tops = tops;
    const StatsArgs S = { out->x, out_grad->x, (const float *)lse->x, out->token, out->head, out_grad->token, out_grad->head, lse->token, lse->head, Hq, d, stats, norms, tops };
    const int ctas = 2 + (int)std::min((T * Hq + 63) / 64, (i64)sms * 2 - 2);
    if (a->type == RP_F16) {
        k_attend_prepare<__half><<<ctas, 1024, 0, stream>>>(P[0], P[1], C, S);
        RP_TRY(rp_op_launched());
        k_attend_tops<<<(unsigned)((T + 255) / 256), 256, 0, stream>>>((const i64 *)start, n_samples, T, Hq, norms, tops);
    }
    else k_attend_prepare<bf16><<<ctas, 1024, 0, stream>>>(P[0], P[1], C, S);
    RP_TRY(rp_op_launched());
    if (a->type == RP_F16) return d <= 64 ? launch<__half, 64>(M, G[0], G[1], P[0].most, sms, stream) : launch<__half, 128>(M, G[0], G[1], P[0].most, sms, stream);
    return d <= 64 ? launch<bf16, 64>(M, G[0], G[1], P[0].most, sms, stream) : launch<bf16, 128>(M, G[0], G[1], P[0].most, sms, stream);
}
