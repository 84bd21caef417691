// Attention of one new token of each sequence against the keys and values of those before it (decoding).
//
//   s = scale q k^T over the keys that the token sees, o = softmax(s) v, lse = log sum exp(s)
//
// Bound by HBM: each visible key and value is read once (for more than 16 query heads to a key head once for every 16, by neighbouring warps), 4 * head_dim bytes for
// 4 * share * head_dim operations (share: query heads to a key head).  The products go
// through the warps' matrix instruction, 16 rows by 8 keys at a time, of which `share` are something: with a few rows to a tile there is nothing that fuller
// instructions could add.
// The keys that a sequence's token sees are cut into as many chunks as there are 128s in them, 128 at most; a chunk and a key head are a unit of one warp, which takes them in
// tiles of 4 KB (16 keys of 128) through a ring of its own in shared memory.  Of n chunks each has every n-th tile, so that warps side by side read what lies side by side
// (1000 sequences of 1000 keys, 2 GB: 346 us, 392 with chunks in whole pieces).  Warps stay resident and take units in
// turn, and the ring runs on into the next unit; no warp waits for another.  The cut goes by the sequence alone, so that its bits do not depend on the others of the
// batch.  A second kernel adds up the chunks, in their order.
// 64 ragged sequences, 16 heads on 4, 128 wide (643 MB): 108 us, 91 % of the measured copy rate; 250 with a window of 1000, 8 heads of 64 (445 MB) 83 us, 81 %; 1000 of 1000 keys
// (2 GB) 327 us, 96 %; four of up to 6000 keys (52 MB) 16.8 us, where the tiles of a chunk, one after the other, take as long as the launches.  Cut by 192: 110, 81, 318 and 18.6 us.
// A sequence has 128 chunks at most, for which the second kernel has lanes, so one long cache with few key heads leaves warps without work: a sequence of 131072 keys, 128 wide,
// takes 60 us with one key head or two (67 and 134 MB, 1.1 and 2.2 TB/s), 82 with eight (6.5 TB/s); one of 1048576 with one key head 413.
#include <algorithm>
#include <climits>

#include "rp_attend.cuh"

#define STEP_WARPS 4
#define STEP_THREADS (32 * STEP_WARPS)
#define STEP_CHUNK 128                   // keys of a chunk at least, where there are several
#define STEP_CHUNKS 128                  // chunks of a sequence at most
#define STEP_ROWS 16                     // query heads of a unit at most

#define STEP_TABLE 32                    // sequences whose places a warp works out for itself: a launch less (four sequences 17.5 us for 18.9; by more than a lane each it is slower, 64 of them 115 for 112)

struct StepHead { int status, pad[3]; };
struct StepPlan {
    const i64 *start, *length;
    i64 T;
    int N, window, sinks, most, tile;        // most: room for chunks; tile: keys that a warp takes at a time
    int *from;                               // [N + 1] chunks of the sequences before, when there are many
    int2 *place;                             // [N] first row, rows that are filled
};
// Rows of a sequence, and how they are cut: the first `ahead` ones, their number rounded up to whole tiles, then those from `first` on.
__device__ __forceinline__ int2 step_place(const StepPlan &P, int i)
{
    const i64 from = max(P.start[i], (i64)0), room = max(min(P.start[i + 1], P.T) - from, (i64)0);
    return make_int2((int)min(from, P.T), (int)(P.length ? min(max(P.length[i], (i64)0), room) : room));          // (rows: less than 2^31)
}
struct StepSeen {
    int ahead, first, seen, n;               // n: chunks, of which each has every n-th tile
    __device__ __forceinline__ StepSeen(const StepPlan &P, int filled)
    {
        first = P.window ? max(filled - P.window, 0) : 0;
        ahead = min(P.sinks, first);
        seen = ((ahead + P.tile - 1) & -P.tile) + filled - first;
        n = min(max(seen / STEP_CHUNK, 1), STEP_CHUNKS);         // (one without keys as well: it writes the outputs)
    }
};

// More sequences than a warp has lanes for, or none long enough for the second kernel: counts the chunks before each.
__global__ void __launch_bounds__(1024) k_step_plan(StepPlan P, StepHead *head)
{
    rp_let_next_launch_start();
    __shared__ int sums[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int total = 0;
    for (int i0 = 0; i0 < P.N; i0 += 1024) {
        const int i = i0 + threadIdx.x;
        int n = 0;
        if (i < P.N) {
            const int2 place = step_place(P, i);
            P.place[i] = place;
            n = StepSeen(P, place.y).n;
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
        if (i < P.N) P.from[i] = total + before + x - n;
        __syncthreads();
        total += all;
    }
    if (threadIdx.x == 0) { P.from[P.N] = total; head->status = 0; }
}

struct StepArgs {
    StepPlan plan;
    bool table, keys;                        // table: a warp works out the places for itself; keys: is there a cache at all?
    int2 *where;                             // [N] first item and number of items, for the second kernel
    int Hq, share, groups, d, units;         // groups: of 16 query heads to a key head; units: of a chunk
    float scale;
    const void *q;
    i64 q_token, q_head;
    void *out;
    i64 o_token, o_head;
    float *lse;
    i64 l_token, l_head;
    float2 *tops;                            // [item][Hq] maximum and sum of a chunk
    float *parts;                            // [item][Hq][d] its values
    StepHead *head;
    int *states;                             // of the CTAs: whether a wait ran out
    int ctas, each;                          // each: query heads that a CTA of the second kernel takes at a time
    u64 wait_ns;
};

__device__ __forceinline__ void load_matrices(u32 at, u32 *r)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_matrices_across(u32 at, u32 *r)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
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

// Places x0, x0 + stride, .. before x1 of the keys that a token sees, a tile at each.
struct StepItem { int base, sample, chunks, x0, x1, ahead, first, stride; };
struct StepTable {
    const int *from;
    const int2 *place;
    int step, coarse;                        // a 32nd of the sequences to a lane: chunks before its first one
    int2 own;                                // with one sequence to a lane, its place
    // Chunk c of the call: the last sequence that has none behind it.  By a warp, which looks at 32 sequences at a time.
    __device__ __forceinline__ StepItem item(const StepPlan &P, int c) const
    {
        const int lane = threadIdx.x & 31, head = max(__popc(__ballot_sync(0xffffffffu, coarse <= c)) - 1, 0);
        int lo = head * step, n = min(step, P.N - lo), before = __shfl_sync(0xffffffffu, coarse, head);
        int2 at = make_int2(__shfl_sync(0xffffffffu, own.x, head), __shfl_sync(0xffffffffu, own.y, head));
        if (step > 1) {
            while (n > 1) {
                const int some = (n + 31) >> 5;
                const u32 hit = __ballot_sync(0xffffffffu, lane * some < n && from[lo + lane * some] <= c);
                const int skip = max(__popc(hit) - 1, 0) * some;
                lo += skip;
                n = min(some, n - skip);
            }
            before = from[lo];
            at = place[lo];
        }
        const StepSeen S(P, at.y);
        StepItem it;
        it.base = at.x; it.sample = lo; it.chunks = S.n; it.x0 = (c - before) * P.tile; it.x1 = S.seen; it.stride = S.n * P.tile;
        it.ahead = S.ahead; it.first = S.first;
        return it;
    }
};
// K and V pass through once: they go out of L2 before what the second kernel reads.
__device__ __forceinline__ u64 passing()
{
    u64 p;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ void tma_load3_passing(u32 dst, const CUtensorMap *map, int x, int y, int z, u32 bar, u64 policy)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4}], [%5], %6;"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy) : "memory");
}

// A tile is 4 KB of keys and as many of values.  Two of them for a warp, 64 KB a CTA and two CTAs to an SM; more under way make the reads slower (three: 64 sequences 111 us for
// 108, 1000 of 1000 keys 346 for 327).
template <int D> struct StepSmem {
    static constexpr int KEYS = 2048 / D, TILE = 4096, STAGES = 2;
    alignas(1024) unsigned char ring[STEP_WARPS][STAGES][2][TILE];
    u64 full[STEP_WARPS][STAGES];
    Waits waits;
};

// FEW: eight query heads at most, whose places the instruction's other eight rows give the weights' lower halves.
template <typename X, int D, bool FEW>
__global__ void __launch_bounds__(STEP_THREADS, 2)
k_attend_step(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const StepArgs A)
{
    typedef StepSmem<D> Smem;
    constexpr int STAGES = Smem::STAGES, PANELS = D / 64, KEYS = Smem::KEYS, PANEL = KEYS * 128, NT = D / 8, KS = D / 16, NK = KEYS / 8, R = FEW ? 1 : 2;
    constexpr float LIFT = std::is_same<X, bf16>::value ? 1.0f : 32768.0f;            // float16: weights of 1 as 2^15, so that small ones stay something
    extern __shared__ __align__(1024) unsigned char raw[];
    Smem &sm = *(Smem *)(raw + ((1024 - (rp_smem(raw) & 1023)) & 1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const u32 ring = rp_smem(sm.ring[warp]), full = rp_smem(sm.full[warp]);
    Waits *const waits = &sm.waits;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STEP_WARPS * STAGES; ++i) bar_init(rp_smem(&sm.full[0][0]) + 8 * i, 1);
        waits->start(A.wait_ns);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (A.keys) { tma_prefetch(&map_k); tma_prefetch(&map_v); }
    }
    __syncthreads();
    rp_let_next_launch_start();
    rp_wait_for_launch_before();
    const int N = A.plan.N;
    StepTable table = { A.plan.from, A.plan.place, (N + 31) >> 5, INT_MAX, make_int2(0, 0) };
    int chunks;
    if (A.table) {
        int n = 0;
        if (lane < N) {
            table.own = step_place(A.plan, lane);
            n = StepSeen(A.plan, table.own.y).n;
        }
        int x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        chunks = __shfl_sync(0xffffffffu, x, 31);
        if (lane < N) {
            table.coarse = x - n;
            if (blockIdx.x == 0 && warp == 0) A.where[lane] = make_int2(x - n, x <= A.plan.most ? n : 0);
        }
    } else {
        chunks = table.from[N];
        if (lane * table.step < N) table.coarse = table.from[lane * table.step];
        if (table.step == 1 && lane < N) table.own = table.place[lane];
        if (A.where)
            for (int i = blockIdx.x * STEP_THREADS + threadIdx.x; i < N; i += gridDim.x * STEP_THREADS) {
                const int at = table.from[i], n = table.from[i + 1] - at;
                A.where[i] = make_int2(at, at <= A.plan.most - n ? n : 0);
            }
    }
    const int total = min(chunks, A.plan.most) * A.units, mine = blockIdx.x * STEP_WARPS + warp, step = gridDim.x * STEP_WARPS;
    const float sl = A.scale * RP_LOG2E;
    const u64 policy = passing();

    // The tiles that the warp copies, in the order in which it takes them.
    int unit_in = mine, at = 0, hk_in = 0;
    StepItem to;
    u32 copied = 0;
    auto open = [&]() {                                  // the next unit with keys
        for (; unit_in < total; unit_in += step) {
            to = table.item(A.plan, unit_in / A.units);
            at = to.x0;
            hk_in = unit_in % A.units / A.groups;
            if (to.x0 < to.x1) break;
        }
    };
    open();
    StepItem it = { }, next = { };
    const auto item = [&](int unit) { return unit == unit_in ? to : table.item(A.plan, unit / A.units); };          // (mostly the one that is being copied)
    if (mine < total) it = item(mine);
    auto copy = [&](int stage) {                         // the next tile, if there is one
        // (the warp's answer, not each lane's: another warp may give up at any time, and all 32 lanes look for the next unit together)
        if (unit_in >= total || __any_sync(0xffffffffu, waits->gave_up)) return;
        if (lane == 0) {
            const int whole = (to.ahead + KEYS - 1) & ~(KEYS - 1), row = to.base + (at < whole ? at : to.first + at - whole);
            const u32 dst = ring + stage * 2 * Smem::TILE, bar = full + 8 * stage;
            bar_expect(bar, 2 * Smem::TILE);
            for (int p = 0; p < PANELS; ++p) {
                tma_load3_passing(dst + p * PANEL, &map_k, p * 64, hk_in, row, bar, policy);
                tma_load3_passing(dst + Smem::TILE + p * PANEL, &map_v, p * 64, hk_in, row, bar, policy);
            }
        }
        ++copied;
        if (to.x1 - at <= to.stride) { unit_in += step; open(); }
        else at += to.stride;
    };
    for (int s = 0; s < STAGES; ++s) copy(s);

    u32 q[KS][2 * R];
    auto load_q = [&](int unit, int sample) {
        if (unit >= total) return;
        const int hg = unit % A.units, first = hg % A.groups * STEP_ROWS, rows = min(A.share - first, STEP_ROWS);
        const X *from = (const X *)A.q + sample * A.q_token + (hg / A.groups * A.share + first) * A.q_head;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int i = 0; i < 2 * R; ++i) {
                const int r = g + i % R * 8, c = s * 16 + t * 2 + i / R * 8;
                q[s][i] = r < rows && c < A.d ? *(const u32 *)(from + r * A.q_head + c) : 0u;
            }
    };
    load_q(mine, it.sample);
    auto look = [&](int unit) {                          // the next unit, and its queries
        if (unit >= total) return;
        next = item(unit);
        load_q(unit, next.sample);
    };
    u32 taken = 0;
    int stage = 0;
    for (int unit = mine; unit < total; unit += step, it = next) {
        const int hg = unit % A.units, hk = hg / A.groups, h0 = hk * A.share + hg % A.groups * STEP_ROWS, rows = min(A.share - hg % A.groups * STEP_ROWS, STEP_ROWS);
        const int whole = (it.ahead + KEYS - 1) & ~(KEYS - 1);
        float o[NT][4], m[2] = { -INFINITY, -INFINITY }, l[2] = { 0.0f, 0.0f };
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][i] = 0.0f;
        bool ok = true;
        for (int x = it.x0, last = it.x0 >= it.x1; !last; x += it.stride) {
            if (!(ok = bar_wait_warp(full + 8 * stage, taken / STAGES & 1, waits))) break;
            ++taken;
            last = it.x1 - x <= it.stride;
            const u32 kt = ring + stage * 2 * Smem::TILE, vt = kt + Smem::TILE;
            const int there = min(x < whole ? it.ahead - x : it.x1 - x, KEYS);           // keys of the tile; behind them may be anything
            float s[NK][4] = { };
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const u32 a[4] = { q[ks][0], FEW ? 0u : q[ks][1], q[ks][R], FEW ? 0u : q[ks][2 * R - 1] };
#pragma unroll
                for (int n = 0; n < NK; n += 2) {
                    u32 b[4];
                    const int r = n * 8 + (lane >> 4) * 8 + (lane & 7), p = 2 * ks + ((lane >> 3) & 1);
                    load_matrices(kt + (p >> 3) * PANEL + r * 128 + (((p & 7) ^ (r & 7)) << 4), b);
                    rp_multiply(s[n], a, b, X());
                    rp_multiply(s[n + 1], a, b + 2, X());
                }
            }
            if (last) look(unit + step);        // while this one is finished
            float top[R];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                top[i] = m[i];
#pragma unroll
                for (int n = 0; n < NK; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        s[n][2 * i + j] = n * 8 + t * 2 + j < there ? s[n][2 * i + j] * sl : -INFINITY;
                        top[i] = fmaxf(top[i], s[n][2 * i + j]);
                    }
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
            }
            if (__any_sync(0xffffffffu, top[0] > m[0] || top[R - 1] > m[R - 1])) {
                float f[R];
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    f[i] = top[i] == m[i] ? 1.0f : rp_exp2(m[i] - top[i]);
                    l[i] *= f[i];
                    m[i] = top[i];
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[n][i] *= f[i / 2 % R];
            }
            u32 high[NK][R], low[NK][R];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float less = m[i] == -INFINITY ? 0.0f : m[i];
#pragma unroll
                for (int n = 0; n < NK; ++n) {
                    const float a = rp_exp2(s[n][2 * i] - less), b = rp_exp2(s[n][2 * i + 1] - less);
                    l[i] += a + b;
                    two_pairs<X>(a * LIFT, b * LIFT, high[n][i], low[n][i]);
                }
            }
            const auto values = [&](auto part) {
#pragma unroll
                for (int kk = 0; kk < NK; kk += 2) {
                    u32 keep[2] = { 0xffffffffu, 0xffffffffu };      // values behind the keys are cleared: 0 times NaN would not be 0
                    if constexpr (decltype(part)::value) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int n = there - (kk * 8 + i * 8 + t * 2);
                            keep[i] = n >= 2 ? 0xffffffffu : n == 1 ? 0xffffu : 0u;
                        }
                    }
                    const u32 a[4] = { high[kk][0], FEW ? low[kk][0] : high[kk][R - 1], high[kk + 1][0], FEW ? low[kk + 1][0] : high[kk + 1][R - 1] };
                    const u32 rest[4] = { low[kk][0], low[kk][R - 1], low[kk + 1][0], low[kk + 1][R - 1] };
#pragma unroll
                    for (int n = 0; n < NT; n += 2) {
                        u32 b[4];
                        const int r = kk * 8 + ((lane >> 3) & 1) * 8 + (lane & 7), p = n + (lane >> 4);
                        load_matrices_across(vt + (p >> 3) * PANEL + r * 128 + (((p & 7) ^ (r & 7)) << 4), b);
                        if constexpr (decltype(part)::value) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) b[i] &= keep[i & 1];
                        }
                        rp_multiply(o[n], a, b, X());
                        rp_multiply(o[n + 1], a, b + 2, X());
                        if (!FEW) { rp_multiply(o[n], rest, b, X()); rp_multiply(o[n + 1], rest, b + 2, X()); }
                    }
                }
            };
            if (there < KEYS) values(std::true_type()); else values(std::false_type());
            __syncwarp();
            copy(stage);
            stage = stage + 1 == STAGES ? 0 : stage + 1;
        }
        if (it.x0 >= it.x1 || !ok) look(unit + step);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
            if (!ok || waits->gave_up) { l[i] = NAN; m[i] = 0.0f; }
        }
        if (FEW) {
#pragma unroll
            for (int n = 0; n < NT; ++n) { o[n][0] += o[n][2]; o[n][1] += o[n][3]; }
        }
        const int item = unit / A.units;
#pragma unroll
        for (int i = 0; i < R; ++i) {
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
            const bool none = it.x1 <= it.x0 && l[i] == 0.0f;        // no key at all: nothing, and the log of nothing
            const float f = none ? 0.0f : 1.0f / (l[i] * LIFT);
            X *out = (X *)A.out + it.sample * A.o_token + h * A.o_head;
#pragma unroll
            for (int n = 0; n < NT; ++n)
                if (n * 8 < A.d) *(u32 *)(out + n * 8 + t * 2) = rp_pair(o[n][2 * i] * f, o[n][2 * i + 1] * f, X());
            if (t == 0 && A.lse) A.lse[it.sample * A.l_token + h * A.l_head] = none ? -INFINITY : (m[i] + log2f(l[i])) * 0.6931471805599453f;
        }
        __syncwarp();
    }
    // nobody may leave while copies are under way (whoever should have waited for them may have given up)
    for (u32 f = taken; f < copied; ++f) rp_drain(full + 8 * (f % STAGES), f / STAGES & 1);
    __syncthreads();
    if (threadIdx.x == 0) {
        if (A.where) A.states[blockIdx.x] = waits->gave_up;
        else if (waits->gave_up) A.head->status = RP_ERR_TIMEOUT;
    }
}

// Sequences of several chunks: up to STEP_FEW of them are added up by a warp, more by a CTA, each warp every fourth one; a lane has four columns.  Which of the two goes by the
// sequence alone.  (1000 sequences of three chunks, 16 heads: 10 us behind the first kernel, 34 with a CTA for each query head.)
#define STEP_FEW 16
// Chunks first, first + every, .. of a sequence and query head (`mine` of them, 32 at most): their sums, with their largest maximum as it was or a larger one.
struct StepSum {
    float top, sum;
    float4 o;
    template <typename Top>
    __device__ __forceinline__ StepSum(const StepArgs &A, i64 first, int every, int mine, int h, int lane, const Top &top_of)
    {
        const int e = lane * 4;
        const float2 y = lane < mine ? A.tops[(first + every * lane) * A.Hq + h] : make_float2(-INFINITY, 0.0f);
        const float *from = A.parts + (first * A.Hq + h) * A.d + (e < A.d ? e : 0);
        const i64 step = (i64)every * A.Hq * A.d;
        constexpr int AHEAD = 8;
        float4 z[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) z[u] = u < mine ? *(const float4 *)(from + u * step) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        top = y.x;
#pragma unroll
        for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        top = top_of(top);
        const float f = y.x == top ? 1.0f : rp_exp2(y.x - top);
        sum = lane < mine ? y.y * f : 0.0f;
#pragma unroll
        for (int x = 16; x; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
        o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int c0 = 0; c0 < mine; c0 += AHEAD) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const float w = __shfl_sync(0xffffffffu, f, (c0 + u) & 31);
                if (c0 + u < mine) { o.x = fmaf(z[u].x, w, o.x); o.y = fmaf(z[u].y, w, o.y); o.z = fmaf(z[u].z, w, o.z); o.w = fmaf(z[u].w, w, o.w); }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (c0 + AHEAD + u < mine) z[u] = *(const float4 *)(from + (c0 + AHEAD + u) * step);
        }
    }
};
template <typename X>
__global__ void __launch_bounds__(STEP_THREADS) k_step_join(const StepArgs A)
{
    constexpr float LIFT = std::is_same<X, bf16>::value ? 1.0f : 32768.0f;
    static_assert(STEP_CHUNKS <= 32 * STEP_WARPS && STEP_FEW <= 32, "a lane for each chunk of a warp");
    __shared__ float4 part[STEP_WARPS][32];
    __shared__ float tops[STEP_WARPS], sums[STEP_WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = lane * 4;
    rp_wait_for_launch_before();
    if (blockIdx.x == 0) {
        int late = 0;
        for (int i = threadIdx.x; i < A.ctas; i += STEP_THREADS) late |= A.states[i];
        late = __syncthreads_or(late);
        if (threadIdx.x == 0) A.head->status = late ? RP_ERR_TIMEOUT : RP_OK;
    }
    const auto hand_out = [&](int sample, int h, float top, float sum, const float4 &o) {
        const float g = 1.0f / (sum * LIFT);
        if (e < A.d) *(uint2 *)((X *)A.out + sample * A.o_token + h * A.o_head + e) = make_uint2(rp_pair(o.x * g, o.y * g, X()), rp_pair(o.z * g, o.w * g, X()));
        if (lane == 0 && A.lse) A.lse[sample * A.l_token + h * A.l_head] = (top + log2f(sum)) * 0.6931471805599453f;
    };
    // `each` query heads (of one sequence or of neighbouring ones) at a time
    const i64 units = (i64)A.plan.N * A.Hq;
    for (i64 u0 = (i64)blockIdx.x * A.each; u0 < units; u0 += (i64)gridDim.x * A.each) {
        const i64 unit = u0 + warp;
        const int sample = (int)(unit / A.Hq), h = (int)(unit % A.Hq);
        const int2 at = warp < A.each && unit < units ? A.where[sample] : make_int2(0, 0);
        if (at.y > 1 && at.y <= STEP_FEW) {
            const StepSum s(A, at.x, 1, at.y, h, lane, [](float top) { return top; });
            hand_out(sample, h, s.top, s.sum, s.o);
        }
        if (!__syncthreads_or(at.y > STEP_FEW)) continue;
        for (int v = 0; v < A.each && u0 + v < units; ++v) {
            const int sample = (int)((u0 + v) / A.Hq), h = (int)((u0 + v) % A.Hq);
            const int2 at = A.where[sample];
            if (at.y <= STEP_FEW) continue;
            const StepSum s(A, at.x + warp, STEP_WARPS, (at.y - warp + STEP_WARPS - 1) / STEP_WARPS, h, lane, [&](float top) {
                if (lane == 0) tops[warp] = top;
                __syncthreads();
                for (int w = 0; w < STEP_WARPS; ++w) top = fmaxf(top, tops[w]);
                return top;
            });
            part[warp][lane] = s.o;
            if (lane == 0) sums[warp] = s.sum;
            __syncthreads();
            if (warp == 0) {
                float sum = 0.0f;
                float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int w = 0; w < STEP_WARPS; ++w) {
                    const float4 a = part[w][lane];
                    o.x += a.x; o.y += a.y; o.z += a.z; o.w += a.w;
                    sum += sums[w];
                }
                hand_out(sample, h, s.top, sum, o);
            }
            __syncthreads();
        }
    }
}

// ---------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------
struct StepSpace { i64 states, from, place, where, tops, parts, all; };
static int step_units(const rp_attend_config *a) { return a->kv_heads * ((a->q_heads / a->kv_heads + STEP_ROWS - 1) / STEP_ROWS); }
static i64 step_most(i64 T, int N, int window, int sinks)
{
    i64 each = STEP_CHUNKS;
    if (window) each = std::min(each, std::max(((i64)window + sinks + 31) / STEP_CHUNK, (i64)1));
    return std::min((T + 31ll * N) / STEP_CHUNK + N, N * each);
}
static bool step_several(i64 T, int window, int sinks) { return T + 31 >= 2 * STEP_CHUNK && (!window || (i64)window + sinks + 31 >= 2 * STEP_CHUNK); }
#define STEP_MOST_CTAS 512                               // (two on each of 148 SMs)
static StepSpace step_space(const rp_attend_config *a, i64 T, int N, int window, int sinks)
{
    const i64 most = step_most(T, N, window, sinks);
    const auto up = [](i64 x) { return (x + 15) / 16 * 16; };
    StepSpace s;
    s.states = sizeof(StepHead);
    s.from = s.states + 4 * STEP_MOST_CTAS;
    s.place = up(s.from + 4ll * (N + 1));
    s.where = s.place + 8ll * N;
    s.tops = up(s.where + 8ll * N);
    s.parts = up(s.tops + most * a->q_heads * 8);
    s.all = s.parts + most * a->q_heads * a->head_dim * 4;
    return s;
}
static int check_step(const rp_attend_config *a, int window, int sinks, i64 T, int N)
{
    RP_TRY(rp_attend_check(a, T, N));
    if (window < 0 || sinks < 0) return RP_ERR_ARG;
    return (T / 64 + 2ll * N) * a->q_heads >= (1ll << 31) ? RP_ERR_RANGE : RP_OK;             // (units are counted in 32 bits, and step_most() of them are less than T / 128 + 1.25 N)
}

extern "C" int64_t rp_attend_step_workspace(const rp_attend_config *a, int32_t window, int32_t sinks, int64_t n_tokens, int32_t n_samples)
{
    return check_step(a, window, sinks, n_tokens, n_samples) == RP_OK ? step_space(a, n_tokens, n_samples, window, sinks).all : 0;
}

template <typename X, int D, bool FEW>
static int launch(const CUtensorMap &k, const CUtensorMap &v, StepArgs &A, i64 units, int sms, cudaStream_t stream)
{
    const size_t smem = sizeof(StepSmem<D>) + 1024;
    RP_CUDA(cudaFuncSetAttribute(k_attend_step<X, D, FEW>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    A.ctas = (int)std::min(std::min((i64)sms * 2, (i64)STEP_MOST_CTAS), (units + STEP_WARPS - 1) / STEP_WARPS);
    cudaLaunchConfig_t how = {};
    how.gridDim = dim3((unsigned)A.ctas);
    how.blockDim = dim3(STEP_THREADS);
    how.dynamicSmemBytes = smem;
    how.stream = stream;
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    how.attrs = &early; how.numAttrs = A.table ? 0 : 1;                  // (behind the plan)
    RP_CUDA(cudaLaunchKernelEx(&how, k_attend_step<X, D, FEW>, k, v, (const StepArgs)A));
    RP_TRY(rp_op_launched());
    if (!A.where) return RP_OK;
    // (As many CTAs as there are query heads, while all of them are resident; of more a warp takes one.)
    const i64 joins = (i64)A.plan.N * A.Hq;
    A.each = joins > (i64)sms * 16 ? STEP_WARPS : 1;
    how.gridDim = dim3((unsigned)std::min((i64)sms * 16, (joins + A.each - 1) / A.each));
    how.dynamicSmemBytes = 0;
    how.numAttrs = 1;
    RP_CUDA(cudaLaunchKernelEx(&how, k_step_join<X>, (const StepArgs)A));
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
    const bool several = step_several(n_tokens, window, sinks);
    const int tile = a->head_dim <= 64 ? StepSmem<64>::KEYS : StepSmem<128>::KEYS;
    StepArgs A = {};
    StepPlan &P = A.plan;
    P.start = (const i64 *)start; P.length = (const i64 *)length; P.T = n_tokens; P.N = N; P.window = window; P.sinks = sinks;
    P.most = (int)step_most(n_tokens, N, window, sinks); P.tile = tile; P.from = (int *)(w + space.from); P.place = (int2 *)(w + space.place);
    A.table = several && N <= STEP_TABLE;
    A.where = several ? (int2 *)(w + space.where) : nullptr;
    A.head = (StepHead *)w; A.states = (int *)(w + space.states);
    CUtensorMap mk = {}, mv = {};
    if (n_tokens) {
        RP_TRY(rp_tensor_map(&mk, a->type, k->x, n_tokens, a->kv_heads, a->head_dim, k->token, k->head, tile));
        RP_TRY(rp_tensor_map(&mv, a->type, v->x, n_tokens, a->kv_heads, a->head_dim, v->token, v->head, tile));
    }
    if (!A.table) {
        k_step_plan<<<1, 1024, 0, stream>>>(P, A.head);
        RP_TRY(rp_op_launched());
    }
    A.Hq = a->q_heads; A.share = a->q_heads / a->kv_heads; A.units = step_units(a); A.groups = A.units / a->kv_heads; A.d = a->head_dim; A.scale = a->scale;
    A.q = q->x; A.q_token = q->token; A.q_head = q->head; A.out = out->x; A.o_token = out->token; A.o_head = out->head; A.keys = n_tokens > 0;
    if (lse && lse->x) { A.lse = (float *)lse->x; A.l_token = lse->token; A.l_head = lse->head; }
    A.tops = (float2 *)(w + space.tops); A.parts = (float *)(w + space.parts);
    A.wait_ns = (u64)g_attend_wait_ns;
    const int sms = rp_op_sms(dev.device);
    const i64 units = (i64)P.most * A.units;
    // Up to eight query heads of a key head: half the exponentials and half the products with values (64 ragged sequences of 16 heads on 4: 131 us for 138).
    const bool few = A.share <= 8, narrow = a->head_dim <= 64;
    const auto go = [&](auto type) {
        typedef decltype(type) X;
        if (narrow) return few ? launch<X, 64, true>(mk, mv, A, units, sms, stream) : launch<X, 64, false>(mk, mv, A, units, sms, stream);
        return few ? launch<X, 128, true>(mk, mv, A, units, sms, stream) : launch<X, 128, false>(mk, mv, A, units, sms, stream);
    };
    return a->type == RP_F16 ? go(__half()) : go(bf16());
}
