// Attention with a sliding window inside the samples of a packed row, forward.
//
//   s = scale q k^T over the tokens j <= i of a sample with i - j < window or j < sinks, p = exp(s - m), o = p v / sum p, lse = m + log sum p, m a running maximum
//
// As the attention without a window: two tiles of 128 queries of a head to a CTA, a group of four warps with the softmax of each, scores, weights and outputs in tensor
// memory.  But a block has few tiles of keys (ten at a window of 1024), so what happens between blocks counts: nothing starts anew there.  Keys and values go through
// one ring, whose stages hold the values of one step and the keys of the next, across the blocks' ends; each tile's queries are copied as soon as its last scores are
// there, by a warp of their own; one warp looks up the blocks to come; and the products of a block begin while the one before is handed over.
// From where the window has left a sample's first token behind, tiles of which some rows see nothing are taken last (AttendOrder).  First tokens that the window has left
// behind are a step of their own, as narrow as they are.  Head sizes between 64 and 128 are worked on as 128 columns, the ones behind head_dim zeros: a head of 96 costs what
// one of 128 does.
// Bound by the hand-overs between the softmax and the products of a tile, with two tiles in turn, and by what a block costs beside its tiles: a tile of 128 keys adds 0.95 us
// at head_dim 128, of which the tensor cores need 1024 cycles, and a block 4 to 5 us more - the tiles of which each row sees a part, the last products, the handing over.
// 32768 tokens of one sample, 16 heads on 4, 128 wide: 125 us with a window of 128, 298 with 1024 (907 TFLOP/s of what is seen; 339 with 4 first tokens), 925 with 4096
// (1115).  Tried without gain: a warp for each tile's products, weights handed over in halves, queries of two blocks in shared memory at head_dim 64.
#include <algorithm>

#include "rp_attend.cuh"

#define ATTEND_LIST_WARP 11

// Parts of the two tiles in a step, for the warp that issues products: a tile takes part, it is the last step of its block, it is not the first; for both, the keys are the
// first tokens.  A stage's word has these for its values' step, 8 bits on for its keys', and 16 bits on how many of its values are the sample's.
enum : u32 { STEP_TAKES = 1, STEP_LAST = 4, STEP_MORE = 16, STEP_FEW = 64, STEP_END = 128 };

template <int D> struct WindowSmem {
    static constexpr int TILE = 128 * D * 2, STAGES = D == 128 ? 2 : 4;
    alignas(1024) unsigned char q[2][TILE];
    alignas(1024) unsigned char v[STAGES][TILE];
    alignas(1024) unsigned char k[STAGES][TILE];
    alignas(16) unsigned char rows[8][4096];            // of each warp, 64 columns of what it hands over
    u64 q_full[2], q_empty[2], kv_full[STAGES], kv_empty[STAGES], s_full[2], p_full[2], o_full[2], block_full[2], block_empty[2], done;
    u32 tmem;
    alignas(16) volatile int block[2][4];               // blocks to come: the item, its sample's first row and length, its own first row
    volatile u32 step[STAGES];                          // of a stage: what the products go by
    Waits waits;
};

template <typename X, int D>
__global__ void __launch_bounds__(ATTEND_THREADS, 1)
k_attend_window(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const AttendArgs A)
{
    typedef WindowSmem<D> Smem;
    constexpr int STAGES = Smem::STAGES, PANELS = D / 64, PANEL = 128 * 128;
    // Weights of float16 times 2^7, up to 2^15 with what a maximum may lag behind: small ones stay something.
    constexpr float LIFT = std::is_same<X, bf16>::value ? 0.0f : 7.0f;
    extern __shared__ __align__(1024) unsigned char raw[];
    Smem &sm = *(Smem *)(raw + ((1024 - (rp_smem(raw) & 1023)) & 1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { bar_init(rp_smem(&sm.kv_full[s]), 1); bar_init(rp_smem(&sm.kv_empty[s]), 1); }
        for (int i = 0; i < 2; ++i) {
            bar_init(rp_smem(&sm.q_full[i]), 1); bar_init(rp_smem(&sm.q_empty[i]), 1);
            bar_init(rp_smem(&sm.s_full[i]), 1); bar_init(rp_smem(&sm.p_full[i]), 4); bar_init(rp_smem(&sm.o_full[i]), 1);
            bar_init(rp_smem(&sm.block_full[i]), 1); bar_init(rp_smem(&sm.block_empty[i]), 9);
        }
        bar_init(rp_smem(&sm.done), 1);
        sm.waits.start(A.wait_ns);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == ATTEND_COPY_WARP) tmem_alloc(rp_smem(&sm.tmem), 512);
    tmem_before();
    __syncthreads();
    tmem_after();
    const u32 tm = rp_uniform(sm.tmem);
    rp_wait_for_launch_before();             // the list of blocks: nothing of it before this line
    const int total = rp_uniform(A.head->count * A.Hq);
    Waits *const waits = &sm.waits;

    if (warp >= 8) {
        rp_few_registers();
        if (warp == ATTEND_LIST_WARP && lane == 0) {
            tma_prefetch(&map_q);
            u32 copied[2] = { 0, 0 };
            bool ok = true;
            for (int round = 0; ok && (ok = bar_place(round > 1, rp_smem(&sm.block_empty[round & 1]), ((round >> 1) - 1) & 1, waits)); ++round) {
                const int at = rp_attend_item(round, total);
                volatile int *const to = sm.block[round & 1];
                to[0] = at;
                if (at < 0) {
                    bar_arrive(rp_smem(&sm.block_full[round & 1]));
                    break;
                }
                const AttendTile t(A.items, A.start, A.T, at / A.Hq, 256);
                to[1] = (int)t.base; to[2] = t.len; to[3] = t.row0;
                bar_arrive(rp_smem(&sm.block_full[round & 1]));
                // (the second tile is the first to be needed, and to be done with)
                for (int i = t.row0 + 128 < t.len; i >= 0; --i) {
                    if (!(ok = bar_place(copied[i], rp_smem(&sm.q_empty[i]), (copied[i] - 1) & 1, waits))) break;
                    ++copied[i];
                    bar_expect(rp_smem(&sm.q_full[i]), Smem::TILE);
                    for (int p = 0; p < PANELS; ++p)
                        tma_load3(rp_smem(sm.q[i]) + p * PANEL, &map_q, p * 64, at % A.Hq, (int)t.base + t.row0 + 128 * i, rp_smem(&sm.q_full[i]));
                }
            }
            // nobody may leave while copies are under way (whoever should have waited for them may have given up)
            for (int i = 0; i < 2; ++i)
                if (copied[i]) rp_drain(rp_smem(&sm.q_full[i]), (copied[i] - 1) & 1);
        }
        if (warp == ATTEND_COPY_WARP && lane == 0) {
            tma_prefetch(&map_k); tma_prefetch(&map_v);
            u32 fill = 0, how = 0;                      // copies into the ring so far; parts of the step before
            int row = -1, head = 0, behind = 0;         // the step before, whose values go with the next one's keys
            bool ok = true;
            const auto copy = [&](int next, int next_head, int next_behind, u32 next_how) {
                const u32 s = fill % STAGES, turn = fill / STAGES;
                if (!(ok = bar_place(turn, rp_smem(&sm.kv_empty[s]), (turn - 1) & 1, waits))) return;
                sm.step[s] = how | next_how << 8 | (u32)behind << 16;
                bar_expect(rp_smem(&sm.kv_full[s]), row >= 0 && next >= 0 ? 2 * Smem::TILE : Smem::TILE);
                waits->copied = ++fill;
                for (int p = 0; p < PANELS; ++p) {
                    if (row >= 0) tma_load3(rp_smem(sm.v[s]) + p * PANEL, &map_v, p * 64, head, row, rp_smem(&sm.kv_full[s]));
                    if (next >= 0) tma_load3(rp_smem(sm.k[s]) + p * PANEL, &map_k, p * 64, next_head, next, rp_smem(&sm.kv_full[s]));
                }
                row = next; head = next_head; behind = next_behind; how = next_how;
            };
            for (int round = 0; ok && (ok = bar_wait(rp_smem(&sm.block_full[round & 1]), (round >> 1) & 1, waits)); ++round) {
                const int at = sm.block[round & 1][0];
                if (at < 0) break;
                const AttendTile t(sm.block[round & 1]);
                bar_arrive(rp_smem(&sm.block_empty[round & 1]));
                const AttendOrder w(t.row0, t.len, A.window, A.sinks);
                for (int j = 0; ok && j < w.steps; ++j) {
                    const int k0 = w.tile(j) * 128;
                    const u32 parts = (w.active(0, j) ? STEP_TAKES : 0) | (w.active(1, j) ? STEP_TAKES << 1 : 0) | (j == w.last[0] ? STEP_LAST : 0) | (j == w.last[1] ? STEP_LAST << 1 : 0) |
                                      (j > w.first(0) ? STEP_MORE : 0) | (j > 0 ? STEP_MORE << 1 : 0) | (w.first_tokens(j) ? STEP_FEW : 0);
                    copy((int)t.base + k0, at % A.Hq / A.share, min(t.len - k0, 128), parts);
                }
            }
            if (ok && row >= 0) copy(-1, 0, 0, STEP_END);
            else if (ok) {                              // no block at all
                sm.step[0] = STEP_END << 8;
                bar_arrive(rp_smem(&sm.kv_full[0]));
            }
            for (u32 f = fill > (u32)STAGES ? fill - STAGES : 0; f < fill; ++f) rp_drain(rp_smem(&sm.kv_full[f % STAGES]), (f / STAGES) & 1);
        }
        if (warp == ATTEND_MMA_WARP) {
            const u32 shape_s = mma_shape<X>(128, false), shape_o = mma_shape<X>(D, true);
            const int groups = (int)rp_uniform((A.sinks + 31) >> 5);                      // first tokens by 32
            const u32 shape_first = mma_shape<X>(32 * groups, false);
            u32 p0 = 0, p1 = 0, q0 = 0, q1 = 0;             // weights and queries of each tile taken
            // (Between the products of one tile and the next the tensor cores run dry, so this warp works little out: a step's parts come with its stage, in one register of
            // the warp, and branches by it leave the products' operands there.)
            const auto begin = [&](u32 next, u32 stage, int i) {               // a tile's part in the next step: its scores
                if (!(next & (STEP_TAKES << i))) return;
                if (!(next & (STEP_MORE << i))) bar_hold(rp_smem(&sm.q_full[i]), (i ? q1++ : q0++) & 1, waits);
                const u32 a = mma_operand(rp_smem(sm.q[i]), true, 0), b = mma_operand(rp_smem(sm.k[stage]), true, 0), shape = next & STEP_FEW ? shape_first : shape_s;
                if (rp_elect()) {
#pragma unroll
                    for (int x = 0; x < D / 16; ++x) {
                        const u32 off = ((x / 4) * PANEL + (x % 4) * 32) >> 4;
                        mma_ss(tm + i * 128, a + off, b + off, shape, x > 0);
                    }
                    mma_commit(rp_smem(&sm.s_full[i]));
                    if (next & (STEP_LAST << i)) mma_commit(rp_smem(&sm.q_empty[i]));
                }
                __syncwarp();
            };
            const auto finish = [&](u32 step, u32 stage, int i) {              // in the present one: its weights times the values
                bar_hold(rp_smem(&sm.p_full[i]), (i ? p1++ : p0++) & 1, waits);
                tmem_after();
                const u32 v = mma_operand(rp_smem(sm.v[stage]), false, PANEL);
                if (rp_elect()) {
                    if (step & STEP_FEW)
                        for (int x = 0; x < 2 * groups; ++x) mma_ts(tm + 256 + i * D, tm + i * 128 + x * 8, v + x * (2048 >> 4), shape_o, true);
                    else {
#pragma unroll
                        for (int x = 0; x < 8; ++x) mma_ts(tm + 256 + i * D, tm + i * 128 + x * 8, v + x * (2048 >> 4), shape_o, (step & (STEP_MORE << i)) || x > 0);
                    }
                    if (step & (STEP_LAST << i)) mma_commit(rp_smem(&sm.o_full[i]));
                }
                __syncwarp();
            };
            for (u32 used = 0;; ++used) {
                const u32 s = used % STAGES;
                bar_hold(rp_smem(&sm.kv_full[s]), (used / STAGES) & 1, waits);
                const u32 step = rp_uniform(waits->gave_up ? STEP_END << 8 : sm.step[s]), next = step >> 8, behind = step >> 16;
                // values behind the sample's end are another sample's, and those behind the first tokens are not seen: their weights are 0, and 0 times NaN would not be
                if (step & (STEP_TAKES * 3)) {
                    if (behind < 128) rp_clear_rows<D>(sm.v[s], behind, 128, lane);
                    if (step & STEP_FEW) rp_clear_rows<D>(sm.v[s], A.sinks, 32 * groups, lane);
                }
                if (step & STEP_TAKES) finish(step, s, 0);
                begin(next, s, 0);
                if (step & (STEP_TAKES << 1)) finish(step, s, 1);
                begin(next, s, 1);
                mma_commit_warp(rp_smem(&sm.kv_empty[s]));
                if (next & STEP_END) break;
            }
            // nobody may leave while products are under way
            mma_commit_warp(rp_smem(&sm.done));
            if (lane == 0) rp_drain(rp_smem(&sm.done), 0);
        }
    } else {
        rp_many_registers();
        const int i = warp >> 2, row = threadIdx.x & 127;
        const u32 lanes = (u32)(warp & 3) << 21, ts = tm + lanes + i * 128, to = tm + lanes + 256 + i * D;
        const float sl = A.scale * RP_LOG2E;
        const f2 sl2 = rp_f2(sl, sl);
        u32 ss = 0, os = 0;
        // A block as the group sees it: the item (-1: none any more), whether the warp was told of it, the steps that its tile takes part in.  (Beside a row's scores there
        // is no room for much: what a block's steps go by stays in shared memory and is worked out anew in each.)
        struct Block { int at, first, end; bool told; };
        const auto look = [&](int round) {
            Block x;
            volatile int *const block = sm.block[round & 1];
            x.told = bar_wait_warp(rp_smem(&sm.block_full[round & 1]), (round >> 1) & 1, waits);
            x.at = x.told ? block[0] : rp_attend_item(round, total);
            x.first = x.end = 0;
            if (x.at < 0) return x;
            const AttendTile t = x.told ? AttendTile(block) : AttendTile(A.items, A.start, A.T, x.at / A.Hq, 256);
            const AttendOrder order(t.row0, t.len, A.window, A.sinks);
            if (t.row0 + 128 * i < t.len) { x.first = order.first(i); x.end = order.last[i] + 1; }
            return x;
        };
        Block next = look(0);
        for (int round = 0; next.at >= 0; ++round) {
            volatile int *const block = sm.block[round & 1];
            const int at = next.at, first = next.first, nk = next.end;
            const bool told = next.told;
            if (nk == 0) {                               // no rows of its own
                if (told) bar_arrive_warp(rp_smem(&sm.block_empty[round & 1]), lane);
                next = look(round + 1);
                continue;
            }
            float m = -INFINITY, l = 0.0f;
            bool ok = told;                              // (what is not told is not worked out: a wait has run out)
            for (int j = first; ok && j < nk; ++j) {
                // columns that the row sees: those before `lim`, of these the ones from `from` on and the `ahead` first; whether there are others (1: behind, 2: before)
                const int row0 = block[3], len = block[2], r0 = row0 + 128 * i, r = r0 + row;
                const AttendOrder w(row0, len, A.window, A.sinks);
                if (i == 1 && j == w.hole) continue;
                const int k0 = w.tile(j) * 128, lim = min(len, r + 1) - k0, from = r - A.window + 1 - k0, ahead = A.sinks - k0;
                const int hidden = (k0 + 128 > len || k0 + 127 > r0 ? 1 : 0) | (k0 <= r0 + 127 - A.window ? 2 : 0);
                const bool first_tokens = w.first_tokens(j), held = r < len;
                if (!(ok = bar_wait_warp(rp_smem(&sm.s_full[i]), ss & 1, waits))) break;
                ++ss;
                tmem_after();
                // the row's maximum with the tile's
                const auto grow = [&](float top) {
                    if (j == first) { m = top; return; }
                    // (a maximum that grows by less than 2^8 stays: weights up to 256 and their sums lose nothing; -inf, as long as no score is above it, goes with the
                    // first that is; rows behind the sample's end are other samples', which do not matter)
                    const float grown = held ? (top - m) * sl : 0.0f;
                    if (__any_sync(0xffffffffu, grown > 8.0f)) {
                        const float up = fmaxf(top, m), f = m == up ? 1.0f : rp_exp2((m - up) * sl);
                        m = up;
                        l *= f;
#pragma unroll
                        for (int c = 0; c < D; c += 32) {
                            u32 o[32];
                            tmem_load32(to + c, o);
                            tmem_loaded();
#pragma unroll
                            for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
                            tmem_store32(to + c, o);
                        }
                    }
                };
                if (first_tokens) {
                    // first tokens from afar: the same ones for all rows, 32 columns at a time
                    float top = -INFINITY;
                    for (int g = 0; g < A.sinks; g += 32) {
                        u32 s[32];
                        tmem_load32(ts + g, s);
                        tmem_loaded();
#pragma unroll
                        for (int c = 0; c < 32; ++c) top = g + c < A.sinks ? fmaxf(top, __uint_as_float(s[c])) : top;
                    }
                    grow(top);
                    const float less = m == -INFINITY ? LIFT : fmaf(-m, sl, LIFT);
                    for (int g = 0; g < A.sinks; g += 64) {
                        u32 p[32];
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            u32 s[32];
                            if (!u || g + 32 < A.sinks) {
                                tmem_load32(ts + g + 32 * u, s);
                                tmem_loaded();
                            }
#pragma unroll
                            for (int c = 0; c < 32; c += 2) {
                                const int k = g + 32 * u + c;
                                const float a = k < A.sinks ? rp_exp2(fmaf(__uint_as_float(s[c]), sl, less)) : 0.0f;
                                const float b = k + 1 < A.sinks ? rp_exp2(fmaf(__uint_as_float(s[c + 1]), sl, less)) : 0.0f;
                                l += a + b;
                                p[16 * u + c / 2] = rp_pair(a, b, X());
                            }
                        }
                        tmem_store32(ts + g / 2, p);
                    }
                    tmem_stored();
                    tmem_before();
                    bar_arrive_warp(rp_smem(&sm.p_full[i]), lane);
                    continue;
                }
                u32 s[128];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_load32(ts + 32 * c, s + 32 * c);
                tmem_loaded();
                if (hidden == 1) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) s[c] = c < lim ? s[c] : 0xff800000u;
                } else if (hidden == 2 && ahead <= 0) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) s[c] = c >= from ? s[c] : 0xff800000u;
                } else if (hidden) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) s[c] = c < lim && (c >= from || c < ahead) ? s[c] : 0xff800000u;
                }
                float top = rp_max3(__uint_as_float(s[0]), __uint_as_float(s[1]), __uint_as_float(s[2])), top1 = __uint_as_float(s[3]);
#pragma unroll
                for (int c = 4; c < 128; c += 4) {
                    top = rp_max3(top, __uint_as_float(s[c]), __uint_as_float(s[c + 1]));
                    top1 = rp_max3(top1, __uint_as_float(s[c + 2]), __uint_as_float(s[c + 3]));
                }
                grow(fmaxf(top, top1));
                const float less = m == -INFINITY ? LIFT : fmaf(-m, sl, LIFT);
                const f2 shift = rp_f2(less, less);
                f2 sum0 = rp_f2(0.0f, 0.0f), sum1 = sum0;
#pragma unroll
                for (int c = 0; c < 64; ++c) {
                    const f2 e = rp_exp2(rp_fma(rp_f2(__uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1])), sl2, shift));
                    if (c & 1) sum1 = rp_add(sum1, e); else sum0 = rp_add(sum0, e);
                    float a, b;
                    rp_parts(e, a, b);
                    s[c] = rp_pair(a, b, X());
                }
                float a, b;
                rp_parts(rp_add(sum0, sum1), a, b);
                l += a + b;
                tmem_store32(ts, s);
                tmem_store32(ts + 32, s + 32);
                tmem_stored();
                tmem_before();
                bar_arrive_warp(rp_smem(&sm.p_full[i]), lane);
            }
            next = look(round + 1);                      // (while the last products are made)
            if (ok) ok = bar_wait_warp(rp_smem(&sm.o_full[i]), os & 1, waits) && !waits->gave_up;
            ++os;
            tmem_after();
            const float f = ok ? 1.0f / l : NAN;
            const AttendTile u = told ? AttendTile(block) : AttendTile(A.items, A.start, A.T, at / A.Hq, 256);
            const int r0 = u.row0 + 128 * i, r = r0 + row, h = at % A.Hq;
            X *const out = (X *)A.out + u.base * A.o_token + h * A.o_head;
            // through shared memory, 64 columns at a time: rows of 128 bytes go out whole (each lane its own row, 16 bytes at a time: 2000 cycles for 500)
            unsigned char *const rows = sm.rows[warp];
            u32 o[D];
#pragma unroll
            for (int c = 0; c < D; c += 32) tmem_load32(to + c, o + c);
            tmem_loaded();
#pragma unroll
            for (int c = 0; c < D; c += 64) {
                float v[64];
#pragma unroll
                for (int x = 0; x < 64; ++x) v[x] = __uint_as_float(o[c + x]) * f;
#pragma unroll
                for (int x = 0; x < 8; ++x) *(Pack8<X> *)(rows + lane * 128 + ((x ^ (lane & 7)) << 4)) = rp_close8<X>(v + 8 * x);
                __syncwarp();
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int y = x * 4 + (lane >> 3), p = lane & 7, q = r0 + (row & ~31) + y;
                    const Pack8<X> w = *(const Pack8<X> *)(rows + y * 128 + ((p ^ (y & 7)) << 4));
                    if (q < u.len && c + 8 * p < A.d) rp_store8(out + q * A.o_token + c + 8 * p, w);
                }
                __syncwarp();
            }
            if (r < u.len && A.lse) A.lse[(u.base + r) * A.l_token + h * A.l_head] = ok ? fmaf(m, A.scale, logf(l * exp2f(-LIFT))) : NAN;
            __syncwarp();
            tmem_before();
            if (told) bar_arrive_warp(rp_smem(&sm.block_empty[round & 1]), lane);
        }
    }
    __syncwarp();
    __syncthreads();
    if (threadIdx.x == 0 && sm.waits.gave_up) *A.status = RP_ERR_TIMEOUT;
    if (warp == ATTEND_COPY_WARP) tmem_free(tm, 512);
}

template <typename X, int D>
static int launch(const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, const AttendArgs &A, int ctas, cudaStream_t stream)
{
    const size_t smem = sizeof(WindowSmem<D>) + 1024;
    RP_CUDA(cudaFuncSetAttribute(k_attend_window<X, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t how = {};                         // (barriers, tensor memory and maps are got ready beside the planning)
    how.gridDim = dim3((unsigned)ctas);
    how.blockDim = dim3(ATTEND_THREADS);
    how.dynamicSmemBytes = smem;
    how.stream = stream;
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    how.attrs = &early; how.numAttrs = 1;
    RP_CUDA(cudaLaunchKernelEx(&how, k_attend_window<X, D>, q, k, v, A));
    return rp_op_launched();
}
int rp_launch_attend_window(int type, int d, const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, const AttendArgs &A, int ctas, cudaStream_t stream)
{
    if (type == RP_F16) return d <= 64 ? launch<__half, 64>(q, k, v, A, ctas, stream) : launch<__half, 128>(q, k, v, A, ctas, stream);
    return d <= 64 ? launch<bf16, 64>(q, k, v, A, ctas, stream) : launch<bf16, 128>(q, k, v, A, ctas, stream);
}
