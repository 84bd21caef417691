// Attention inside the samples of a packed row, forward.
//
//   s = scale q k^T over the tokens of a sample, p = exp(s - m), o = p v / sum p, lse = m + log sum p, m a running maximum
//
// A tile of 128 queries and 128 keys is 2 * 128 * 128 * head_dim multiply-adds (1024 cycles of an SM's tensor cores at head_dim 128) and 128 * 128 exponentials (1024
// cycles of its special function units).  What bounds it are the hand-overs between the warps of a tile: at 4097 tokens the tensor cores are busy for 34 % of the
// time, the special function units for 43 %.
// A CTA takes 256 queries of a head as two tiles of 128, each with four warps of its own for the softmax (a thread has a row, so a row's maximum and sum
// need no exchange); while one tile's weights are worked out, the tensor cores work on the other's.  One warp copies keys and values into a ring of
// shared memory, one issues the products.  Scores and outputs live in tensor memory (2 x 128 + 2 x head_dim columns), the weights take the
// scores' place as the operand of the second product.  Outputs are scaled again only when a row's maximum has grown by more than 2^8.
// CTAs stay resident and take blocks of queries in the order of falling work.
// 12289 tokens in two samples, 16 heads on 4, 128 wide, causal: 322 us, 1100 TFLOP/s (357 under the power cap of a long run); 32768 tokens in five 1284 us, 1206 TFLOP/s.  A product of 128 x 128 x 16 takes
// 64 cycles, to which each wait and commit of the warp that issues adds 50 to 150.  Tried: two warps that issue, one a tile (449 us for 381 then); a part of the
// exponentials by a polynomial beside the special function unit (323 to 360 for 322).
#include <algorithm>

#include "rp_attend.cuh"

__global__ void __launch_bounds__(1024) k_attend_plan(AttendPlan P, AttendClears C)
{
    rp_let_next_launch_start();
    if (blockIdx.x == 0) rp_attend_plan(P);
    else rp_attend_clear(C, P.start, P.N, P.T, blockIdx.x - 1, gridDim.x - 1);
}

// ---------------------------------------------------------------------------------------
// the kernel
// ---------------------------------------------------------------------------------------
// A stage holds the values of one tile and the keys of the next, which are waited for and let go of together: of nk tiles there are nk + 1 stages, the first without
// values, the last without keys.
template <int D> struct FwdSmem {
    static constexpr int TILE = 128 * D * 2, STAGES = D == 128 ? 2 : 4;
    alignas(1024) unsigned char q[2][TILE];
    alignas(1024) unsigned char v[STAGES][TILE];
    alignas(1024) unsigned char k[STAGES][TILE];
    u64 q_full, q_empty, kv_full[STAGES], kv_empty[STAGES], s_full[2], p_full[2], o_full[2], done;
    u32 tmem;
    Waits waits;
};

template <typename X, int D>
__global__ void __launch_bounds__(ATTEND_THREADS, 1)
k_attend(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const AttendArgs A)
{
    typedef FwdSmem<D> Smem;
    constexpr int STAGES = Smem::STAGES, PANELS = D / 64, PANEL = 128 * 128;
    // Weights of float16 times 2^7, up to 2^15 with what a maximum may lag behind: as 2^-25 and less of the largest they would be lost from the product with the values, and
    // many of them are something (131072 keys 17.5 under the largest: 0.0033 of their values).
    constexpr float LIFT = std::is_same<X, bf16>::value ? 0.0f : 7.0f;
    extern __shared__ __align__(1024) unsigned char raw[];
    Smem &sm = *(Smem *)(raw + ((1024 - (rp_smem(raw) & 1023)) & 1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        bar_init(rp_smem(&sm.q_full), 1); bar_init(rp_smem(&sm.q_empty), 1);
        for (int s = 0; s < STAGES; ++s) { bar_init(rp_smem(&sm.kv_full[s]), 1); bar_init(rp_smem(&sm.kv_empty[s]), 1); }
        for (int i = 0; i < 2; ++i) { bar_init(rp_smem(&sm.s_full[i]), 1); bar_init(rp_smem(&sm.p_full[i]), 4); bar_init(rp_smem(&sm.o_full[i]), 1); }
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
        if (warp == ATTEND_COPY_WARP && lane == 0) {
            tma_prefetch(&map_q); tma_prefetch(&map_k); tma_prefetch(&map_v);
            u32 blocks = 0, fill = 0;                   // copies of queries and into the ring so far
            bool ok = true;
            for (int round = 0; ok; ++round) {
                const int at = rp_attend_item(round, total);
                if (at < 0) break;
                const AttendTile t(A.items, A.start, A.T, at / A.Hq, 256);
                const int h = at % A.Hq, hk = h / A.share;
                if (!(ok = bar_place(round, rp_smem(&sm.q_empty), (round - 1) & 1, waits))) break;
                ++blocks;
                const int tiles = t.row0 + 128 < t.len ? 2 : 1;
                bar_expect(rp_smem(&sm.q_full), tiles * Smem::TILE);
                for (int i = 0; i < tiles; ++i)
                    for (int p = 0; p < PANELS; ++p)
                        tma_load3(rp_smem(sm.q[i]) + p * PANEL, &map_q, p * 64, h, (int)t.base + t.row0 + 128 * i, rp_smem(&sm.q_full));
                const int nk = rp_attend_tiles(t, tiles - 1, A.causal);
                for (int j = 0; j <= nk; ++j, ++fill) {
                    const u32 s = fill % STAGES, turn = fill / STAGES;
                    if (!(ok = bar_place(turn, rp_smem(&sm.kv_empty[s]), (turn - 1) & 1, waits))) break;
                    bar_expect(rp_smem(&sm.kv_full[s]), j && j < nk ? 2 * Smem::TILE : Smem::TILE);
                    waits->copied = fill + 1;
                    for (int p = 0; p < PANELS; ++p) {
                        if (j) tma_load3(rp_smem(sm.v[s]) + p * PANEL, &map_v, p * 64, hk, (int)t.base + (j - 1) * 128, rp_smem(&sm.kv_full[s]));
                        if (j < nk) tma_load3(rp_smem(sm.k[s]) + p * PANEL, &map_k, p * 64, hk, (int)t.base + j * 128, rp_smem(&sm.kv_full[s]));
                    }
                }
            }
            // nobody may leave while copies are under way (whoever should have waited for them may have given up)
            for (u32 f = fill > (u32)STAGES ? fill - STAGES : 0; f < fill; ++f) rp_drain(rp_smem(&sm.kv_full[f % STAGES]), (f / STAGES) & 1);
            if (blocks) rp_drain(rp_smem(&sm.q_full), (blocks - 1) & 1);
        }
        if (warp == ATTEND_MMA_WARP) {
            const u32 shape_s = mma_shape<X>(128, false), shape_o = mma_shape<X>(D, true);
            u32 used = 0, p0 = 0, p1 = 0;                   // stages taken; weights taken of each tile
            auto scores = [&](int i, u32 stage) {           // tile i's scores for the keys in a stage
                const u32 a = mma_operand(rp_smem(sm.q[i]), true, 0), b = mma_operand(rp_smem(sm.k[stage]), true, 0);
                if (rp_elect()) {
#pragma unroll
                    for (int x = 0; x < D / 16; ++x) {
                        const u32 off = ((x / 4) * PANEL + (x % 4) * 32) >> 4;
                        mma_ss(tm + i * 128, a + off, b + off, shape_s, x > 0);
                    }
                    mma_commit(rp_smem(&sm.s_full[i]));
                }
                __syncwarp();
            };
            auto outputs = [&](int i, u32 stage, bool more) {          // its weights times the values in a stage
                const u32 v = mma_operand(rp_smem(sm.v[stage]), false, PANEL);
                if (rp_elect()) {
#pragma unroll
                    for (int x = 0; x < 8; ++x) mma_ts(tm + 256 + i * D, tm + i * 128 + x * 8, v + x * (2048 >> 4), shape_o, more || x > 0);
                }
                __syncwarp();
            };
            for (int round = 0;; ++round) {
                const int at = rp_attend_item(round, total);
                if (at < 0 || rp_uniform(waits->gave_up)) break;
                const AttendTile t(A.items, A.start, A.T, at / A.Hq, 256);
                const int left = rp_uniform(t.len - t.row0), tiles = left > 128 ? 2 : 1, len = rp_uniform(t.len);
                const int n0 = rp_uniform(rp_attend_tiles(t, 0, A.causal)), n1 = tiles == 2 ? rp_uniform(rp_attend_tiles(t, 1, A.causal)) : 0, nk = max(n0, n1);
                bar_hold(rp_smem(&sm.q_full), round & 1, waits);
                bar_hold(rp_smem(&sm.kv_full[used % STAGES]), (used / STAGES) & 1, waits);
                scores(0, used % STAGES);
                if (tiles == 2) scores(1, used % STAGES);
                mma_commit_warp(rp_smem(&sm.kv_empty[used % STAGES]));
                if (nk == 1) mma_commit_warp(rp_smem(&sm.q_empty));
                ++used;
                for (int j = 0; j < nk; ++j, ++used) {
                    const u32 s = used % STAGES;
                    // (what is copied has mostly come when the weights have)
                    bar_hold(rp_smem(&sm.kv_full[s]), (used / STAGES) & 1, waits);
                    // values behind the sample's end are another sample's: their weights are 0, and 0 times NaN would not be
                    if (len - j * 128 < 128) rp_clear_rows<D>(sm.v[s], len - j * 128, 128, lane);
                    if (j < n0) {
                        bar_hold(rp_smem(&sm.p_full[0]), p0++ & 1, waits);
                        tmem_after();
                        outputs(0, s, j > 0);
                        if (j == n0 - 1) mma_commit_warp(rp_smem(&sm.o_full[0]));
                        else scores(0, s);
                    }
                    if (j < n1) {
                        bar_hold(rp_smem(&sm.p_full[1]), p1++ & 1, waits);
                        tmem_after();
                        outputs(1, s, j > 0);
                        if (j == n1 - 1) mma_commit_warp(rp_smem(&sm.o_full[1]));
                        else scores(1, s);
                    }
                    mma_commit_warp(rp_smem(&sm.kv_empty[s]));
                    if (j == nk - 2) mma_commit_warp(rp_smem(&sm.q_empty));
                }
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
        for (int round = 0;; ++round) {
            const int at = rp_attend_item(round, total);
            if (at < 0) break;
            const AttendTile t(A.items, A.start, A.T, at / A.Hq, 256);
            const int h = at % A.Hq, r0 = t.row0 + 128 * i, r = r0 + row;
            if (r0 >= t.len) continue;
            const int nk = rp_attend_tiles(t, i, A.causal);
            float m = -INFINITY, l = 0.0f;
            bool ok = true;
            for (int j = 0; j < nk; ++j) {
                if (!(ok = bar_wait_warp(rp_smem(&sm.s_full[i]), ss & 1, waits))) break;
                ++ss;
                tmem_after();
                u32 s[128];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_load32(ts + 32 * c, s + 32 * c);
                tmem_loaded();
                if (j * 128 + 128 > t.len || (A.causal && j * 128 + 127 > r0)) {
                    const int lim = (A.causal ? min(t.len, r + 1) : t.len) - j * 128;
#pragma unroll
                    for (int c = 0; c < 128; ++c) s[c] = c < lim ? s[c] : 0xff800000u;
                }
                float top = __uint_as_float(s[0]);
#pragma unroll
                for (int c = 1; c < 128; ++c) top = fmaxf(top, __uint_as_float(s[c]));
                if (j == 0) m = top;
                else {
                    // (a maximum that grows by less than 2^8 stays: weights up to 256 and their sums lose nothing; -inf, as long as no score is above it, goes with the
                    // first that is; rows behind the sample's end are other samples', which do not matter)
                    const float grown = r < t.len ? (top - m) * sl : 0.0f;
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
                }
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
            if (ok) ok = bar_wait_warp(rp_smem(&sm.o_full[i]), os & 1, waits) && !waits->gave_up;
            ++os;
            tmem_after();
            const float f = ok ? 1.0f / l : NAN;
            X *out = (X *)A.out + (t.base + r) * A.o_token + h * A.o_head;
#pragma unroll
            for (int c = 0; c < D; c += 32) {
                u32 o[32];
                tmem_load32(to + c, o);
                tmem_loaded();
                float v[32];
#pragma unroll
                for (int x = 0; x < 32; ++x) v[x] = __uint_as_float(o[x]) * f;
#pragma unroll
                for (int x = 0; x < 32; x += 8)
                    if (r < t.len && c + x < A.d) rp_store8(out + c + x, rp_close8<X>(v + x));
                __syncwarp();
            }
            if (r < t.len && A.lse) A.lse[(t.base + r) * A.l_token + h * A.l_head] = ok ? fmaf(m, A.scale, logf(l * exp2f(-LIFT))) : NAN;
            __syncwarp();
            tmem_before();
        }
    }
    __syncwarp();
    __syncthreads();
    if (threadIdx.x == 0 && sm.waits.gave_up) *A.status = RP_ERR_TIMEOUT;
    if (warp == ATTEND_COPY_WARP) tmem_free(tm, 512);
}

// ---------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------
int rp_tensor_map(CUtensorMap *map, int type, const void *x, i64 tokens, int heads, int dim, i64 token_stride, i64 head_stride, int rows)
{
    typedef CUresult (*Encode)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                               const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static Encode encode = nullptr;                      // the same value from every thread that fills it in
    if (!encode) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult how;
        RP_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &how));
        if (!fn || how != cudaDriverEntryPointSuccess) return RP_ERR_CUDA;
        encode = (Encode)fn;
    }
    if (heads == 1) head_stride = 8;                     // (not used)
    if (tokens == 1) token_stride = 8;
    const cuuint64_t size[3] = { (cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)tokens };
    const cuuint64_t stride[2] = { (cuuint64_t)head_stride * 2, (cuuint64_t)token_stride * 2 };
    const cuuint32_t box[3] = { 64, 1, (cuuint32_t)rows }, one[3] = { 1, 1, 1 };
    const CUresult e = encode(map, type == RP_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, (void *)x, size, stride, box, one,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return e == CUDA_SUCCESS ? RP_OK : RP_ERR_ARG;
}

int rp_attend_check(const rp_attend_config *a, i64 T, int N)
{
    if (!a || T < 0 || N < 1 || a->q_heads < 1 || a->kv_heads < 1 || a->head_dim < 1 || (a->type != RP_F16 && a->type != RP_BF16) || a->causal < 0 || a->causal > 1 ||
        !(a->scale > 0.0f) || !(a->scale < INFINITY))
        return RP_ERR_ARG;
    if (a->q_heads % a->kv_heads || a->head_dim % 8) return RP_ERR_SHAPE;
    if (a->head_dim > 128 || a->q_heads > 65536 || T >= (1ll << 31) - 512 || N > (1 << 24)) return RP_ERR_RANGE;
    if ((T / 64 + N) * a->q_heads >= (1ll << 31)) return RP_ERR_RANGE;
    return RP_OK;
}
int rp_attend_view(const rp_view *v, i64 T, int heads, RpOpDevice &dev)
{
    if (!v || !v->x || !rp_aligned(v->x, 16)) return RP_ERR_ARG;
    if ((T > 1 && (v->token < 1 || v->token % 8 || v->token >= (1ll << 39))) || (heads > 1 && (v->head < 1 || v->head % 8 || v->head >= (1ll << 39)))) return RP_ERR_ARG;
    return dev.hold(v->x);
}
i64 g_attend_wait_ns = 2000000000;
extern "C" int rp_debug_set_wait_limit(int64_t nanoseconds)
{
    if (nanoseconds < 0) return RP_ERR_ARG;
    g_attend_wait_ns = nanoseconds;
    return RP_OK;
}
static i64 plan_bytes(i64 T, int N, int rows) { return (i64)sizeof(AttendHead) + 8 * (T / rows + N); }

extern "C" int64_t rp_attend_workspace(const rp_attend_config *a, int64_t n_tokens, int32_t n_samples)
{
    if (rp_attend_check(a, n_tokens, n_samples) != RP_OK) return 0;
    return plan_bytes(n_tokens, n_samples, 256);
}

template <typename X, int D>
static int launch(const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, const AttendArgs &A, int ctas, cudaStream_t stream)
{
    const size_t smem = sizeof(FwdSmem<D>) + 1024;
    RP_CUDA(cudaFuncSetAttribute(k_attend<X, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t how = {};                         // (barriers, tensor memory and maps are got ready beside the planning)
    how.gridDim = dim3((unsigned)ctas);
    how.blockDim = dim3(ATTEND_THREADS);
    how.dynamicSmemBytes = smem;
    how.stream = stream;
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    how.attrs = &early; how.numAttrs = 1;
    RP_CUDA(cudaLaunchKernelEx(&how, k_attend<X, D>, q, k, v, A));
    return rp_op_launched();
}

// Limits of a window besides those of the attention: sums of a place and the window stay inside 32 bits.
int rp_attend_check_window(const rp_attend_config *a, int window, int sinks, i64 T, int N)
{
    RP_TRY(rp_attend_check(a, T, N));
    if (!a->causal || window < 1 || sinks < 0) return RP_ERR_ARG;
    return sinks > ATTEND_SINKS || T >= (1 << 30) - 512 ? RP_ERR_RANGE : RP_OK;
}

static int attend(const rp_attend_config *a, int window, int sinks, i64 n_tokens, const rp_view *q, const rp_view *k, const rp_view *v, const int64_t *start,
                  int n_samples, const rp_view *out, const rp_view *lse, void *workspace, i64 workspace_bytes, void *cuda_stream)
{
    if (!start || !rp_aligned(start, 8) || !workspace || !rp_aligned(workspace, 16) || workspace_bytes < rp_attend_workspace(a, n_tokens, n_samples)) return RP_ERR_ARG;
    RpOpDevice dev;
    if (n_tokens == 0) {
        RP_TRY(rp_op_enter(dev, workspace));
        RP_CUDA(cudaMemsetAsync(workspace, 0, sizeof(AttendHead), (cudaStream_t)cuda_stream));
        return RP_OK;
    }
    const rp_view *const places[] = { out, lse, q, k, v };
    if (rp_attend_shared(places, 2, 3)) return RP_ERR_ARG;
    RP_TRY(rp_attend_view(q, n_tokens, a->q_heads, dev));
    RP_TRY(rp_attend_view(k, n_tokens, a->kv_heads, dev));
    RP_TRY(rp_attend_view(v, n_tokens, a->kv_heads, dev));
    RP_TRY(rp_attend_view(out, n_tokens, a->q_heads, dev));
    if (lse && lse->x && !rp_aligned(lse->x, 4)) return RP_ERR_ARG;
    RP_TRY(rp_op_enter(dev, start, workspace, lse ? lse->x : nullptr));
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    AttendHead *head = (AttendHead *)workspace;
    int2 *items = (int2 *)(head + 1);
    AttendPlan P = {};
    P.start = (const i64 *)start; P.T = n_tokens; P.N = n_samples; P.rows = 256; P.causal = a->causal; P.by_key = 0;
    P.window = window; P.sinks = sinks; P.most = (int)(n_tokens / 256 + n_samples);
    P.head = head; P.items = items;
    AttendClears C = {};
    C.x[C.n++] = { out->x, out->token, out->head, a->q_heads, a->head_dim, 2 };
    if (lse && lse->x) C.x[C.n++] = { lse->x, lse->token, lse->head, a->q_heads, 1, 4 };
    CUtensorMap mq, mk, mv;
    RP_TRY(rp_tensor_map(&mq, a->type, q->x, n_tokens, a->q_heads, a->head_dim, q->token, q->head, 128));
    RP_TRY(rp_tensor_map(&mk, a->type, k->x, n_tokens, a->kv_heads, a->head_dim, k->token, k->head, 128));
    RP_TRY(rp_tensor_map(&mv, a->type, v->x, n_tokens, a->kv_heads, a->head_dim, v->token, v->head, 128));
    k_attend_plan<<<1 + 32, 1024, 0, stream>>>(P, C);
    RP_TRY(rp_op_launched());
    AttendArgs A = {};
    A.head = head; A.items = items; A.start = (const i64 *)start; A.T = n_tokens; A.N = n_samples; A.Hq = a->q_heads; A.share = a->q_heads / a->kv_heads;
    A.d = a->head_dim; A.causal = a->causal; A.window = window; A.sinks = sinks; A.scale = a->scale; A.out = out->x; A.o_token = out->token; A.o_head = out->head;
    if (lse && lse->x) { A.lse = (float *)lse->x; A.l_token = lse->token; A.l_head = lse->head; }
    A.status = &head->status; A.wait_ns = (u64)g_attend_wait_ns;
    const int ctas = (int)std::min((i64)rp_op_sms(dev.device), (i64)P.most * a->q_heads);
    const bool half = a->type == RP_F16, narrow = a->head_dim <= 64;
    if (window) return rp_launch_attend_window(a->type, a->head_dim, mq, mk, mv, A, ctas, stream);
    if (half) return narrow ? launch<__half, 64>(mq, mk, mv, A, ctas, stream) : launch<__half, 128>(mq, mk, mv, A, ctas, stream);
    return narrow ? launch<bf16, 64>(mq, mk, mv, A, ctas, stream) : launch<bf16, 128>(mq, mk, mv, A, ctas, stream);
}

extern "C" int rp_attend(const rp_attend_config *a, int64_t n_tokens, const rp_view *q, const rp_view *k, const rp_view *v, const int64_t *start,
                         int32_t n_samples, const rp_view *out, const rp_view *lse, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    RP_TRY(rp_attend_check(a, n_tokens, n_samples));
    return attend(a, 0, 0, n_tokens, q, k, v, start, n_samples, out, lse, workspace, workspace_bytes, cuda_stream);
}

extern "C" int rp_attend_window(const rp_attend_config *a, int32_t window, int32_t sinks, int64_t n_tokens, const rp_view *q, const rp_view *k, const rp_view *v,
                                const int64_t *start, int32_t n_samples, const rp_view *out, const rp_view *lse, void *workspace, int64_t workspace_bytes,
                                void *cuda_stream)
{
    RP_TRY(rp_attend_check_window(a, window, sinks, n_tokens, n_samples));
    return attend(a, rp_attend_window_of(window, n_tokens), sinks, n_tokens, q, k, v, start, n_samples, out, lse, workspace, workspace_bytes, cuda_stream);
}
