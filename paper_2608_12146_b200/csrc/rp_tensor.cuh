// Tensor cores, tensor memory and bulk copies of sm_100a as the attention kernels use them: thin wrappers of the PTX instructions.
#pragma once

#include <cuda.h>

#include <type_traits>

#include "rp_ops.cuh"

__device__ __forceinline__ u32 rp_smem(const void *p) { return (u32)__cvta_generic_to_shared(p); }

// ---- barriers ---------------------------------------------------------------------------
__device__ __forceinline__ void bar_init(u32 bar, u32 count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(u32 bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// One arrival for a warp, behind what all its lanes have done.
__device__ __forceinline__ void bar_arrive_warp(u32 bar, int lane)
{
    __syncwarp();
    if (lane == 0) bar_arrive(bar);
    __syncwarp();
}
__device__ __forceinline__ void bar_expect(u32 bar, u32 bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(u32 bar, u32 parity)
{
    u32 done;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ u64 rp_nanoseconds()
{
    u64 t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// A CTA's waits, in its shared memory: whoever waits for longer than the limit sets `gave_up`, and all others stop waiting when they see it.
struct Waits {
    volatile int gave_up;
    volatile u32 copied;                                 // how often something was copied: a CTA that goes on is not stuck, however long one of its warps has nothing to do
    u64 limit;                                           // nanoseconds; 0: nothing is waited for
    __device__ __forceinline__ void start(u64 ns) { gave_up = ns == 0; copied = 0; limit = ns; }
};
// Waits for the end of a barrier's phase, up to the limit without a copy (two seconds; a step of these kernels takes microseconds): false when it ran out.
__device__ __forceinline__ bool bar_wait_long(u32 bar, u32 parity, Waits *w)
{
    u64 since = rp_nanoseconds();
    u32 seen = w->copied;
    for (u32 n = 0;; ++n) {
        if (w->gave_up) return false;
        if (bar_try(bar, parity)) return true;
        if ((n & 63) != 63) continue;
        const u64 now = rp_nanoseconds();
        if (w->copied != seen) { seen = w->copied; since = now; }
        else if (now - since > w->limit) { w->gave_up = 1; return false; }
    }
}
__device__ __forceinline__ bool bar_wait(u32 bar, u32 parity, Waits *w)
{
    if (bar_try(bar, parity)) return true;
    return bar_wait_long(bar, parity, w);
}

// The same for a whole warp, which goes on together.
__device__ __forceinline__ bool bar_wait_warp(u32 bar, u32 parity, Waits *w)
{
    return __all_sync(0xffffffffu, bar_wait(bar, parity, w));
}

// The same for the warp that copies: a place that is free again, or has not been used yet.  Nothing is copied any more once a wait has run out, since who has let go of
// a place then need not be done with it.
__device__ __forceinline__ bool bar_place(bool used, u32 bar, u32 parity, Waits *w)
{
    return (!used || bar_wait(bar, parity, w)) && !w->gave_up;
}

// The same for the warp that issues products, which does not ask: when a wait ran out it goes on to the end of its block with whatever there is, all its waits end at once
// from then on, and the blocks that are handed over afterwards are marked.  (A vote and a branch less a wait: 50 of 125 cycles in which the tensor cores run dry.)
__device__ __forceinline__ void bar_hold(u32 bar, u32 parity, Waits *w)
{
    if (!bar_try(bar, parity)) bar_wait_long(bar, parity, w);
    __syncwarp();
}

// ---- bulk copies ------------------------------------------------------------------------
__device__ __forceinline__ void tma_load3(u32 dst, const CUtensorMap *map, int x, int y, int z, u32 bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_prefetch(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor memory ----------------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(u32 dst, u32 columns)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(u32 at, u32 columns) { asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns)); }
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 32 columns of the warp's 32 rows: lane = row, r[i] = column i.  Valid after tmem_loaded().
__device__ __forceinline__ void tmem_load32(u32 at, u32 *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store32(u32 at, const u32 *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
                   "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
                   "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(at)
                 : "memory");
}

// ---- matrix products --------------------------------------------------------------------
// Operands in shared memory lie in panels of 64 elements (128 bytes) a row, rows one after the other, as a copy with the 128-byte swizzle
// leaves them; eight rows are 1024 bytes.
// `along_k`: rows are rows (or columns) of the product and the 64 elements run along the summed dimension; a step of 16 of those is 32 bytes on.
// Otherwise the rows run along the summed dimension; a step of 16 is 2048 bytes on, the next 64 elements are `panel` bytes on.
// A value that all lanes of a warp have alike, in a register that the warp has once: the products take their operands from such, and what is worked out from
// such ones in branches and loops that go by them stays there (moved over one by one for each product, they issue at half the rate).
__device__ __forceinline__ u32 rp_uniform(u32 x) { return __reduce_or_sync(0xffffffffu, x); }
// Descriptor of an operand: the low word has its address, the high word is fixed (eight rows of 128 bytes, version, swizzle).
#define MMA_HIGH ((1024u >> 4) | (1u << 14) | (2u << 29))
__device__ __forceinline__ u32 mma_operand(u32 at, bool along_k, u32 panel) { return ((at & 0x3ffffu) >> 4) | ((along_k ? 1u : panel >> 4) << 16); }
// 16-bit operands, 32-bit sums, 128 rows, `n` columns; `b_rows_k`: B's rows run along the summed dimension.
template <typename X> __device__ __forceinline__ constexpr u32 mma_shape(int n, bool b_rows_k)
{
    return (1u << 4) | ((std::is_same<X, bf16>::value ? 1u : 0u) << 7) | ((std::is_same<X, bf16>::value ? 1u : 0u) << 10) |
           ((b_rows_k ? 1u : 0u) << 16) | ((u32)(n >> 3) << 17) | ((128u >> 4) << 24);
}
// Whoever of the warp's lanes issues products; the whole warp asks.  The compiler knows then that one lane goes in, and the operands that the instructions take are
// worked out once for the warp, in registers of its own.  (An attention block of ten tiles 26.5 us with a comparison of the lane's number at each instruction, 23.5 with
// this choice at each, 22.5 with a branch for all products of a tile.)
__device__ __forceinline__ bool rp_elect()
{
    u32 r;
    asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(r)::"memory");
    return r != 0;
}
// One step of 16 along the summed dimension; `more`: added to what the accumulator holds.  By the lane that rp_elect() chooses.
__device__ __forceinline__ void mma_ss(u32 d, u32 a, u32 b, u32 shape, bool more)
{
    asm volatile("{\n .reg .pred p;\n .reg .b64 x, y;\n setp.ne.u32 p, %4, 0;\n mov.b64 x, {%1, %5};\n mov.b64 y, {%2, %5};\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n}"
                 ::"r"(d), "r"(a), "r"(b), "r"(shape), "r"((u32)more), "r"(MMA_HIGH) : "memory");
}
__device__ __forceinline__ void mma_ts(u32 d, u32 a, u32 b, u32 shape, bool more)           // A from tensor memory, two elements a column
{
    asm volatile("{\n .reg .pred p;\n .reg .b64 y;\n setp.ne.u32 p, %4, 0;\n mov.b64 y, {%2, %5};\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n}"
                 ::"r"(d), "r"(a), "r"(b), "r"(shape), "r"((u32)more), "r"(MMA_HIGH) : "memory");
}
// The barrier is arrived at when all products that the chosen lane has issued are done: by that lane, or by the whole warp.
__device__ __forceinline__ void mma_commit(u32 bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mma_commit_warp(u32 bar)
{
    if (rp_elect()) mma_commit(bar);
    __syncwarp();
}

// ---- host: a tensor [tokens][heads][dim] as 64-element panels of `rows` tokens of one head ----
int rp_tensor_map(CUtensorMap *map, int type, const void *x, i64 tokens, int heads, int dim, i64 token_stride, i64 head_stride, int rows);
