// What the operators on a window's tokens share: the checks of their arrays, element types, and finding a token's sample.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <string.h>

#include "rp_common.cuh"

typedef __nv_bfloat16 bf16;

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
// The GPU that holds a call's arrays, made current for its launches and put back at the end of the call.
struct RpOpDevice {
    int device = -1, before = -1;
    ~RpOpDevice() { if (before >= 0 && before != device) cudaSetDevice(before); }
    // Arrays that kernels cannot reach where they are, or that lie on two GPUs, are refused; NULL is skipped.
    int hold(const void *p)
    {
        if (!p) return RP_OK;
        cudaPointerAttributes at;
        if (cudaPointerGetAttributes(&at, p) != cudaSuccess) { cudaGetLastError(); return RP_ERR_ARG; }
        if (at.type == cudaMemoryTypeManaged) return RP_OK;
        if (at.type != cudaMemoryTypeDevice || (device >= 0 && at.device != device)) return RP_ERR_ARG;
        device = at.device;
        return RP_OK;
    }
    int enter()
    {
        RP_CUDA(cudaGetDevice(&before));
        if (device < 0) device = before;                 // managed memory alone
        if (device != before) RP_CUDA(cudaSetDevice(device));
        return RP_OK;
    }
};
template <typename... P>
static inline int rp_op_enter(RpOpDevice &d, const P *...p)
{
    int st = RP_OK;
    ((st = st == RP_OK ? d.hold((const void *)p) : st), ...);
    return st == RP_OK ? d.enter() : st;
}
int rp_op_sms(int device);                               // SMs of a GPU (148 on a B200)
int rp_count_args(const void *routes, int bytes, i64 T, int L, int k, int E);
int rp_launch_starts(const int *lengths, int N, i64 *start, cudaStream_t stream);
int rp_launch_count(int device, const void *routes, int bytes, i64 T, int L, int k, int E, i64 ts, i64 ls, const i64 *start, int N, int *demand,
                    cudaStream_t stream);
static inline int rp_op_launched(int n = 1)
{
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return rp_fail(e);
    g_rp_launches += n;
    return RP_OK;
}
static inline bool rp_aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
static inline int rp_type_bytes(int type) { return type == RP_F32 ? 4 : 2; }

// ---------------------------------------------------------------------------------------
// device side
// ---------------------------------------------------------------------------------------
// The last i with start[i] <= t: -1 before the first sample, n behind the last one.  Reads start[0..n] and nothing else, whatever it holds.
__device__ __forceinline__ int rp_sample_of(const i64 *__restrict__ start, int n, i64 t)
{
    u32 lo = 0, hi = (u32)n + 1;                         // (n may be 2^31 - 1)
    while (lo < hi) {
        const u32 mid = (lo + hi) >> 1;
        if (__ldg(start + mid) <= t) lo = mid + 1; else hi = mid;
    }
    return (int)(lo - 1);
}

// Recorded choices of an expert: 1 byte without a sign, 2, 4 or 8 with one.
__device__ __forceinline__ i64 rp_load_route(const void *routes, int bytes, i64 at)
{
    switch (bytes) {
        case 1: return ((const unsigned char *)routes)[at];
        case 2: return ((const short *)routes)[at];
        case 4: return ((const int *)routes)[at];
        default: return ((const i64 *)routes)[at];
    }
}
__device__ __forceinline__ void rp_store_route(void *routes, int bytes, i64 at, int e)
{
    switch (bytes) {
        case 1: ((unsigned char *)routes)[at] = (unsigned char)e; break;
        case 2: ((short *)routes)[at] = (short)e; break;
        case 4: ((int *)routes)[at] = e; break;
        default: ((i64 *)routes)[at] = e; break;
    }
}

__device__ __forceinline__ float rp_float(float x) { return x; }
__device__ __forceinline__ float rp_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float rp_float(bf16 x) { return __bfloat162float(x); }
template <typename X> __device__ __forceinline__ X rp_round(float x);       // to nearest, ties to even
template <> __device__ __forceinline__ float rp_round<float>(float x) { return x; }
template <> __device__ __forceinline__ __half rp_round<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ bf16 rp_round<bf16>(float x) { return __float2bfloat16_rn(x); }

// Eight elements as they lie in memory, and as floats.
template <typename X> struct Pack8 { uint4 w[sizeof(X) / 2]; };
template <typename X> __device__ __forceinline__ Pack8<X> rp_load8(const X *p)
{
    Pack8<X> v;
#pragma unroll
    for (int i = 0; i < (int)sizeof(X) / 2; ++i) v.w[i] = *(const uint4 *)((const char *)p + 16 * i);
    return v;
}
template <typename X> __device__ __forceinline__ void rp_store8(X *p, const Pack8<X> &v)
{
#pragma unroll
    for (int i = 0; i < (int)sizeof(X) / 2; ++i) *(uint4 *)((char *)p + 16 * i) = v.w[i];
}
__device__ __forceinline__ void rp_open8(const Pack8<float> &v, float *f)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        f[4 * i] = __uint_as_float(v.w[i].x); f[4 * i + 1] = __uint_as_float(v.w[i].y);
        f[4 * i + 2] = __uint_as_float(v.w[i].z); f[4 * i + 3] = __uint_as_float(v.w[i].w);
    }
}
__device__ __forceinline__ void rp_open8(const Pack8<bf16> &v, float *f)
{
    const u32 w[4] = { v.w[0].x, v.w[0].y, v.w[0].z, v.w[0].w };
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void rp_open8(const Pack8<__half> &v, float *f)
{
    const u32 w[4] = { v.w[0].x, v.w[0].y, v.w[0].z, v.w[0].w };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __half2 h;
        memcpy(&h, &w[i], 4);
        const float2 x = __half22float2(h);
        f[2 * i] = x.x; f[2 * i + 1] = x.y;
    }
}
__device__ __forceinline__ u32 rp_pair(float a, float b, bf16) { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); u32 w; memcpy(&w, &h, 4); return w; }
__device__ __forceinline__ u32 rp_pair(float a, float b, __half) { const __half2 h = __floats2half2_rn(a, b); u32 w; memcpy(&w, &h, 4); return w; }
template <typename X> __device__ __forceinline__ Pack8<X> rp_close8(const float *f)
{
    Pack8<X> v;
    v.w[0] = make_uint4(rp_pair(f[0], f[1], X()), rp_pair(f[2], f[3], X()), rp_pair(f[4], f[5], X()), rp_pair(f[6], f[7], X()));
    return v;
}
template <> __device__ __forceinline__ Pack8<float> rp_close8<float>(const float *f)
{
    Pack8<float> v;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        v.w[i] = make_uint4(__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]), __float_as_uint(f[4 * i + 2]), __float_as_uint(f[4 * i + 3]));
    return v;
}

// Two floats that one instruction works on.
struct f2 { u64 v; };
__device__ __forceinline__ f2 rp_f2(float x, float y) { f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(x), "f"(y)); return r; }
__device__ __forceinline__ void rp_parts(f2 a, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(a.v)); }
__device__ __forceinline__ f2 rp_mul(f2 a, f2 b) { f2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ f2 rp_fma(f2 a, f2 b, f2 c) { f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }
__device__ __forceinline__ f2 rp_add(f2 a, f2 b) { f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }

__device__ __forceinline__ float rp_exp2(float x)        // 2^x by the special function unit: 2 ulp
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
#define RP_LOG2E 1.4426950408889634f
__device__ __forceinline__ f2 rp_exp2(f2 x)
{
    float a, b;
    rp_parts(x, a, b);
    return rp_f2(rp_exp2(a), rp_exp2(b));
}

// Launch of `f` for one of the three element types, in a scope where X names it.
#define RP_FOR_TYPE(type, ...)                                     \
    switch (type) {                                                \
        case RP_F32: { typedef float X; __VA_ARGS__; break; }      \
        case RP_F16: { typedef __half X; __VA_ARGS__; break; }     \
        default: { typedef bf16 X; __VA_ARGS__; break; }           \
    }
