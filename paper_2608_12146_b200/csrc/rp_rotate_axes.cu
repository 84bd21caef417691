// Rotation by positions on several axes: the entries.
#include "rp_rotate.cuh"

extern "C" int rp_rotate_axes(const rp_rotary *r, int64_t n_tokens, const double *inv_freq, const rp_axes *axes, const rp_heads *q, const rp_heads *k,
                              void *cuda_stream)
{
    return rotate<true>(r, n_tokens, inv_freq, nullptr, 0, nullptr, axes, q, k, false, nullptr, 0, (cudaStream_t)cuda_stream);
}

extern "C" int rp_rotate_axes_grad(const rp_rotary *r, int64_t n_tokens, const double *inv_freq, const rp_axes *axes, const rp_heads *q, const rp_heads *k,
                                   void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    return rotate<true>(r, n_tokens, inv_freq, nullptr, 0, nullptr, axes, q, k, true, (float *)workspace, workspace_bytes, (cudaStream_t)cuda_stream);
}
