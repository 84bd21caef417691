// Rotation by the position in the sample: the entries.
#include "rp_rotate.cuh"

extern "C" int rp_rotate(const rp_rotary *r, int64_t n_tokens, const double *inv_freq, const int64_t *start, int32_t n_samples,
                         const int64_t *first_position, const rp_heads *q, const rp_heads *k, void *cuda_stream)
{
    return rotate<false>(r, n_tokens, inv_freq, (const i64 *)start, n_samples, (const i64 *)first_position, nullptr, q, k, false, nullptr, 0, (cudaStream_t)cuda_stream);
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
    return rotate<false>(r, n_tokens, inv_freq, (const i64 *)start, n_samples, (const i64 *)first_position, nullptr, q, k, true, (float *)workspace, workspace_bytes,
                  (cudaStream_t)cuda_stream);
}
