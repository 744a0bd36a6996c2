// Layer normalisation of node rows and its backward pass (contracts in include/sar.h):
//   xhat = (x - mean) rstd,  y = gamma xhat + beta,  mean and 1/rstd = sqrt(var + eps) taken over a row's C columns;
//   g = gamma gy,  gx = rstd (g - <g, 1>/C - xhat <g, xhat>/C),  dgamma = sum over the rows of gy xhat,  dbeta = sum of gy.
// Each pass reads and writes its arrays once and is bound by memory where rows are whole vectors, by instructions otherwise.  A group of G lanes holds a row in registers between its
// sums and its result, so the variance is the mean of squared deviations (no cancellation) without a second read; the sums
// over the rows are carried in registers from row to row, then one record per block, which a second launch adds up in a fixed
// order (no atomics).  With a checkpoint the normalised rows leave the forward pass as 8-bit codes as well, and the backward
// pass reads those in place of x and mean.
#include "sar_ln.cuh"
#include "sar_reduce.cuh"

namespace sar {

static sar_status ln_check(int32_t C, sar_dtype t) {
    if (t != SAR_F32 && t != SAR_BF16) return SAR_ERR_INVALID_ARG;
    return C > kLnMostColumns ? SAR_ERR_UNSUPPORTED : SAR_OK;
}

static sar_status ln_zero(int32_t C, float *dgamma, float *dbeta, cudaStream_t st) {
    for (float *p : {dgamma, dbeta})
        if (p) SAR_CUDA_TRY(cudaMemsetAsync(p, 0, (size_t)C * 4, st));
    return SAR_OK;
}

}  // namespace sar

using namespace sar;

extern "C" {

size_t sar_ln_workspace_bytes_rows(int64_t n, int32_t C) {
    if (n < 0 || C < 1 || C > kLnMostColumns) return 0;
    return (size_t)ln_records_most(n, C) * 2 * C * 4 + 256;
}
size_t sar_ln_workspace_bytes(int32_t C) { return sar_ln_workspace_bytes_rows(INT64_MAX, C); }

static sar_status ln_fwd_entry(int64_t n, int32_t C, sar_dtype t, const void *x, const float *gamma, const float *beta, float eps, void *y,
                               float *mean, float *rstd, int8_t *codes, uint8_t *scales, bool ckpt, void *stream) {
    if (n < 0 || C < 1 || !(eps >= 0.f) || (n > 0 && (!x || !y || (ckpt && (!rstd || !codes || !scales))))) return SAR_ERR_INVALID_ARG;
    SAR_TRY(ln_check(C, t));
    const LnShape s = ln_shape(C, t, kLnFwd, ln_alignment({x, y}), ln_alignment({codes}));
    SAR_TRY(check_elem_align({mean, rstd, gamma, beta}, 4));
    SAR_TRY(check_elem_align({x, y}, sar_elem_size(t)));
    if (n == 0) return SAR_OK;
    LnArgs a = ln_args(n, C);
    a.x = x;
    a.y = y;
    a.gamma = gamma;
    a.beta = beta;
    a.eps = eps;
    a.mean = mean;
    a.rstd = rstd;
    a.codes = codes;
    a.scales = scales;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return (t == SAR_F32 ? ln_forward_f32 : ln_forward_bf16)(s, a, ckpt, st);
}

sar_status sar_ln_fwd(int64_t n, int32_t C, sar_dtype t, const void *x, const float *gamma, const float *beta, float eps, void *y,
                      float *mean, float *rstd, void *stream) {
    return ln_fwd_entry(n, C, t, x, gamma, beta, eps, y, mean, rstd, nullptr, nullptr, false, stream);
}

sar_status sar_ln_fwd_ckpt8(int64_t n, int32_t C, sar_dtype t, const void *x, const float *gamma, const float *beta, float eps, void *y,
                            float *rstd, int8_t *codes, uint8_t *scales, void *stream) {
    return ln_fwd_entry(n, C, t, x, gamma, beta, eps, y, nullptr, rstd, codes, scales, true, stream);
}

static sar_status ln_bwd_entry(int64_t n, bool grouped, int32_t groups, const int64_t *offsets, int32_t C, sar_dtype t, const void *x, const float *mean, const int8_t *codes, const uint8_t *scales,
                               bool ckpt, const float *rstd, const float *gamma, const void *gy, void *gx, float *dgamma, float *dbeta,
                               void *workspace, size_t workspace_bytes, void *stream) {
    if (n < 0 || C < 1 || (n > 0 && (!rstd || !gy || !gx || (ckpt ? !codes || !scales : !x || !mean)))) return SAR_ERR_INVALID_ARG;
    if (grouped && (groups < 1 || (!offsets && n > 0))) return SAR_ERR_INVALID_ARG;
    SAR_TRY(ln_check(C, t));
    if (grouped && groups > SAR_MAX_GROUPS) return SAR_ERR_UNSUPPORTED;
    SAR_TRY(check_elem_align({offsets}, 8));
    const LnShape s = ln_shape(C, t, ckpt ? kLnBwd8 : kLnBwd, ln_alignment({x, gy, gx}), ln_alignment({codes}));
    SAR_TRY(check_elem_align({mean, rstd, gamma, dgamma, dbeta}, 4));
    SAR_TRY(check_elem_align({x, gy, gx}, sar_elem_size(t)));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (n == 0) return ln_zero(C, dgamma, dbeta, st);
    LnGroupedArgs a{ln_args(n, C), offsets, groups};
    a.x = x;
    a.gy = gy;
    a.y = gx;
    a.gamma = gamma;
    a.mean_in = mean;
    a.rstd_in = rstd;
    a.codes = const_cast<int8_t *>(codes);
    a.scales = const_cast<uint8_t *>(scales);
    const bool sums = dgamma || dbeta;
    if (sums) {
        if (!workspace || !sar_aligned(workspace, 16) || workspace_bytes < (size_t)ln_records_most(n, C) * 2 * C * 4) return SAR_ERR_WORKSPACE;
        a.partial = static_cast<float *>(workspace);
    }
    unsigned records = 0;
    if (grouped) SAR_TRY((t == SAR_F32 ? ln_backward_grouped_f32 : ln_backward_grouped_bf16)(s, a, ckpt, &records, st));
    else SAR_TRY((t == SAR_F32 ? ln_backward_f32 : ln_backward_bf16)(s, a, ckpt, &records, st));
    return sums ? reduce_partials("ln_reduce", (int)records, 2 * C, C, a.partial, 1.0, dgamma, dbeta, st) : SAR_OK;
}

sar_status sar_ln_bwd(int64_t n, int32_t C, sar_dtype t, const void *x, const float *mean, const float *rstd, const float *gamma,
                      const void *gy, void *gx, float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes, void *stream) {
    return ln_bwd_entry(n, false, 0, nullptr, C, t, x, mean, nullptr, nullptr, false, rstd, gamma, gy, gx, dgamma, dbeta, workspace, workspace_bytes, stream);
}

sar_status sar_ln_bwd_grouped(int64_t n, int32_t groups, int32_t C, sar_dtype t, const int64_t *offsets, const void *x, const float *mean,
                              const float *rstd, const float *gamma, const void *gy, void *gx, float *dgamma, float *dbeta,
                              void *workspace, size_t workspace_bytes, void *stream) {
    return ln_bwd_entry(n, true, groups, offsets, C, t, x, mean, nullptr, nullptr, false, rstd, gamma, gy, gx, dgamma, dbeta, workspace, workspace_bytes, stream);
}

sar_status sar_ln_bwd_ckpt8(int64_t n, int32_t C, sar_dtype t, const int8_t *codes, const uint8_t *scales, const float *rstd,
                            const float *gamma, const void *gy, void *gx, float *dgamma, float *dbeta, void *workspace,
                            size_t workspace_bytes, void *stream) {
    return ln_bwd_entry(n, false, 0, nullptr, C, t, nullptr, nullptr, codes, scales, true, rstd, gamma, gy, gx, dgamma, dbeta, workspace, workspace_bytes, stream);
}

sar_status sar_ln_bwd_ckpt8_grouped(int64_t n, int32_t groups, int32_t C, sar_dtype t, const int64_t *offsets, const int8_t *codes,
                                    const uint8_t *scales, const float *rstd, const float *gamma, const void *gy, void *gx, float *dgamma,
                                    float *dbeta, void *workspace, size_t workspace_bytes, void *stream) {
    return ln_bwd_entry(n, true, groups, offsets, C, t, nullptr, nullptr, codes, scales, true, rstd, gamma, gy, gx, dgamma, dbeta, workspace, workspace_bytes, stream);
}

}  // extern "C"
