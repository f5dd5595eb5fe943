// Layer norm over the channels of each row, and its backward pass.
//   mean = sum_c x / C, var = sum_c (x - mean)^2 / C, rstd = 1 / sqrt(var + eps)
//   y = (x - mean) rstd gamma + beta
// Backward, with xh = (x - mean) rstd and a = dy gamma:
//   dx = rstd (a - sum_c a / C - xh sum_c (a xh) / C)
//   dgamma = sum_m dy xh, dbeta = sum_m dy
// Rows are read in the storage type or, in the backward, from an 8-bit
// checkpoint (code8.h); sums and statistics are fp32.
#include "code8.h"
#include "timing.h"

namespace plstm {
namespace {

constexpr int kNormThreads = 256;
constexpr int kNormParts = 256;     // row ranges of the weights' gradients
constexpr int kNormMaxC = 16384;

__device__ inline float wave_sum(float v)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

template <typename T>
__device__ inline float load_row(const T *x, const uint16_t *, long long i)
{
    return Store<T>::load(x, i);
}
__device__ inline float load_row(const int8_t *x, const uint16_t *scale, long long i)
{
    return (float)x[i] * bf16_to_f32(scale[i >> 6]);
}

// A wave per row.
template <typename T>
__global__ void __launch_bounds__(kNormThreads)
k_norm_fwd(const T *__restrict__ x, const T *__restrict__ gamma, const T *__restrict__ beta,
           T *__restrict__ y, float2 *__restrict__ stats, long long M, int C, float eps)
{
    const long long m = (long long)blockIdx.x * (kNormThreads / 64) + threadIdx.x / 64;
    if (m >= M) return;
    const int lane = threadIdx.x & 63;
    const long long at = m * C;
    float s = 0.0f;
    for (int c = lane; c < C; c += 64) s += Store<T>::load(x, at + c);
    const float mean = wave_sum(s) / (float)C;
    float v = 0.0f;
    for (int c = lane; c < C; c += 64) {
        const float d = Store<T>::load(x, at + c) - mean;
        v += d * d;
    }
    const float rstd = 1.0f / sqrtf(wave_sum(v) / (float)C + eps);
    for (int c = lane; c < C; c += 64)
        Store<T>::store(y, at + c,
                        (Store<T>::load(x, at + c) - mean) * rstd * Store<T>::load(gamma, c) +
                            Store<T>::load(beta, c));
    if (stats && lane == 0) stats[m] = make_float2(mean, rstd);
}

template <typename T, typename X>
__global__ void __launch_bounds__(kNormThreads)
k_norm_dx(const X *__restrict__ x, const uint16_t *__restrict__ xscale,
          const T *__restrict__ gamma, const float2 *__restrict__ stats,
          const T *__restrict__ dy, T *__restrict__ dx, long long M, int C)
{
    const long long m = (long long)blockIdx.x * (kNormThreads / 64) + threadIdx.x / 64;
    if (m >= M) return;
    const int lane = threadIdx.x & 63;
    const long long at = m * C;
    const float2 st = stats[m];
    float sa = 0.0f, sb = 0.0f;
    for (int c = lane; c < C; c += 64) {
        const float a = Store<T>::load(dy, at + c) * Store<T>::load(gamma, c);
        sa += a;
        sb += a * ((load_row(x, xscale, at + c) - st.x) * st.y);
    }
    sa = wave_sum(sa) / (float)C;
    sb = wave_sum(sb) / (float)C;
    for (int c = lane; c < C; c += 64) {
        const float a = Store<T>::load(dy, at + c) * Store<T>::load(gamma, c);
        const float xh = (load_row(x, xscale, at + c) - st.x) * st.y;
        Store<T>::store(dx, at + c, st.y * (a - sa - xh * sb));
    }
}

// Partial sums of dgamma and dbeta over the rows m = part, part + kNormParts, ...
// part [kNormParts][2][C].
template <typename T, typename X>
__global__ void __launch_bounds__(kNormThreads)
k_norm_dw(const X *__restrict__ x, const uint16_t *__restrict__ xscale,
          const float2 *__restrict__ stats, const T *__restrict__ dy, float *__restrict__ part,
          long long M, int C)
{
    const int c = blockIdx.x * kNormThreads + threadIdx.x;
    if (c >= C) return;
    float g = 0.0f, b = 0.0f;
    for (long long m = blockIdx.y; m < M; m += kNormParts) {
        const float2 st = stats[m];
        const float d = Store<T>::load(dy, m * C + c);
        g += d * ((load_row(x, xscale, m * C + c) - st.x) * st.y);
        b += d;
    }
    part[(long long)blockIdx.y * 2 * C + c] = g;
    part[(long long)blockIdx.y * 2 * C + C + c] = b;
}

__global__ void __launch_bounds__(kNormThreads)
k_norm_dw_sum(const float *__restrict__ part, float *__restrict__ dgamma,
              float *__restrict__ dbeta, int C)
{
    const int c = blockIdx.x * kNormThreads + threadIdx.x;
    if (c >= 2 * C) return;
    float s = 0.0f;
    for (int k = 0; k < kNormParts; ++k) s += part[(long long)k * 2 * C + c];
    (c < C ? dgamma[c] : dbeta[c - C]) = s;
}

int check_rows(int64_t M, int32_t C, int32_t dtype)
{
    if (M < 1 || C < 1) return PLSTM_EINVAL;
    if (dtype != PLSTM_F32 && dtype != PLSTM_BF16) return PLSTM_EINVAL;
    if (C > kNormMaxC || M > (1LL << 32) || M > (1LL << 38) / C) return PLSTM_EUNSUPPORTED;
    return PLSTM_OK;
}

template <typename T, typename X>
int norm_backward(long long M, int C, const X *x, const uint16_t *xscale, const T *gamma,
                  const float2 *stats, const T *dy, T *dx, float *dgamma, float *dbeta,
                  float *part, hipStream_t st)
{
    if (dx) {
        k_norm_dx<T, X><<<(unsigned)((M + 3) / 4), kNormThreads, 0, st>>>(x, xscale, gamma, stats,
                                                                         dy, dx, M, C);
        PLSTM_LAUNCH_CHECK();
    }
    const unsigned cols = (unsigned)((C + kNormThreads - 1) / kNormThreads);
    k_norm_dw<T, X><<<dim3(cols, kNormParts), kNormThreads, 0, st>>>(x, xscale, stats, dy, part,
                                                                    M, C);
    PLSTM_LAUNCH_CHECK();
    k_norm_dw_sum<<<(unsigned)((2 * C + kNormThreads - 1) / kNormThreads), kNormThreads, 0, st>>>(
        part, dgamma, dbeta, C);
    PLSTM_LAUNCH_CHECK();
    return PLSTM_OK;
}

template <typename T>
int norm_backward_from(long long M, int C, const void *x, const void *xscale, const void *gamma,
                       const void *stats, const void *dy, void *dx, void *dgamma, void *dbeta,
                       void *ws, hipStream_t st)
{
    if (xscale)
        return norm_backward<T, int8_t>(M, C, (const int8_t *)x, (const uint16_t *)xscale,
                                        (const T *)gamma, (const float2 *)stats, (const T *)dy,
                                        (T *)dx, (float *)dgamma, (float *)dbeta, (float *)ws, st);
    return norm_backward<T, T>(M, C, (const T *)x, nullptr, (const T *)gamma,
                               (const float2 *)stats, (const T *)dy, (T *)dx, (float *)dgamma,
                               (float *)dbeta, (float *)ws, st);
}

}  // namespace
}  // namespace plstm

using namespace plstm;

extern "C" {

size_t pyramid_layer_norm_workspace_size(int64_t M, int32_t C)
{
    if (check_rows(M, C, PLSTM_F32) != PLSTM_OK) return 0;
    return align_up((size_t)kNormParts * 2 * C * sizeof(float), 256);
}

int pyramid_layer_norm_forward(int64_t M, int32_t C, int32_t dtype, float eps, const void *x,
                               const void *gamma, const void *beta, void *y, void *stats,
                               void *xq, void *xscale, void *stream)
{
    const int rc = check_rows(M, C, dtype);
    if (rc != PLSTM_OK) return rc;
    if (!(eps > 0.0f) || !x || !gamma || !beta || !y || !xq != !xscale) return PLSTM_EINVAL;
    const size_t e = dtype_size(dtype);
    if (!aligned_to(x, e) || !aligned_to(gamma, e) || !aligned_to(beta, e) || !aligned_to(y, e) ||
        !aligned_to(stats, 8) || !aligned_to(xq, 16) || !aligned_to(xscale, 16))
        return PLSTM_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    timing_begin("norm_fwd", st);
    if (xq) {
        const int prc = checkpoint8_pack((long long)M * C, dtype, x, (int8_t *)xq,
                                         (uint16_t *)xscale, st);
        if (prc != PLSTM_OK) return prc;
    }
    const unsigned grid = (unsigned)((M + 3) / 4);
    if (dtype == PLSTM_F32)
        k_norm_fwd<<<grid, kNormThreads, 0, st>>>((const float *)x, (const float *)gamma,
                                                  (const float *)beta, (float *)y,
                                                  (float2 *)stats, M, C, eps);
    else
        k_norm_fwd<<<grid, kNormThreads, 0, st>>>((const uint16_t *)x, (const uint16_t *)gamma,
                                                  (const uint16_t *)beta, (uint16_t *)y,
                                                  (float2 *)stats, M, C, eps);
    PLSTM_LAUNCH_CHECK();
    timing_end(xq ? 2 : 1, st);
    return PLSTM_OK;
}

int pyramid_layer_norm_backward(int64_t M, int32_t C, int32_t dtype, const void *x,
                                const void *xscale, const void *gamma, const void *stats,
                                const void *dy, void *dx, void *dgamma, void *dbeta, void *ws,
                                size_t ws_bytes, void *stream)
{
    int rc = check_rows(M, C, dtype);
    if (rc != PLSTM_OK) return rc;
    if (!x || !gamma || !stats || !dy || !dgamma || !dbeta || !ws) return PLSTM_EINVAL;
    const size_t e = dtype_size(dtype);
    if (!aligned_to(x, xscale ? 16 : e) || !aligned_to(xscale, 16) || !aligned_to(gamma, e) ||
        !aligned_to(stats, 8) || !aligned_to(dy, e) || !aligned_to(dx, e) ||
        !aligned_to(dgamma, 4) || !aligned_to(dbeta, 4) || !aligned_to(ws, 16))
        return PLSTM_EINVAL;
    if (ws_bytes < pyramid_layer_norm_workspace_size(M, C)) return PLSTM_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    timing_begin("norm_bwd", st);
    rc = dtype == PLSTM_F32
             ? norm_backward_from<float>(M, C, x, xscale, gamma, stats, dy, dx, dgamma, dbeta, ws,
                                         st)
             : norm_backward_from<uint16_t>(M, C, x, xscale, gamma, stats, dy, dx, dgamma, dbeta,
                                            ws, st);
    if (rc == PLSTM_OK) timing_end(dx ? 3 : 2, st);
    return rc;
}

}  // extern "C"
