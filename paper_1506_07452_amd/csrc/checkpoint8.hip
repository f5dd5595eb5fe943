// 8-bit activation checkpoints: pack and unpack (format in code8.h).
#include "code8.h"
#include "timing.h"

namespace plstm {
namespace {

constexpr int kPackThreads = 256;

// A wave per block of 64 elements, a lane per element.
template <typename T>
__global__ void __launch_bounds__(kPackThreads)
k_pack8(const T *__restrict__ x, int8_t *__restrict__ q, uint16_t *__restrict__ scale, long long n)
{
    const long long i = (long long)blockIdx.x * kPackThreads + threadIdx.x;
    const float v = i < n ? Store<T>::load(x, i) : 0.0f;
    uint32_t top = float_bits(v) & 0x7fffffffu;
    for (int d = 32; d; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    const uint16_t s = code_scale(top);
    if (i >= n) return;
    const Coder c(s);
    q[i] = (int8_t)c.code(v);
    if ((i & 63) == 0) scale[i >> 6] = s;
}

template <typename T>
__global__ void __launch_bounds__(kPackThreads)
k_unpack8(const int8_t *__restrict__ q, const uint16_t *__restrict__ scale, T *__restrict__ x,
          long long n)
{
    const long long i = (long long)blockIdx.x * kPackThreads + threadIdx.x;
    if (i >= n) return;
    Store<T>::store(x, i, (float)q[i] * bf16_to_f32(scale[i >> 6]));
}

}  // namespace

int checkpoint8_pack(long long n, int dtype, const void *x, int8_t *q, uint16_t *scale,
                     hipStream_t st)
{
    const unsigned grid = (unsigned)((n + kPackThreads - 1) / kPackThreads);
    if (dtype == PLSTM_F32)
        k_pack8<<<grid, kPackThreads, 0, st>>>((const float *)x, q, scale, n);
    else
        k_pack8<<<grid, kPackThreads, 0, st>>>((const uint16_t *)x, q, scale, n);
    PLSTM_LAUNCH_CHECK();
    return PLSTM_OK;
}

}  // namespace plstm

using namespace plstm;

extern "C" {

int64_t pyramid_checkpoint8_scales(int64_t n) { return n < 1 ? 0 : code_blocks(n); }

int pyramid_checkpoint8_pack(int64_t n, int32_t dtype, const void *x, void *q, void *scale,
                             void *stream)
{
    if (n < 1 || (dtype != PLSTM_F32 && dtype != PLSTM_BF16)) return PLSTM_EINVAL;
    if (!x || !q || !scale || !aligned_to(x, 16) || !aligned_to(q, 16) || !aligned_to(scale, 16))
        return PLSTM_EINVAL;
    if (n > (1LL << 38)) return PLSTM_EUNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    timing_begin("pack8", st);
    const int rc = checkpoint8_pack(n, dtype, x, (int8_t *)q, (uint16_t *)scale, st);
    if (rc == PLSTM_OK) timing_end(1, st);
    return rc;
}

int pyramid_checkpoint8_unpack(int64_t n, int32_t dtype, const void *q, const void *scale,
                               void *x, void *stream)
{
    if (n < 1 || (dtype != PLSTM_F32 && dtype != PLSTM_BF16)) return PLSTM_EINVAL;
    if (!x || !q || !scale || !aligned_to(x, 16) || !aligned_to(q, 16) || !aligned_to(scale, 16))
        return PLSTM_EINVAL;
    if (n > (1LL << 38)) return PLSTM_EUNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    const unsigned grid = (unsigned)((n + kPackThreads - 1) / kPackThreads);
    timing_begin("unpack8", st);
    if (dtype == PLSTM_F32)
        k_unpack8<<<grid, kPackThreads, 0, st>>>((const int8_t *)q, (const uint16_t *)scale,
                                                 (float *)x, n);
    else
        k_unpack8<<<grid, kPackThreads, 0, st>>>((const int8_t *)q, (const uint16_t *)scale,
                                                 (uint16_t *)x, n);
    PLSTM_LAUNCH_CHECK();
    timing_end(1, st);
    return PLSTM_OK;
}

}  // extern "C"
