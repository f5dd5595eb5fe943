// 8-bit activation checkpoints: pack and unpack (format in code8.h).
#include "rows.h"
#include "timing.h"

namespace plstm {
namespace {

constexpr int kPackThreads = 256;
constexpr int kPackUnroll = 4;      // pieces of 16 bytes that a lane has in flight
constexpr int kPackBlocks = 4096;

// Bound by bytes: 25165824 fp32 values in 23 us (5.5 TB/s), 134217728 bf16 values in 76
// to 89 us (4.6 to 5.4 TB/s).
// A lane per 16 bytes of x; a block of 64 elements is 16 lanes (fp32) or 8
// (bf16).  A workgroup takes kPackUnroll consecutive stretches of a piece a lane,
// all loaded before the first is coded.
template <typename T>
__global__ void __launch_bounds__(kPackThreads)
k_pack8(const T *__restrict__ x, int8_t *__restrict__ q, uint16_t *__restrict__ scale, long long n)
{
    constexpr int N = Piece<T>::N;
    constexpr long long stretch = (long long)kPackThreads * N;
    for (long long at0 = blockIdx.x * stretch * kPackUnroll + threadIdx.x * N; at0 - threadIdx.x * N < n;
         at0 += gridDim.x * stretch * kPackUnroll) {
        u32x4 raw[kPackUnroll];
#pragma unroll
        for (int t = 0; t < kPackUnroll; ++t) {
            const long long at = at0 + t * stretch, left = n - at;
            raw[t] = load_piece(x + at, left > N ? N : (int)left);
        }
        loads_issued();
#pragma unroll
        for (int t = 0; t < kPackUnroll; ++t) {
            const long long at = at0 + t * stretch, left = n - at;
            float v[N];
            Piece<T>::unpack(raw[t], v);
            const uint16_t s = code_scale(lanes_max<kCodeBlock / N>(top_bits<N>(v)));
            const Coder c(s);
            uint32_t code[N];
            code_piece<T>(c, v, code);
            store_codes<N>(q + at, left > N ? N : (int)left, code, c.keep);
            if ((at & (kCodeBlock - 1)) == 0 && left > 0) scale[at >> 6] = s;
        }
    }
}

// The same shape the other way round: 20 us (6.2 TB/s, the codes still in the cache) and
// 65 us (6.3 TB/s).
template <typename T>
__global__ void __launch_bounds__(kPackThreads)
k_unpack8(const int8_t *__restrict__ q, const uint16_t *__restrict__ scale, T *__restrict__ x,
          long long n)
{
    constexpr int N = Piece<T>::N;
    constexpr long long stretch = (long long)kPackThreads * N;
    for (long long at0 = blockIdx.x * stretch * kPackUnroll + threadIdx.x * N; at0 < n;
         at0 += gridDim.x * stretch * kPackUnroll) {
        RawCodes<N> raw[kPackUnroll];
#pragma unroll
        for (int t = 0; t < kPackUnroll; ++t) {
            const long long at = at0 + t * stretch, left = n - at;
            raw[t] = load_coded<N>(q, scale, at, left > N ? N : (int)left);
        }
        loads_issued();
#pragma unroll
        for (int t = 0; t < kPackUnroll; ++t) {
            const long long at = at0 + t * stretch, left = n - at;
            float v[N];
            unpack_coded<N>(raw[t], at, v);
            store_piece(x + at, left > N ? N : (int)left, v);
        }
    }
}

unsigned pack_grid(long long n, int dtype)
{
    const long long each = (long long)kPackThreads * kPackUnroll * (dtype == PLSTM_F32 ? 4 : 8);
    const long long blocks = (n + each - 1) / each;
    return (unsigned)(blocks < kPackBlocks ? blocks : kPackBlocks);
}

}  // namespace

int checkpoint8_pack(long long n, int dtype, const void *x, int8_t *q, uint16_t *scale,
                     hipStream_t st)
{
    const unsigned grid = pack_grid(n, dtype);
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
    const unsigned grid = pack_grid(n, dtype);
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
