// Sequences of [B][T][I] tensors for the convolution and the selective scan (host and
// device): positions of a sweep, rows with a pitch, activations.
#pragma once

#include "rows.h"

namespace plstm {

// Position s = 0 .. n - 1 of a sequence of n steps is step s, or n - 1 - s in reverse.
// Positions from n on hold nothing and stand for the steps of the same number.
__device__ inline long long step_of(long long s, long long n, int reverse)
{
    return reverse && s < n ? n - 1 - s : s;
}
__device__ inline long long length_of(const int32_t *lengths, long long b, long long T)
{
    if (!lengths) return T;
    const long long n = lengths[b];
    return n < 0 ? 0 : n > T ? T : n;
}

// sigmoid; exp(-|a|) <= 1, so nothing overflows.
__device__ inline float sigmoid_of(float a)
{
    const float e = __builtin_amdgcn_exp2f(fabsf(a) * -1.44269504f);
    const float r = __builtin_amdgcn_rcpf(1.0f + e);
    return a < 0.0f ? e * r : r;
}
// SiLU a sigmoid(a), and its derivative sigmoid (1 + a (1 - sigmoid)); 1 - sigmoid is
// sigmoid(-a), not a difference.
__device__ inline float silu_of(float a) { return a * sigmoid_of(a); }
__device__ inline float silu_slope(float a, float &silu)
{
    const float e = __builtin_amdgcn_exp2f(fabsf(a) * -1.44269504f);
    const float r = __builtin_amdgcn_rcpf(1.0f + e), x = e * r;
    const float s = a < 0.0f ? x : r, t = a < 0.0f ? r : x;
    silu = a * s;
    return s * fmaf(a, t, 1.0f);
}

// A launch has fewer than 2^32 work items.  Calls launch(first, workgroups) for pieces of at most half of that of `all` workgroups of
// THREADS; returns the number of launches.
template <int THREADS, typename F>
inline int in_launches(long long all, F launch)
{
    constexpr long long most = (1LL << 31) / THREADS;
    int n = 0;
    for (long long first = 0; first < all; first += most, ++n)
        launch((unsigned)first, (unsigned)(all - first < most ? all - first : most));
    return n;
}

// Pieces of tensors too large for the caches: read for the last time, or written for a later launch.  Non-temporal accesses
// leave the caches to what is read twice, and no written lines behind that the next launch waits to have written back: group norm of
// 1 x 2764800 x 16 fp32 248 us, without 297, of 8 x 262144 x 64 bf16 388, 454; the convolution of 2 x 8192 x 2048 92, 96;
// AdamW of 66 million elements 329, 345.  Smaller ones make no difference here and may be in a cache for their reader.
constexpr long long kStreamBytes = 64LL << 20;      // of a tensor, from which on it is accessed so
template <bool STREAM, typename T>
__device__ inline u32x4 load_last(const T *p, int have)
{
    if (STREAM && have >= Piece<T>::N) return __builtin_nontemporal_load((const typename Piece<T>::V *)p);
    return load_piece<T>(p, have);
}
template <bool STREAM, typename T>
__device__ inline void store_out(T *p, int have, const float *v)
{
    if (STREAM && have >= Piece<T>::N) {
        const typename Piece<T>::V w = Piece<T>::packed(v);
        __builtin_nontemporal_store(w, (typename Piece<T>::V *)p);
    } else {
        store_piece<T>(p, have, v);
    }
}

// 4 elements from any element on: 16 bytes of fp32, 8 of bf16; raw bits.
template <typename T> struct Four;
template <> struct Four<float> {
    u32x4 w;
    __device__ void load(const float *p, int have) { w = load_piece<float>(p, have); }
    __device__ void get(float *v) const { Piece<float>::unpack(w, v); }
    __device__ void zero() { w = u32x4{0, 0, 0, 0}; }
    template <bool STREAM = false>
    __device__ static void store(float *p, int have, const float *v) { store_out<STREAM>(p, have, v); }
};
template <> struct Four<uint16_t> {
    typedef uint32_t V __attribute__((ext_vector_type(2), aligned(2)));
    uint32_t w[2];
    __device__ void load(const uint16_t *p, int have)
    {
        if (have >= 4) {
            const V r = *(const V *)p;
            w[0] = r[0];
            w[1] = r[1];
        } else {
            w[0] = have > 0 ? p[0] : 0;
            w[0] |= have > 1 ? (uint32_t)p[1] << 16 : 0;
            w[1] = have > 2 ? p[2] : 0;
        }
    }
    __device__ void get(float *v) const
    {
        v[0] = bits_float(w[0] << 16);
        v[1] = bits_float(w[0] & 0xffff0000u);
        v[2] = bits_float(w[1] << 16);
        v[3] = bits_float(w[1] & 0xffff0000u);
    }
    __device__ void zero() { w[0] = w[1] = 0; }
    template <bool STREAM = false>
    __device__ static void store(uint16_t *p, int have, const float *v)
    {
        if (have >= 4) {
            const V w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            if (STREAM) __builtin_nontemporal_store(w, (V *)p);
            else *(V *)p = w;
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (j < have) p[j] = (uint16_t)pack_bf16(v[j], v[j]);
        }
    }
};

}  // namespace plstm
