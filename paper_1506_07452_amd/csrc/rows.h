// 16-byte pieces of rows in the storage types, and sums over groups of lanes
// (device side).  Pieces start at any element: global memory takes 16-byte
// accesses at any address, so rows of odd lengths need no other path than a
// last piece that is read and written element by element.
#pragma once

#include "code8.h"

namespace plstm {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Two fp32 values rounded to bf16 (nearest, ties to even; NaN kept quiet) in
// one conversion, the first in the low half.
__device__ inline uint32_t pack_bf16(float a, float b)
{
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// All loads so far are issued before anything that follows.  Loads give raw bits for
// this: left to itself the scheduler converts values as they come, and waits for
// each of a lane's loads in turn.
__device__ inline void loads_issued() { __builtin_amdgcn_sched_barrier(0); }

template <typename T> struct Piece;

template <> struct Piece<float> {
    static constexpr int N = 4;
    typedef uint32_t V __attribute__((ext_vector_type(4), aligned(4)));
    __device__ static void unpack(u32x4 w, float *v)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = bits_float(w[j]);
    }
    __device__ static u32x4 packed(const float *v)
    {
        return u32x4{float_bits(v[0]), float_bits(v[1]), float_bits(v[2]), float_bits(v[3])};
    }
};

template <> struct Piece<uint16_t> {
    static constexpr int N = 8;
    typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2)));
    __device__ static void unpack(u32x4 w, float *v)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = bits_float(w[j] << 16);
            v[2 * j + 1] = bits_float(w[j] & 0xffff0000u);
        }
    }
    __device__ static u32x4 packed(const float *v)
    {
        return u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                     pack_bf16(v[6], v[7])};
    }
};

// Elements [0, have) of a piece; the others read as 0 and are not written.
template <typename T>
__device__ inline u32x4 load_piece(const T *p, int have)
{
    constexpr int N = Piece<T>::N, per = N / 4;
    if (have >= N) return *(const typename Piece<T>::V *)p;
    u32x4 w = {0, 0, 0, 0};
    if (have > 0) {
#pragma unroll
        for (int j = 0; j < N - 1; ++j)
            if (j < have) w[j / per] |= per == 1 ? float_bits(Store<T>::load(p, j))
                                                 : float_bits(Store<T>::load(p, j)) >> 16 << (16 * (j % per));
    }
    return w;
}
template <typename T>
__device__ inline void store_piece(T *p, int have, const float *v)
{
    constexpr int N = Piece<T>::N;
    if (have >= N) {
        *(typename Piece<T>::V *)p = Piece<T>::packed(v);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < have) Store<T>::store(p, j, v[j]);
    }
}

// N = 4 or 8 codes, each in the low byte of its word, as bytes.
template <int N>
__device__ inline void store_codes(int8_t *q, int have, const uint32_t *c, uint32_t keep)
{
    typedef uint32_t V __attribute__((ext_vector_type(N / 4), aligned(1)));
    V w;
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
        const uint32_t lo = __builtin_amdgcn_perm(c[4 * j + 1], c[4 * j], 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(c[4 * j + 3], c[4 * j + 2], 0x04000c0cu);
        w[j] = (lo | hi) & keep;
    }
    if (have >= N) {
        *(V *)q = w;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < have) q[j] = (int8_t)(w[j / 4] >> (8 * (j % 4)));
    }
}

// N codes at flat elements at .. at + have - 1 of a checkpoint, with the scales of
// the blocks that they are in (two at most), in raw bits.
template <int N> struct RawCodes {
    uint32_t w[N / 4];
    uint32_t s0, s1;
};
template <int N>
__device__ inline RawCodes<N> load_coded(const int8_t *q, const uint16_t *scale, long long at,
                                         int have)
{
    typedef uint32_t V __attribute__((ext_vector_type(N / 4), aligned(1)));
    RawCodes<N> r;
#pragma unroll
    for (int j = 0; j < N / 4; ++j) r.w[j] = 0;
    r.s0 = r.s1 = 0;
    if (have <= 0) return r;
    if (have >= N) {
        have = N;
        const V w = *(const V *)(q + at);
#pragma unroll
        for (int j = 0; j < N / 4; ++j) r.w[j] = w[j];
    } else {
#pragma unroll
        for (int j = 0; j < N - 1; ++j)
            if (j < have) r.w[j / 4] |= (uint32_t)(uint8_t)q[at + j] << (8 * (j % 4));
    }
    r.s0 = scale[at >> 6];
    r.s1 = scale[(at + have - 1) >> 6];
    return r;
}
template <int N>
__device__ inline void unpack_coded(const RawCodes<N> &r, long long at, float *v)
{
    const int turn = kCodeBlock - (int)(at & (kCodeBlock - 1));
    const float s0 = bits_float(r.s0 << 16), s1 = bits_float(r.s1 << 16);
#pragma unroll
    for (int j = 0; j < N; ++j)
        v[j] = (float)(int)(int8_t)(r.w[j / 4] >> (8 * (j % 4))) * (j < turn ? s0 : s1);
}

// Largest / sum over aligned groups of G lanes (a power of two <= 64), in every
// lane.  Up to 16 lanes by data-parallel moves: once lanes that differ in the
// lower bits agree, a mirrored half row or row stands for the lane across.
template <int CTRL>
__device__ inline uint32_t moved(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
template <int G, typename F>
__device__ inline uint32_t over_lanes(uint32_t v, F f)
{
    if (G >= 2) v = f(v, moved<0xb1>(v));       // quad_perm 1 0 3 2
    if (G >= 4) v = f(v, moved<0x4e>(v));       // quad_perm 2 3 0 1
    if (G >= 8) v = f(v, moved<0x141>(v));      // row_half_mirror
    if (G >= 16) v = f(v, moved<0x140>(v));     // row_mirror
    if (G >= 32) v = f(v, (uint32_t)__shfl_xor((int)v, 16));
    if (G >= 64) v = f(v, (uint32_t)__shfl_xor((int)v, 32));
    return v;
}
template <int G>
__device__ inline float lanes_sum(float v)
{
    return bits_float(over_lanes<G>(float_bits(v), [](uint32_t a, uint32_t b) {
        return float_bits(bits_float(a) + bits_float(b));
    }));
}
template <int CTRL>
__device__ inline double moved(double v)
{
    const uint64_t w = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = moved<CTRL>((uint32_t)w), hi = moved<CTRL>((uint32_t)(w >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int G>
__device__ inline double lanes_sum(double v)
{
    if (G >= 2) v += moved<0xb1>(v);
    if (G >= 4) v += moved<0x4e>(v);
    if (G >= 8) v += moved<0x141>(v);
    if (G >= 16) v += moved<0x140>(v);
    if (G >= 32) v += __shfl_xor(v, 16);
    if (G >= 64) v += __shfl_xor(v, 32);
    return v;
}
template <int G>
__device__ inline uint32_t lanes_max(uint32_t v)
{
    return over_lanes<G>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

// Bits of the largest magnitude of N values, a NaN the largest of all.
template <int N>
__device__ inline uint32_t top_bits(const float *v)
{
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) top = max(top, float_bits(v[j]) & 0x7fffffffu);
    return top;
}

// Codes of a piece of a block whose largest magnitude has bits `top`.
template <typename T>
__device__ inline void code_piece(const Coder &c, const float *v, uint32_t *q)
{
#pragma unroll
    for (int j = 0; j < Piece<T>::N; ++j)
        q[j] = Piece<T>::N == 8 ? c.code_bf16(v[j]) : c.code(v[j]);
}

}  // namespace plstm
