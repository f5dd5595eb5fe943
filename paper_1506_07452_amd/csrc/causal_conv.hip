// Short causal convolution along the middle axis of [B][T][I], a filter of K taps for each
// channel, and its backward pass.  Over sweep positions s (sequence.h), x_s for s < 0 being
// the state's row K - 1 + s (zeros without one):
//   a_s = bias + sum_k w[k] x_{s - (K - 1) + k},  y_s = act(a_s)
// Backward, with da_s = dy_s act'(a_s), a computed again from x:
//   dx_s = sum_k w[k] da_{s + K - 1 - k}  (+ what the last K - 1 inputs get as the state after),
//   dw[k] = sum_s da_s x_{s - (K - 1) + k},  dbias = sum_s da_s
// A lane has 4 channels and walks a run of positions with the last K inputs in registers,
// so x is read once (and K - 1 rows more a run); everything is bound by bytes.  2 x 8192 x 2048 bf16, 4 taps: forward
// 28 to 34 us (134 MB, 4 to 4.8 TB/s), backward 55 (201 MB, 3.7 TB/s).  The backward waits: its two dozen instructions an element are
// 16 to 20 us, but all lanes run at once, one run each, and a run of 32 positions loads some 15 times one after another (the rows
// before it, single positions at either end, turns of four), nothing ahead of its turn.
#include <algorithm>

#include "sequence.h"
#include "timing.h"

namespace plstm {
namespace {

constexpr int kConvMaxK = 8;
constexpr int kConvThreads = 256;
constexpr int kConvParts = 512, kConvMaxParts = 65535;     // workgroups down the positions, each with a part of dw and dbias

struct ConvArgs {
    long long B, T, I, px;                  // px: elements from one row of x to the next
    int act, reverse;
    const int32_t *lengths;
    int run;                                // positions of a run
    long long runs;                         // of a sequence
    long long pieces;                       // of 4 channels
};

// A lane's run of positions and 4 channels.
struct ConvRun {
    long long b, s0, n;                     // sequence, first position, the sequence's length
    long long i;                            // first channel
    int have, count;                        // channels and positions that there are
    __device__ ConvRun(const ConvArgs &a, long long run_of_all, long long piece)
    {
        b = run_of_all / a.runs;
        s0 = (run_of_all - b * a.runs) * a.run;
        n = length_of(a.lengths, b, a.T);
        i = piece * 4;
        have = (int)min(a.I - i, 4LL);
        count = (int)min(a.T - s0, (long long)a.run);
    }
};

template <typename T, int K>
struct Taps {
    float w[K][4], bias[4];
    __device__ Taps(const T *wp, const T *bp, long long i, int have)
    {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            bias[c] = bp && c < have ? Store<T>::load(bp, i + c) : 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k) w[k][c] = c < have ? Store<T>::load(wp, (i + c) * K + k) : 0.0f;
        }
    }
};

// Row of the input at sweep position s < n (the state's below 0), raw.
template <typename T, int K>
__device__ inline Four<T> input_row(const ConvArgs &a, const ConvRun &r, const T *x, const T *state, long long s)
{
    Four<T> v;
    if (s >= 0)
        v.load(x + (r.b * a.T + step_of(s, r.n, a.reverse)) * a.px + r.i, r.have);
    else if (state)
        v.load(state + (r.b * (K - 1) + (K - 1 + s)) * a.I + r.i, r.have);
    else
        v.zero();
    return v;
}

// One past the inputs that a tap reads moves up.
template <int K>
__device__ inline void shift(float (*w)[4])
{
#pragma unroll
    for (int k = 0; k < K - 1; ++k)
#pragma unroll
        for (int c = 0; c < 4; ++c) w[k][c] = w[k + 1][c];
}

template <typename T, int K, bool STREAM>
__global__ void __launch_bounds__(kConvThreads)
k_conv_fwd(ConvArgs a, const T *x, const T *w, const T *bias, const T *state, T *y, T *state_out)
{
    constexpr int U = 8;
    const long long at = (long long)blockIdx.x * kConvThreads + threadIdx.x;
    const long long ri = at / a.pieces;
    if (ri >= a.B * a.runs) return;
    const ConvRun r(a, ri, at - ri * a.pieces);
    const int live = r.n - r.s0 < 0 ? 0 : (int)min(r.n - r.s0, (long long)r.count);
    T *yb = y + r.b * a.T * a.I + r.i;
    if (live > 0) {
        float win[K][4];                    // inputs of positions s - (K - 1) .. s
        Four<T> raw[U], first[K];
#pragma unroll
        for (int k = 0; k < K - 1; ++k) first[k] = input_row<T, K>(a, r, x, state, r.s0 - (K - 1) + k);
        const Taps<T, K> f(w, bias, r.i, r.have);
#pragma unroll
        for (int k = 0; k < K - 1; ++k) first[k].get(win[k + 1]);
        const auto row = [&](const Four<T> &v, T *to) {
            shift<K>(win);
            v.get(win[K - 1]);
            float o[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                o[c] = f.bias[c];
#pragma unroll
                for (int k = 0; k < K; ++k) o[c] = fmaf(f.w[k][c], win[k][c], o[c]);
                if (a.act) o[c] = silu_of(o[c]);
            }
            Four<T>::template store<STREAM>(to, r.have, o);
        };
        // whole turns of whole pieces where the wave has nothing else: loads that ask nothing
        int p = 0;
        const long long s0 = step_of(r.s0, r.n, a.reverse);
        const T *px = x + (r.b * a.T + s0) * a.px + r.i;
        T *py = yb + s0 * a.I;
        const long long sx = a.reverse ? -a.px : a.px, sy = a.reverse ? -a.I : a.I;
        if (__all(r.have == 4))
            for (; __all(p + U <= live); p += U) {
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u].load(px + u * sx, 4);
                loads_issued();
#pragma unroll
                for (int u = 0; u < U; ++u) row(raw[u], py + u * sy);
                px += U * sx;
                py += U * sy;
            }
        for (; p < live; ++p) {
            raw[0] = input_row<T, K>(a, r, x, state, r.s0 + p);
            row(raw[0], yb + step_of(r.s0 + p, r.n, a.reverse) * a.I);
        }
    }
    const float none[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = live; p < r.count; ++p) Four<T>::store(yb + (r.s0 + p) * a.I, r.have, none);
    // the first run's lane, which has read the state: the state after may be the same memory
    if (K > 1 && state_out && r.s0 == 0) {
        Four<T> last[K];
#pragma unroll
        for (int k = 0; k < K - 1; ++k) last[k] = input_row<T, K>(a, r, x, state, r.n - (K - 1) + k);
        loads_issued();
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
            float v[4];
            last[k].get(v);
            Four<T>::store(state_out + (r.b * (K - 1) + k) * a.I + r.i, r.have, v);
        }
    }
}

// PB pieces across and kConvThreads / PB runs down a workgroup; workgroups walk down the runs
// with the parts of dw and dbias in registers.
// Four waves a SIMD where the registers nearly fit (16-bit inputs, up to 4 taps): 2 x 8192 x 2048 bf16 with 4 taps 54.5 us, with
// the compiler's three 62.6; fp32 68 against 63 with what it then spills, 6 taps 191 against 76.
template <typename T, int K, bool STREAM>
__global__ void __launch_bounds__(kConvThreads, sizeof(T) == 2 && K <= 4 ? 4 : 1)
k_conv_bwd(ConvArgs a, int PB, const T *x, const T *w, const T *bias, const T *state, const T *dy,
           const float *dstate_out, T *dx, float *dstate, float *part)
{
    constexpr int U = 4;
    __shared__ float lds[kConvThreads][4];
    const int across = threadIdx.x % PB, down = threadIdx.x / PB, rows = kConvThreads / PB;
    const long long piece = (long long)blockIdx.x * PB + across;
    float dw[K + 1][4];
#pragma unroll
    for (int k = 0; k <= K; ++k)
#pragma unroll
        for (int c = 0; c < 4; ++c) dw[k][c] = 0.0f;
    const long long all = a.B * a.runs;
    if (piece < a.pieces) {
        const int have = (int)min(a.I - piece * 4, 4LL);
        const Taps<T, K> f(w, bias, piece * 4, have);
        const bool pieces = __all(have == 4);
        for (long long ri = (long long)blockIdx.y * rows + down; ri < all; ri += (long long)gridDim.y * rows) {
            const ConvRun r(a, ri, piece);
            T *dxb = dx + r.b * a.T * a.I + r.i;
            const T *dyb = dy + r.b * a.T * a.I + r.i;
            const int live = r.n - r.s0 < 0 ? 0 : (int)min(r.n - r.s0, (long long)r.count);
            const bool before = r.s0 == 0 && dstate;
            // dx of position s needs da of s .. s + K - 1, dstate's those of 0 .. K - 2
            const int end = live > 0 ? live + K - 1 : before ? K - 1 : 0;
            float win[K][4], daw[K][4];     // inputs up to position p, da of p - (K - 1) .. p
            Four<T> first[K];
#pragma unroll
            for (int k = 0; k < K - 1; ++k) {
                first[k].zero();
                if (end > 0) first[k] = input_row<T, K>(a, r, x, state, min(r.s0 - (K - 1) + k, r.n - 1));
            }
#pragma unroll
            for (int k = 0; k < K - 1; ++k) {
                first[k].get(win[k + 1]);
#pragma unroll
                for (int c = 0; c < 4; ++c) daw[k + 1][c] = 0.0f;
            }
            // takes in position q of the run (own: it is not the next one's); its da
            const auto take = [&](const Four<T> &vx, const Four<T> &vd, bool has, bool own) {
                shift<K>(win);
                shift<K>(daw);
                float g[4];
                vx.get(win[K - 1]);
                vd.get(g);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float v = f.bias[c], silu;
#pragma unroll
                    for (int k = 0; k < K; ++k) v = fmaf(f.w[k][c], win[k][c], v);
                    const float da = !has ? 0.0f : a.act ? g[c] * silu_slope(v, silu) : g[c];
                    daw[K - 1][c] = da;
                    if (own) {
#pragma unroll
                        for (int k = 0; k < K; ++k) dw[k][c] = fmaf(da, win[k][c], dw[k][c]);
                        dw[K][c] += da;
                    }
                }
            };
            // the gradient of position q - (K - 1), which has all its da now
            const auto give = [&](float *v) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    v[c] = 0.0f;
#pragma unroll
                    for (int k = 0; k < K; ++k) v[c] = fmaf(f.w[K - 1 - k][c], daw[k][c], v[c]);
                }
            };
            const auto step = [&](int q) {
                Four<T> vx, vd;
                vx.zero();
                vd.zero();
                const long long s = r.s0 + q;
                if (s < r.n) {
                    vx = input_row<T, K>(a, r, x, state, s);
                    vd.load(dyb + step_of(s, r.n, a.reverse) * a.I, r.have);
                }
                take(vx, vd, s < r.n, q < live);
                const long long o = s - (K - 1);
                if (q >= K - 1 ? q - (K - 1) < live : before) {
                    float v[4];
                    give(v);
                    const long long j = o + (K - 1) - r.n;      // row of the state after that this input is
                    if (dstate_out && j >= 0) {
                        const float *e = dstate_out + (r.b * (K - 1) + j) * a.I + r.i;
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (c < r.have) v[c] += e[c];
                    }
                    if (o >= 0)
                        Four<T>::template store<STREAM>(dxb + step_of(o, r.n, a.reverse) * a.I, r.have, v);
                    else
                        Four<float>::store(dstate + (r.b * (K - 1) + (K - 1 + o)) * a.I + r.i, r.have, v);
                }
            };
            int q = 0;
            for (; q < min(K - 1, end); ++q) step(q);
            // whole turns of whole pieces that the wave's sequences have, not their last ones
            const long long s0 = step_of(r.s0 + q, r.n, a.reverse);
            const T *px = x + (r.b * a.T + s0) * a.px + r.i, *pd = dyb + s0 * a.I;
            const long long sx = a.reverse ? -a.px : a.px, sy = a.reverse ? -a.I : a.I;
            T *po = dxb + (s0 - (a.reverse ? -(K - 1) : K - 1)) * a.I;
            if (pieces)
                for (; __all(q + U <= live && r.s0 + q + U + K - 1 <= r.n); q += U) {
                    Four<T> rx[U], rd[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        rx[u].load(px + u * sx, 4);
                        rd[u].load(pd + u * sy, 4);
                    }
                    loads_issued();
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        float v[4];
                        take(rx[u], rd[u], true, true);
                        give(v);
                        Four<T>::template store<STREAM>(po + u * sy, 4, v);
                    }
                    px += U * sx;
                    pd += U * sy;
                    po += U * sy;
                }
            for (; q < end; ++q) step(q);
            const float none[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int p = live; p < r.count; ++p) Four<T>::store(dxb + (r.s0 + p) * a.I, r.have, none);
        }
    }
    // part [blockIdx.y][I][K + 1]: the sums of the workgroup's rows, in their order
#pragma unroll
    for (int k = 0; k <= K; ++k) {
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 4; ++c) lds[threadIdx.x][c] = dw[k][c];
        __syncthreads();
        for (int o = threadIdx.x; o < PB * 4; o += kConvThreads) {
            const long long i = ((long long)blockIdx.x * PB + o / 4) * 4 + o % 4;
            float s = 0.0f;
            for (int d = 0; d < rows; ++d) s += lds[d * PB + o / 4][o % 4];
            if (i < a.I) part[((long long)blockIdx.y * a.I + i) * (K + 1) + k] = s;
        }
    }
}

// dw [I][K] and dbias [I] from the parts, from workgroup `first` of all on, added in 64 bits: 16 lanes an output, each
// every 16th part, then in the lanes' order.
template <int K>
__global__ void __launch_bounds__(256)
k_conv_weights(unsigned first, long long I, int parts, const float *part, float *dw, float *db)
{
    __shared__ double lds[16][16];
    const int o = threadIdx.x % 16, lane = threadIdx.x / 16;
    const long long at = (long long)(first + blockIdx.x) * 16 + o, all = I * (K + 1);
    double s = 0.0;
    if (at < all)
        for (int p = lane; p < parts; p += 16) s += (double)part[(long long)p * all + at];
    lds[lane][o] = s;
    __syncthreads();
    if (lane || at >= all) return;
    for (int d = 1; d < 16; ++d) s += lds[d][o];
    const long long i = at / (K + 1);
    const int k = (int)(at - i * (K + 1));
    if (k < K) {
        if (dw) dw[i * K + k] = (float)s;
    } else if (db) {
        db[i] = (float)s;
    }
}

int check_conv(int64_t B, int64_t T, int64_t I, int32_t K, int32_t dtype)
{
    if (B < 1 || T < 1 || I < 1 || K < 1) return PLSTM_EINVAL;
    if (dtype != PLSTM_F32 && dtype != PLSTM_BF16) return PLSTM_EINVAL;
    if (K > kConvMaxK || B > (1LL << 30) || T > (1LL << 31) || I > (1LL << 30)) return PLSTM_EUNSUPPORTED;
    if (B > (1LL << 30) / I || T > (1LL << 38) / (B * I)) return PLSTM_EUNSUPPORTED;
    return PLSTM_OK;
}

// Positions of a run: short ones while lanes are few, long ones for little of x twice.  Forward and backward in runs of 8 and of
// 32: 2 x 8192 x 2048 164 us, 92; 2 x 2048 x 512 29, 38; 1 x 512 x 1024 28, 34.
ConvArgs conv_args(int64_t B, int64_t T, int64_t I, int32_t act, int32_t reverse, int64_t px,
                   const int32_t *lengths)
{
    ConvArgs a{B, T, I, px ? px : I, act, reverse, lengths, 32, 0, (I + 3) / 4};
    while (a.run > 8 && B * ((T + a.run - 1) / a.run) * a.pieces < (1LL << 18)) a.run /= 2;
    while (B * ((T + a.run - 1) / a.run) * a.pieces >= (1LL << 31)) a.run *= 2;     // lanes of a launch
    a.runs = (T + a.run - 1) / a.run;
    return a;
}

int conv_across(const ConvArgs &a)
{
    int PB = 1;
    while (PB < 64 && PB < a.pieces) PB *= 2;
    return PB;
}
int conv_parts(const ConvArgs &a)
{
    const long long rows = kConvThreads / conv_across(a);
    const long long need = (a.B * a.runs + rows - 1) / rows;
    // two runs a lane from some point on: what it adds up in 32 bits stays short (the parts are added in 64)
    return (int)(need <= kConvParts ? need : std::min<long long>(std::max<long long>(need / 2, kConvParts), kConvMaxParts));
}

bool conv_pitch(int64_t B, int64_t T, int64_t I, int64_t px)
{
    return px == 0 || (px >= I && (px <= (1LL << 40) / (B * T)));
}

}  // namespace
}  // namespace plstm

using namespace plstm;

extern "C" {

size_t pyramid_causal_conv_workspace_size(int64_t B, int64_t T, int64_t I, int32_t K)
{
    if (check_conv(B, T, I, K, PLSTM_F32) != PLSTM_OK) return 0;
    const ConvArgs a = conv_args(B, T, I, 0, 0, 0, nullptr);
    return align_up((size_t)conv_parts(a) * I * (K + 1) * sizeof(float), 256);
}

int pyramid_causal_conv_forward(int64_t B, int64_t T, int64_t I, int32_t K, int32_t dtype,
                                int32_t act, int32_t reverse, const void *x, int64_t x_pitch,
                                const void *w, const void *bias, const int32_t *lengths,
                                const void *state, void *y, void *state_out, void *stream)
{
    const int rc = check_conv(B, T, I, K, dtype);
    if (rc != PLSTM_OK) return rc;
    const size_t e = dtype_size(dtype);
    if ((reverse != 0 && reverse != 1) || (act != 0 && act != 1) || !x || !w || !y) return PLSTM_EINVAL;
    if (!conv_pitch(B, T, I, x_pitch)) return PLSTM_EINVAL;
    if (!aligned_to(x, e) || !aligned_to(w, e) || !aligned_to(bias, e) || !aligned_to(lengths, 4) ||
        !aligned_to(state, e) || !aligned_to(y, e) || !aligned_to(state_out, e))
        return PLSTM_EINVAL;
    const ConvArgs a = conv_args(B, T, I, act, reverse, x_pitch, lengths);
    const long long lanes = a.B * a.runs * a.pieces;
    const dim3 grid((unsigned)((lanes + kConvThreads - 1) / kConvThreads));
    hipStream_t st = (hipStream_t)stream;
    timing_begin("conv_fwd", st);
    const bool stream_out = B * T * I * (int64_t)e >= kStreamBytes;
    const auto go = [&](auto t, auto fn) {
        typedef decltype(t) S;
        fn<<<grid, kConvThreads, 0, st>>>(a, (const S *)x, (const S *)w, (const S *)bias, (const S *)state, (S *)y,
                                          (S *)state_out);
    };
    const auto run = [&](auto k) {
        constexpr int KK = decltype(k)::value;
        if (dtype == PLSTM_F32)
            go(0.0f, stream_out ? k_conv_fwd<float, KK, true> : k_conv_fwd<float, KK, false>);
        else
            go((uint16_t)0, stream_out ? k_conv_fwd<uint16_t, KK, true> : k_conv_fwd<uint16_t, KK, false>);
    };
    switch (K) {
    case 1: run(std::integral_constant<int, 1>()); break;
    case 2: run(std::integral_constant<int, 2>()); break;
    case 3: run(std::integral_constant<int, 3>()); break;
    case 4: run(std::integral_constant<int, 4>()); break;
    case 5: run(std::integral_constant<int, 5>()); break;
    case 6: run(std::integral_constant<int, 6>()); break;
    case 7: run(std::integral_constant<int, 7>()); break;
    default: run(std::integral_constant<int, 8>()); break;
    }
    PLSTM_LAUNCH_CHECK();
    timing_end(1, st);
    return PLSTM_OK;
}

int pyramid_causal_conv_backward(int64_t B, int64_t T, int64_t I, int32_t K, int32_t dtype,
                                 int32_t act, int32_t reverse, const void *x, int64_t x_pitch,
                                 const void *w, const void *bias, const int32_t *lengths,
                                 const void *state, const void *dy, const void *dstate_out,
                                 void *dx, void *dw, void *db, void *dstate, void *ws,
                                 size_t ws_bytes, void *stream)
{
    const int rc = check_conv(B, T, I, K, dtype);
    if (rc != PLSTM_OK) return rc;
    const size_t e = dtype_size(dtype);
    if ((reverse != 0 && reverse != 1) || (act != 0 && act != 1) || !x || !w || !dy || !dx || !dw || !ws)
        return PLSTM_EINVAL;
    if (!conv_pitch(B, T, I, x_pitch)) return PLSTM_EINVAL;
    if (!aligned_to(x, e) || !aligned_to(w, e) || !aligned_to(bias, e) || !aligned_to(lengths, 4) ||
        !aligned_to(state, e) || !aligned_to(dy, e) || !aligned_to(dstate_out, 4) || !aligned_to(dx, e) ||
        !aligned_to(dw, 4) || !aligned_to(db, 4) || !aligned_to(dstate, 4) || !aligned_to(ws, 16))
        return PLSTM_EINVAL;
    if (ws_bytes < pyramid_causal_conv_workspace_size(B, T, I, K)) return PLSTM_EWORKSPACE;
    const ConvArgs a = conv_args(B, T, I, act, reverse, x_pitch, lengths);
    const int PB = conv_across(a), parts = conv_parts(a);
    const dim3 grid((unsigned)((a.pieces + PB - 1) / PB), (unsigned)parts);
    hipStream_t st = (hipStream_t)stream;
    timing_begin("conv_bwd", st);
    const bool stream_out = B * T * I * (int64_t)e >= kStreamBytes;
    const auto go = [&](auto t, auto fn) {
        typedef decltype(t) S;
        fn<<<grid, kConvThreads, 0, st>>>(a, PB, (const S *)x, (const S *)w, (const S *)bias, (const S *)state,
                                          (const S *)dy, (const float *)dstate_out, (S *)dx, (float *)dstate, (float *)ws);
    };
    const auto run = [&](auto k) {
        constexpr int KK = decltype(k)::value;
        if (dtype == PLSTM_F32)
            go(0.0f, stream_out ? k_conv_bwd<float, KK, true> : k_conv_bwd<float, KK, false>);
        else
            go((uint16_t)0, stream_out ? k_conv_bwd<uint16_t, KK, true> : k_conv_bwd<uint16_t, KK, false>);
        return in_launches<256>((I * (KK + 1) + 15) / 16, [&](unsigned first, unsigned n) {
            k_conv_weights<KK><<<n, 256, 0, st>>>(first, I, parts, (const float *)ws, (float *)dw, (float *)db);
        });
    };
    int launches = 0;
    switch (K) {
    case 1: launches = run(std::integral_constant<int, 1>()); break;
    case 2: launches = run(std::integral_constant<int, 2>()); break;
    case 3: launches = run(std::integral_constant<int, 3>()); break;
    case 4: launches = run(std::integral_constant<int, 4>()); break;
    case 5: launches = run(std::integral_constant<int, 5>()); break;
    case 6: launches = run(std::integral_constant<int, 6>()); break;
    case 7: launches = run(std::integral_constant<int, 7>()); break;
    default: launches = run(std::integral_constant<int, 8>()); break;
    }
    PLSTM_LAUNCH_CHECK();
    timing_end(1 + launches, st);
    return PLSTM_OK;
}

}  // extern "C"
