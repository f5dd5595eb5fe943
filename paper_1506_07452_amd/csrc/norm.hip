// Layer norm over the channels of each row, and its backward pass.
//   mean = sum_c x / C, var = sum_c (x - mean)^2 / C, rstd = 1 / sqrt(var + eps)
//   y = (x - mean) rstd gamma + beta
// Backward, with xh = (x - mean) rstd and a = dy gamma:
//   dx = rstd (a - sum_c a / C - xh sum_c (a xh) / C)
//   dgamma = sum_m dy xh, dbeta = sum_m dy
// Rows are read in the storage type or, in the backward, from an 8-bit
// checkpoint (code8.h); statistics and sums are fp32, but the mean's of fp32 rows (Mean).
#include "rows.h"
#include "timing.h"

namespace plstm {
namespace {

constexpr int kNormMaxC = 16384;
constexpr int kNormMaxParts = 512;  // workgroups, each with a part of the weights' gradients
constexpr int kNormFwdBlocks = 8192;

// A row is held in registers by G lanes, K pieces of 16 bytes (N elements)
// each: lane j has elements (j + G k) N .., k < K.  Short rows share a wave,
// long ones take four or sixteen waves.  U rows of a lane group are loaded before
// the first is used, so that short rows keep enough bytes in flight.
template <typename T, int G, int K>
struct Rows {
    static constexpr int N = Piece<T>::N;
    static constexpr int U = G > 64 ? 1 : K == 1 ? 4 : K == 2 ? 2 : 1;
};

// Sum of a value over the G lanes of a group, in every lane.  Groups of several
// waves exchange through `lds` (one slot a wave; not the slots of the exchange
// before it).
template <int G, typename S>
__device__ inline S group_sum(S v, S *lds)
{
    v = lanes_sum<(G < 64 ? G : 64)>(v);
    if (G <= 64) return v;
    constexpr int waves = G > 64 ? G / 64 : 1;
    const int wave = threadIdx.x / 64, first = wave / waves * waves;
    if ((threadIdx.x & 63) == 0) lds[wave] = v;
    __syncthreads();
    // 64-bit additions take long: in the lanes, not sixteen in a row
    if (sizeof(S) == 8) return lanes_sum<waves>(lds[first + (threadIdx.x & (waves - 1))]);
    S s = 0;
#pragma unroll
    for (int w = 0; w < waves; ++w) s += lds[first + w];
    return s;
}

// A row's mean from the sum of its elements: the fp32 mean, which the backward gets,
// and what that leaves of the true one.  fp32 rows are summed in 64 bits: in 32 the sum of C
// equal values of 24 bits rounds, and a row of one value, or one far above its spread, has the
// mean's error times rstd in every xh (0.2 for values of 1000 at C = 5000).  It costs
// nothing where rows share a wave and no codes are made, 3% (C = 4096) to 7% where several waves wait
// for the sum, and 7% in the forward that codes rows of 45.  bf16 values leave 16 bits of an
// fp32 sum free, so rows of one value add up exactly (C <= 2^14).
template <typename T> struct Mean;
template <> struct Mean<float> {
    typedef double S;
    double n, inv;
    explicit Mean(int C) : n((double)C), inv(1.0 / (double)C) {}
    __device__ float of(double sum, float &rest) const
    {
        const float mean = (float)(sum * inv);
        // 0 where the mean is exact, else right to some steps of itself
        rest = (float)fma(-(double)mean, n, sum) * (float)inv;
        return mean;
    }
};
template <> struct Mean<uint16_t> {
    typedef float S;
    float n, inv;
    explicit Mean(int C) : n((float)C), inv(1.0f / (float)C) {}
    __device__ float of(float sum, float &rest) const
    {
        const float m = sum * inv;
        rest = 0.0f;
        return fmaf(fmaf(-m, n, sum), inv, m);
    }
};

// Forward: two sums over a row that is read once, mean first, so that the variance is that of
// the differences.  Bound by bytes: 2764800 fp32 rows of 16 in 59 us (6.0 TB/s, part of y
// staying in the cache), 8192 bf16 rows of 4096 in 29 us (4.7 TB/s).
// CODE: also the 8-bit checkpoint of x.  1: its blocks of 64 elements are aligned
// lanes of a wave.  2: they are not, but the rows of a turn are whole blocks: those go
// through LDS, and lanes take pieces of blocks there.
enum { kNoCode = 0, kCodeInLanes = 1, kCodeInLds = 2 };
template <typename T, int G, int K, int CODE>
__global__ void __launch_bounds__(G > 256 ? G : 256)
k_norm_fwd(const T *__restrict__ x, const T *__restrict__ gamma, const T *__restrict__ beta,
           T *__restrict__ y, float2 *__restrict__ stats, int8_t *__restrict__ xq,
           uint16_t *__restrict__ xscale, long long M, int C, float eps, Mean<T> mean_of)
{
    constexpr int N = Rows<T, G, K>::N, U = Rows<T, G, K>::U;
    constexpr int threads = G > 256 ? G : 256, rows = threads / G;
    typedef typename Mean<T>::S Sum;
    __shared__ Sum lds_sum[2][threads / 64];
    __shared__ float lds_var[2][threads / 64];
    __shared__ __align__(16) T span[CODE == kCodeInLds ? rows * U * G * N : 8];
    const int j = threadIdx.x % G, group = threadIdx.x / G;
    const float inv = 1.0f / (float)C;
    float ga[K][N], be[K][N];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (j + G * k) * N;
        Piece<T>::unpack(load_piece(gamma + c, C - c), ga[k]);
        Piece<T>::unpack(load_piece(beta + c, C - c), be[k]);
    }
    int turn = 0;
    for (long long m0 = (long long)blockIdx.x * rows * U; m0 < M;
         m0 += (long long)gridDim.x * rows * U) {
        u32x4 raw[U][K];
#pragma unroll
        for (int t = 0; t < U; ++t) {
            const long long m = m0 + t * rows + group;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (j + G * k) * N;
                raw[t][k] = load_piece(x + m * C + c, m < M ? C - c : 0);
            }
        }
        loads_issued();
#pragma unroll
        for (int t = 0; t < U; ++t) {
            const long long m = m0 + t * rows + group;
            float v[K][N];
#pragma unroll
            for (int k = 0; k < K; ++k) Piece<T>::unpack(raw[t][k], v[k]);
            if (CODE == kCodeInLds) {
                const int c = j * N, at = (t * rows + group) * C + c;
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (c + i < C) Store<T>::store(span, at + i, v[0][i]);
            }
            if (CODE == kCodeInLanes) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const int c = (j + G * k) * N;
                    const long long at = m * C + c;
                    const uint16_t s =
                        code_scale(lanes_max<kCodeBlock / N>(top_bits<N>(v[k])));
                    const Coder cd(s);
                    uint32_t code[N];
                    code_piece<T>(cd, v[k], code);
                    if (m < M && c < C) {
                        store_codes<N>(xq + at, N, code, cd.keep);
                        if ((at & (kCodeBlock - 1)) == 0) xscale[at >> 6] = s;
                    }
                }
            }
            Sum sum = 0;
            if (sizeof(T) == 4) {
#pragma unroll
                for (int k = 0; k < K; ++k)
                    sum += ((Sum)v[k][0] + v[k][1]) + ((Sum)v[k][2] + v[k][3]);
            } else {
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int i = 0; i < N; ++i) sum += v[k][i];
            }
            float rest;
            const float mean = mean_of.of(group_sum<G>(sum, lds_sum[turn]), rest);
            float var = 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (j + G * k) * N;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    v[k][i] -= mean;
                    if (sizeof(T) == 4) v[k][i] -= rest;
                    if (c + i < C) var = fmaf(v[k][i], v[k][i], var);
                }
            }
            const float rstd = rsqrtf(fmaf(group_sum<G>(var, lds_var[turn]), inv, eps));
            turn ^= 1;
            if (m < M) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const int c = (j + G * k) * N;
                    float o[N];
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        o[i] = fmaf(v[k][i] * rstd, ga[k][i], be[k][i]);
                    store_piece(y + m * C + c, C - c, o);
                }
                if (stats && j == 0) stats[m] = make_float2(mean, rstd);
            }
        }
        if (CODE == kCodeInLds) {
            __syncthreads();
            const int size = rows * U * C;
#pragma unroll
            for (int t = 0; t < U; ++t) {
                const int e = (t * threads + (int)threadIdx.x) * N;
                if (e >= size) continue;        // all 64 elements of a block or none
                float v[N];
                Piece<T>::unpack(*(const u32x4 *)(span + e), v);
                const uint16_t s = code_scale(lanes_max<kCodeBlock / N>(top_bits<N>(v)));
                const Coder cd(s);
                uint32_t code[N];
                code_piece<T>(cd, v, code);
                const long long at = m0 * C + e, left = M * C - at;
                store_codes<N>(xq + at, left < N ? (int)left : N, code, cd.keep);
                if (e % kCodeBlock == 0 && left > 0) xscale[at >> 6] = s;
            }
            __syncthreads();
        }
    }
}

// A piece of x in raw bits and its values: from the storage type, or from codes.
template <typename T, typename X> struct RawX {
    u32x4 w;
    __device__ void load(const T *x, const uint16_t *, long long at, int have)
    {
        w = load_piece(x + at, have);
    }
    __device__ void unpack(long long, float *v) const { Piece<T>::unpack(w, v); }
};
template <typename T> struct RawX<T, int8_t> {
    RawCodes<Piece<T>::N> w;
    __device__ void load(const int8_t *x, const uint16_t *scale, long long at, int have)
    {
        w = load_coded<Piece<T>::N>(x, scale, at, have);
    }
    __device__ void unpack(long long at, float *v) const { unpack_coded(w, at, v); }
};

// Backward in one pass over x and dy: the row's two sums give dx, and the same values
// go into the columns' sums.  Bound by bytes: 2764800 fp32 rows of 16 in 116 us (4.6
// TB/s), 8192 bf16 rows of 4096 in 44 us (4.6 TB/s), 360000 fp32 rows of 45 from codes in 32
// us (4.6 TB/s).
// A workgroup walks every gridDim-th stretch of rows with its columns' sums of
// dy xh and dy in registers; at the end its lane groups' sums are added in
// order and written as its part [2][C] of `part` (dgamma and dbeta themselves
// where it is alone).
template <typename T, typename X, int G, int K>
__global__ void __launch_bounds__(G > 512 ? G : 512)
k_norm_bwd(const X *__restrict__ x, const uint16_t *__restrict__ xscale,
           const T *__restrict__ gamma, const float2 *__restrict__ stats,
           const T *__restrict__ dy, T *__restrict__ dx, float *__restrict__ dgamma,
           float *__restrict__ dbeta, float *__restrict__ part, long long M, int C)
{
    constexpr int N = Rows<T, G, K>::N, U = Rows<T, G, K>::U;
    constexpr int threads = G > 512 ? G : 512, rows = threads / G;
    constexpr int wide = G > 64 ? G : 64, parts = threads / wide;   // sums a column has in the end
    __shared__ float lds[2][2][threads / 64];
    __shared__ float cols[parts > 1 ? parts : 1][parts > 1 ? G * K * N : 1];
    const int j = threadIdx.x % G, group = threadIdx.x / G;
    const float inv = 1.0f / (float)C;
    float ga[K][N], sg[K][N], sb[K][N];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (j + G * k) * N;
        Piece<T>::unpack(load_piece(gamma + c, C - c), ga[k]);
#pragma unroll
        for (int i = 0; i < N; ++i) sg[k][i] = sb[k][i] = 0.0f;
    }
    int turn = 0;
    for (long long m0 = (long long)blockIdx.x * rows * U; m0 < M;
         m0 += (long long)gridDim.x * rows * U) {
        RawX<T, X> rx[U][K];
        u32x4 rd[U][K];
        float2 st[U];
#pragma unroll
        for (int t = 0; t < U; ++t) {
            const long long m = m0 + t * rows + group;
            st[t] = m < M ? stats[m] : make_float2(0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (j + G * k) * N, have = m < M ? C - c : 0;
                rx[t][k].load(x, xscale, m * C + c, have);
                rd[t][k] = load_piece(dy + m * C + c, have);
            }
        }
        loads_issued();
#pragma unroll
        for (int t = 0; t < U; ++t) {
            const long long m = m0 + t * rows + group;
            float v[K][N], d[K][N];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                rx[t][k].unpack(m * C + (j + G * k) * N, v[k]);
                Piece<T>::unpack(rd[t][k], d[k]);
            }
            float ta = 0.0f, tb = 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    // a channel that the row does not have has d = 0, but the mean times
                    // rstd may be infinite
                    const float xh = (j + G * k) * N + i < C ? (v[k][i] - st[t].x) * st[t].y : 0.0f;
                    const float a = d[k][i] * ga[k][i];
                    v[k][i] = xh;
                    ta += a;
                    tb = fmaf(a, xh, tb);
                    sg[k][i] = fmaf(d[k][i], xh, sg[k][i]);
                    sb[k][i] += d[k][i];
                }
            if (!dx) continue;
            ta = group_sum<G>(ta, lds[turn][0]) * inv;
            tb = group_sum<G>(tb, lds[turn][1]) * inv;
            turn ^= 1;
            if (m < M) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const int c = (j + G * k) * N;
                    float o[N];
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        o[i] = st[t].y * (fmaf(d[k][i], ga[k][i], -ta) - v[k][i] * tb);
                    store_piece(dx + m * C + c, C - c, o);
                }
            }
        }
    }
    float *og = gridDim.x == 1 ? dgamma : part + (long long)blockIdx.x * 2 * C;
    float *ob = gridDim.x == 1 ? dbeta : og + C;
    // lanes of a wave with the same columns, then the waves (or wider groups)
    for (int pass = 0; pass < 2; ++pass) {
        float (*s)[N] = pass ? sb : sg;
        float *out = pass ? ob : og;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int w = G; w < 64; w *= 2) s[k][i] += __shfl_xor(s[k][i], w);
        if (parts == 1) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (j + G * k) * N;
#pragma unroll
                for (int i = 0; i < N; i += 4) store_piece(out + c + i, C - c - i, s[k] + i);
            }
            continue;
        }
        if (pass) __syncthreads();
        if (G >= 64 || (threadIdx.x & 63) < G) {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    cols[threadIdx.x / wide][(j + G * k) * N + i] = s[k][i];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += threads) {
            float v = 0.0f;
#pragma unroll
            for (int p = 0; p < parts; ++p) v += cols[p][c];
            out[c] = v;
        }
    }
}

// dgamma and dbeta from `count` parts: 16 columns a workgroup, 64 lanes each with every
// 64th part; then the lanes of a wave, then the waves, in order.  A launch's latency and
// one round of loads: 4 to 5 us.
__global__ void __launch_bounds__(1024)
k_norm_dw_sum(const float *__restrict__ part, int count, float *__restrict__ dgamma,
              float *__restrict__ dbeta, int C)
{
    __shared__ float lds[16][16];
    const int col = threadIdx.x & 15, w = threadIdx.x / 64;
    const int c = blockIdx.x * 16 + col;
    float s = 0.0f;
    if (c < 2 * C) {
#pragma unroll
        for (int i = 0; i < kNormMaxParts / 64; ++i) {
            const int k = (int)(threadIdx.x / 16) + 64 * i;
            s += k < count ? part[(long long)k * 2 * C + c] : 0.0f;
        }
    }
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if ((threadIdx.x & 63) < 16) lds[w][col] = s;
    __syncthreads();
    if (threadIdx.x >= 16 || c >= 2 * C) return;
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += lds[k][col];
    (c < C ? dgamma[c] : dbeta[c - C]) = s;
}

// Workgroups of the backward: what rows there are for, at most kNormMaxParts
// (two for each CU), and fewer for long rows, whose parts cost as much as rows do.
long long norm_parts(long long M, int C, int rows)
{
    const long long need = (M + rows - 1) / rows, most = C > 2048 ? kNormMaxParts / 2 : kNormMaxParts;
    return need < most ? need : most;
}

// fn(G, K) as compile-time constants for rows of C elements of type T.
template <int V> struct Const { static constexpr int value = V; };
template <typename T, typename F>
int with_rows(int C, F fn)
{
    constexpr int N = Piece<T>::N;
    const int pieces = (C + N - 1) / N;
    if (pieces <= 1) return fn(Const<1>(), Const<1>());
    if (pieces <= 2) return fn(Const<2>(), Const<1>());
    if (pieces <= 4) return fn(Const<4>(), Const<1>());
    if (pieces <= 8) return fn(Const<8>(), Const<1>());
    if (pieces <= 16) return fn(Const<16>(), Const<1>());
    if (pieces <= 32) return fn(Const<32>(), Const<1>());
    if (pieces <= 64) return fn(Const<64>(), Const<1>());
    if (pieces <= 128) return fn(Const<64>(), Const<2>());
    if (pieces <= 256) return fn(Const<256>(), Const<1>());
    if (pieces <= 512) return fn(Const<256>(), Const<2>());
    if (pieces <= 1024) return fn(Const<1024>(), Const<1>());
    if (pieces <= 2048) return fn(Const<1024>(), Const<2>());
    if constexpr (N == 4) return fn(Const<1024>(), Const<4>());
    return PLSTM_EUNSUPPORTED;
}

// How the forward codes rows of C elements, G lanes each with U rows in a turn:
// in its lanes where blocks of 64 elements lie in whole rows or whole rows of pieces in a
// block; through LDS where a turn's rows are whole blocks (fp32, 360000 rows of 45: 34 us, 41
// with the pack kernel after it); not at all otherwise.
template <typename T, int G, int K> constexpr int code_rows() { return (G > 256 ? G : 256) / G * Rows<T, G, K>::U; }
template <typename T, int G, int K> int code_mode(int C)
{
    if (C % kCodeBlock == 0 || (kCodeBlock % C == 0 && C >= Piece<T>::N)) return kCodeInLanes;
    if (G <= 64 && K == 1 && code_rows<T, G, K>() * C % kCodeBlock == 0) return kCodeInLds;
    return kNoCode;
}

template <typename T>
int norm_forward(long long M, int C, float eps, const T *x, const T *gamma, const T *beta, T *y,
                 float2 *stats, int8_t *xq, uint16_t *xscale, int *launches, hipStream_t st)
{
    return with_rows<T>(C, [&](auto g, auto k) -> int {
        constexpr int G = decltype(g)::value, K = decltype(k)::value;
        constexpr int threads = G > 256 ? G : 256, rows = code_rows<T, G, K>();
        const long long need = (M + rows - 1) / rows;
        const unsigned grid = (unsigned)(need < kNormFwdBlocks ? need : kNormFwdBlocks);
        const Mean<T> mean_of(C);
        const int mode = xq ? code_mode<T, G, K>(C) : kNoCode;
        *launches = 1;
        if (mode == kCodeInLanes) {
            k_norm_fwd<T, G, K, kCodeInLanes><<<grid, threads, 0, st>>>(
                x, gamma, beta, y, stats, xq, xscale, M, C, eps, mean_of);
        } else if (mode == kCodeInLds) {
            if constexpr (G <= 64 && K == 1)
                k_norm_fwd<T, G, K, kCodeInLds><<<grid, threads, 0, st>>>(
                    x, gamma, beta, y, stats, xq, xscale, M, C, eps, mean_of);
        } else {
            k_norm_fwd<T, G, K, kNoCode><<<grid, threads, 0, st>>>(x, gamma, beta, y, stats,
                                                                  nullptr, nullptr, M, C, eps,
                                                                  mean_of);
            if (xq) {
                PLSTM_LAUNCH_CHECK();
                *launches = 2;
                return checkpoint8_pack(M * C, sizeof(T) == 4 ? PLSTM_F32 : PLSTM_BF16, x, xq,
                                        xscale, st);
            }
        }
        PLSTM_LAUNCH_CHECK();
        return PLSTM_OK;
    });
}

int check_rows(int64_t M, int32_t C, int32_t dtype)
{
    if (M < 1 || C < 1) return PLSTM_EINVAL;
    if (dtype != PLSTM_F32 && dtype != PLSTM_BF16) return PLSTM_EINVAL;
    if (C > kNormMaxC || M > (1LL << 32) || M > (1LL << 38) / C) return PLSTM_EUNSUPPORTED;
    return PLSTM_OK;
}

// `launches` counts the kernels.
template <typename T, typename X>
int norm_backward(long long M, int C, const X *x, const uint16_t *xscale, const T *gamma,
                  const float2 *stats, const T *dy, T *dx, float *dgamma, float *dbeta,
                  float *part, int *launches, hipStream_t st)
{
    return with_rows<T>(C, [&](auto g, auto k) -> int {
        constexpr int G = decltype(g)::value, K = decltype(k)::value;
        constexpr int threads = G > 512 ? G : 512, rows = threads / G * Rows<T, G, K>::U;
        const int count = (int)norm_parts(M, C, rows);
        k_norm_bwd<T, X, G, K><<<(unsigned)count, threads, 0, st>>>(
            x, xscale, gamma, stats, dy, dx, dgamma, dbeta, part, M, C);
        PLSTM_LAUNCH_CHECK();
        *launches = 1;
        if (count > 1) {
            k_norm_dw_sum<<<(unsigned)((2 * C + 15) / 16), 1024, 0, st>>>(part, count, dgamma,
                                                                         dbeta, C);
            PLSTM_LAUNCH_CHECK();
            *launches = 2;
        }
        return PLSTM_OK;
    });
}

template <typename T>
int norm_backward_from(long long M, int C, const void *x, const void *xscale, const void *gamma,
                       const void *stats, const void *dy, void *dx, void *dgamma, void *dbeta,
                       void *ws, int *launches, hipStream_t st)
{
    if (xscale)
        return norm_backward<T, int8_t>(M, C, (const int8_t *)x, (const uint16_t *)xscale,
                                        (const T *)gamma, (const float2 *)stats, (const T *)dy,
                                        (T *)dx, (float *)dgamma, (float *)dbeta, (float *)ws,
                                        launches, st);
    return norm_backward<T, T>(M, C, (const T *)x, nullptr, (const T *)gamma,
                               (const float2 *)stats, (const T *)dy, (T *)dx, (float *)dgamma,
                               (float *)dbeta, (float *)ws, launches, st);
}

}  // namespace
}  // namespace plstm

using namespace plstm;

extern "C" {

size_t pyramid_layer_norm_workspace_size(int64_t M, int32_t C)
{
    if (check_rows(M, C, PLSTM_F32) != PLSTM_OK) return 0;
    return align_up((size_t)norm_parts(M, C, 1) * 2 * C * sizeof(float), 256);
}

int pyramid_layer_norm_forward(int64_t M, int32_t C, int32_t dtype, float eps, const void *x,
                               const void *gamma, const void *beta, void *y, void *stats,
                               void *xq, void *xscale, void *stream)
{
    int rc = check_rows(M, C, dtype);
    if (rc != PLSTM_OK) return rc;
    if (!(eps > 0.0f) || !x || !gamma || !beta || !y || !xq != !xscale) return PLSTM_EINVAL;
    const size_t e = dtype_size(dtype);
    if (!aligned_to(x, e) || !aligned_to(gamma, e) || !aligned_to(beta, e) || !aligned_to(y, e) ||
        !aligned_to(stats, 8) || !aligned_to(xq, 16) || !aligned_to(xscale, 16))
        return PLSTM_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    timing_begin("norm_fwd", st);
    int launches = 0;
    rc = dtype == PLSTM_F32
             ? norm_forward(M, C, eps, (const float *)x, (const float *)gamma,
                            (const float *)beta, (float *)y, (float2 *)stats, (int8_t *)xq,
                            (uint16_t *)xscale, &launches, st)
             : norm_forward(M, C, eps, (const uint16_t *)x, (const uint16_t *)gamma,
                            (const uint16_t *)beta, (uint16_t *)y, (float2 *)stats, (int8_t *)xq,
                            (uint16_t *)xscale, &launches, st);
    if (rc == PLSTM_OK) timing_end(launches, st);
    return rc;
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
    int launches = 0;
    rc = dtype == PLSTM_F32
             ? norm_backward_from<float>(M, C, x, xscale, gamma, stats, dy, dx, dgamma, dbeta, ws,
                                         &launches, st)
             : norm_backward_from<uint16_t>(M, C, x, xscale, gamma, stats, dy, dx, dgamma, dbeta,
                                            ws, &launches, st);
    if (rc == PLSTM_OK) timing_end(launches, st);
    return rc;
}

}  // extern "C"
