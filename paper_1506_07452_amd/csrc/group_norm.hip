// Group norm over channels-last volumes [N][V][C], an activation behind it, and the
// backward pass.  A group is Cg = C / G consecutive channels of a volume:
//   mean, var over its V Cg values, rstd = 1 / sqrt(var + eps), xh = (x - mean) rstd
//   v = gamma xh + beta,  y = act(v)
// Backward, with dv = dy act'(v) (v computed again) and a = gamma dv:
//   dx = rstd (a - mean_g(a) - xh mean_g(a xh)),  dgamma = sum dv xh,  dbeta = sum dv
// A thread has one 16-byte piece of a row's channels and walks down the rows, so channels
// keep their sums in registers.  Volumes that fit the registers of a workgroup are read
// once; others are read twice, the sums of slabs of rows going through memory between, the second time from the end, whose rows the
// caches still have.  Everything is bound by bytes: 1 x 2764800 x 16 fp32 33 + 5 + 56 us forward (531 MB with x
// twice, 5.6 TB/s), 65 + 6 + 84 backward (885 MB, 5.7 TB/s); 8 x 262144 x 64 bf16 49 + 5 + 91 and 102 + 5 + 137.
// A held volume: 64 x 64 x 32 bf16 forward and backward 30 us, by slabs 34; 300 x 256 x 32 31, 41.
// Sums of x and x^2 are 64-bit: squares of fp32 are exact, so the variance of values at
// 1000 times their spread still has 10 digits, and the order of the sums does not show.
#include "sequence.h"
#include "timing.h"

namespace plstm {
namespace {

constexpr int kGnMaxC = 16384;
constexpr int kGnThreads = 256;
constexpr int kGnSmall = 1024;          // threads of a workgroup that holds a volume
constexpr int kGnHeldC = 2048;         // channels that the sums of such a workgroup have LDS for
// Workgroups that a call aims at: 1 x 2764800 x 16 fp32 245 us with 768, 249 with 1024, 253 with 2048, 324 with 256;
// 8 x 262144 x 64 bf16 386, 389, 414, 622 (512: 243 and 393).
constexpr int kGnBlocks = 768;

struct GnArgs {
    long long N, V;
    int C, G, Cg, act;
    float eps;
    int pieces, across, rows;           // of a row; threads across and down a workgroup
    long long slab;                     // rows of a slab
    int slabs;                          // of a volume
};

// A thread's piece of channels.
template <typename T> struct GnColumn {
    static constexpr int N = Piece<T>::N;
    int row, c, have;                   // first row; first channel; channels (0: an idle thread)
    __device__ GnColumn(const GnArgs &a, int block)
    {
        const int piece = block * a.across + (int)threadIdx.x % a.across;
        row = (int)threadIdx.x / a.across;
        c = piece * N;
        have = row >= a.rows || piece >= a.pieces ? 0 : min(a.C - c, N);
    }
};

// Sums over the rows of a workgroup: every thread has a value of each of its N
// channels; f(channel of the workgroup, sum) runs in some thread for every channel, in a
// fixed order of additions.  lds: sum_rows_lds() values.
template <int NT, int N, typename S, typename F>
__device__ inline void sum_rows(const GnArgs &a, S *lds, const S *v, F f)
{
    S *second = lds + NT * N;
    const int outs = a.across * N;
    int parts = NT / outs;
    parts = parts < 1 ? 1 : parts > a.rows ? a.rows : parts;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; ++j) lds[threadIdx.x * N + j] = v[j];
    __syncthreads();
    for (int o = threadIdx.x; o < outs * parts; o += NT) {
        const int part = o / outs, out = o - part * outs;
        S s = 0;
        for (int r = part; r < a.rows; r += parts) s += lds[r * outs + out];
        second[o] = s;
    }
    __syncthreads();
    for (int out = threadIdx.x; out < outs; out += NT) {
        S s = second[out];
        for (int p = 1; p < parts; ++p) s += second[p * outs + out];
        f(out, s);
    }
}
template <int NT, int N> __host__ __device__ constexpr int sum_rows_lds(int across = NT)
{
    return NT * N + (across * N > NT ? across * N : NT);
}

// What a group's sums make of it; mean = the fp32 mean + rest.
struct GroupStats {
    float mean, rest, rstd;
    __device__ GroupStats() {}
    __device__ GroupStats(double s1, double s2, double n, float eps)
    {
        const double m = s1 / n, var = s2 / n - m * m;
        mean = (float)m;
        rest = (float)(m - (double)mean);
        // not a maximum: a NaN stays one
        rstd = (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + (double)eps));
    }
};

// part [n slabs + slab][C][2]: sums of x and x^2 of a slab's rows.
template <typename T>
__global__ void __launch_bounds__(kGnThreads)
k_gn_sums(GnArgs a, const T *x, double *part)
{
    constexpr int N = Piece<T>::N, U = 4;
    __shared__ double lds[sum_rows_lds<kGnThreads, N>()];
    const long long n = blockIdx.x / (unsigned)a.slabs, slab = blockIdx.x - n * a.slabs;
    const GnColumn<T> col(a, blockIdx.y);
    const long long end = min(a.V, (slab + 1) * a.slab);
    double s1[N], s2[N];
#pragma unroll
    for (int j = 0; j < N; ++j) s1[j] = s2[j] = 0.0;
    if (col.have) {
        const T *p = x + n * a.V * a.C + col.c;
        for (long long r = slab * a.slab + col.row; r < end; r += U * a.rows) {
            u32x4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long long q = r + u * a.rows;
                raw[u] = load_piece<T>(p + q * a.C, q < end ? col.have : 0);
            }
            loads_issued();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float v[N];
                Piece<T>::unpack(raw[u], v);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const double d = (double)v[j];
                    s1[j] += d;
                    s2[j] = fma(d, d, s2[j]);
                }
            }
        }
    }
    const int first = blockIdx.y * a.across * N;
    double *to = part + (long long)blockIdx.x * a.C * 2;
    sum_rows<kGnThreads, N>(a, lds, s1, [&](int o, double s) { if (first + o < a.C) to[(first + o) * 2] = s; });
    sum_rows<kGnThreads, N>(a, lds, s2, [&](int o, double s) { if (first + o < a.C) to[(first + o) * 2 + 1] = s; });
}

// Sums of two values over a workgroup of 1024, in a fixed order.
__device__ inline void sum1024(double &x, double &y, double (*lds)[2])
{
    x = lanes_sum<64>(x);
    y = lanes_sum<64>(y);
    if ((threadIdx.x & 63) == 0) {
        lds[threadIdx.x / 64][0] = x;
        lds[threadIdx.x / 64][1] = y;
    }
    __syncthreads();
    x = lanes_sum<16>(lds[threadIdx.x & 15][0]);
    y = lanes_sum<16>(lds[threadIdx.x & 15][1]);
}

// A thread's share of the parts of group g of volume n: f(channel, the part's two sums), four at a time so that their loads
// are under way together.
template <typename F>
__device__ inline void over_parts(const GnArgs &a, const double *part, long long n, int g, F f)
{
    const int all = a.slabs * a.Cg;
    const double2 *p = (const double2 *)part + n * a.slabs * a.C + g * a.Cg;
    for (int k = threadIdx.x; k < all; k += 4096) {
        double2 v[4];
        int c[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int e = min(k + 1024 * u, all - 1), slab = e / a.Cg;
            c[u] = e - slab * a.Cg;
            v[u] = p[(long long)slab * a.C + c[u]];
        }
        loads_issued();
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (k + 1024 * u < all) f(g * a.Cg + c[u], v[u]);
    }
}

// A group a workgroup, from group `first` of all on.
__global__ void __launch_bounds__(1024)
k_gn_stats(GnArgs a, unsigned first, const double *part, GroupStats *st, float *stats)
{
    __shared__ double lds[16][2];
    const unsigned at = first + blockIdx.x;
    const long long n = at / (unsigned)a.G;
    const int g = (int)(at - n * a.G);
    double s1 = 0.0, s2 = 0.0;
    over_parts(a, part, n, g, [&](int, double2 v) {
        s1 += v.x;
        s2 += v.y;
    });
    sum1024(s1, s2, lds);
    if (threadIdx.x) return;
    const GroupStats r(s1, s2, (double)a.V * a.Cg, a.eps);
    st[at] = r;
    if (stats) {
        stats[2 * (long long)at] = r.mean;
        stats[2 * (long long)at + 1] = r.rstd;
    }
}

// v = (x - mean) scale + shift for a thread's channels.
template <int N> struct GnAffine {
    float mean[N], scale[N], shift[N];
    template <typename T, typename F>
    __device__ void fill(const GnArgs &a, int c, int have, const T *gamma, const T *beta, F stats_of)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const bool has = j < have;
            const GroupStats s = stats_of(has ? (c + j) / a.Cg : 0);
            mean[j] = s.mean;
            scale[j] = has ? s.rstd * Store<T>::load(gamma, c + j) : 0.0f;
            shift[j] = has ? fmaf(-s.rest, scale[j], Store<T>::load(beta, c + j)) : 0.0f;
        }
    }
    __device__ void apply(const float *x, int act, float *y) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float v = fmaf(x[j] - mean[j], scale[j], shift[j]);
            y[j] = act ? silu_of(v) : v;
        }
    }
};

// The statistics of a volume's groups, made by a workgroup of 256 for itself from few parts (C <= 256 channels).
__device__ inline void few_stats(const GnArgs &a, const double *part, long long n, double2 *sums, GroupStats *st)
{
    const int subs = 256 / a.C, sub = (int)threadIdx.x / a.C, c = (int)threadIdx.x - sub * a.C;
    double2 s = make_double2(0.0, 0.0);
    if (sub < subs) {
        const double2 *p = (const double2 *)part + n * a.slabs * a.C + c;
#pragma unroll 4
        for (int k = sub; k < a.slabs; k += subs) {
            const double2 v = p[k * a.C];
            s.x += v.x;
            s.y += v.y;
        }
        sums[threadIdx.x] = s;
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, all = subs * a.Cg;
    for (int g = threadIdx.x / 64; g < a.G; g += 4) {
        double x = 0.0, y = 0.0;
        for (int e = lane; e < all; e += 64) {
            const double2 v = sums[e / a.Cg * a.C + g * a.Cg + e % a.Cg];
            x += v.x;
            y += v.y;
        }
        x = lanes_sum<64>(x);
        y = lanes_sum<64>(y);
        if (lane == 0) st[g] = GroupStats(x, y, (double)a.V * a.Cg, a.eps);
    }
    __syncthreads();
}

// FEW: from the parts themselves, a launch less (then stats, where wanted, is written here).
template <typename T, bool STREAM, bool FEW>
__global__ void __launch_bounds__(kGnThreads)
k_gn_apply(GnArgs a, const T *x, const T *gamma, const T *beta, const GroupStats *st, T *y, const double *part, float *stats)
{
    constexpr int N = Piece<T>::N, U = 4;
    __shared__ double2 sums[FEW ? 256 : 1];
    __shared__ GroupStats few[FEW ? 256 : 1];
    // from the end, whose rows were read last
    const long long id = gridDim.x - 1 - blockIdx.x, n = id / a.slabs, slab = id - n * a.slabs;
    const GnColumn<T> col(a, blockIdx.y);
    if constexpr (FEW) {
        few_stats(a, part, n, sums, few);
        if (stats && slab == 0)
            for (int g = threadIdx.x; g < a.G; g += kGnThreads) {
                stats[2 * (n * a.G + g)] = few[g].mean;
                stats[2 * (n * a.G + g) + 1] = few[g].rstd;
            }
    }
    if (!col.have) return;
    GnAffine<N> f;
    f.fill(a, col.c, col.have, gamma, beta, [&](int g) {
        if constexpr (FEW) return few[g];
        else return st[n * a.G + g];
    });
    const long long end = min(a.V, (slab + 1) * a.slab), at = n * a.V * a.C + col.c;
    for (long long r = slab * a.slab + col.row; r < end; r += U * a.rows) {
        u32x4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long q = r + u * a.rows;
            raw[u] = load_last<STREAM>(x + at + q * a.C, q < end ? col.have : 0);
        }
        loads_issued();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long q = r + u * a.rows;
            if (q >= end) break;
            float v[N];
            Piece<T>::unpack(raw[u], v);
            f.apply(v, a.act, v);
            store_out<STREAM>(y + at + q * a.C, col.have, v);
        }
    }
}

// A volume in the registers of a workgroup, K rows a thread; from volume `first` on.
template <typename T, int NT, int K>
__global__ void __launch_bounds__(NT)
k_gn_small_fwd(GnArgs a, unsigned first, const T *x, const T *gamma, const T *beta, T *y, float *stats)
{
    constexpr int N = Piece<T>::N;
    extern __shared__ double dyn[];
    double *lds = dyn, *ch = dyn + sum_rows_lds<NT, N>(a.across);       // ch [C][2]
    GroupStats *st = (GroupStats *)(ch + 2 * a.C);
    const long long n = first + blockIdx.x;
    const GnColumn<T> col(a, 0);
    const long long at = n * a.V * a.C + col.c;
    u32x4 raw[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const long long q = col.row + (long long)k * a.rows;
        raw[k] = load_piece<T>(x + at + q * a.C, q < a.V ? col.have : 0);
    }
    loads_issued();
    double s1[N], s2[N];
#pragma unroll
    for (int j = 0; j < N; ++j) s1[j] = s2[j] = 0.0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float v[N];
        Piece<T>::unpack(raw[k], v);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const double d = (double)v[j];
            s1[j] += d;
            s2[j] = fma(d, d, s2[j]);
        }
    }
    sum_rows<NT, N>(a, lds, s1, [&](int o, double s) { if (o < a.C) ch[2 * o] = s; });
    sum_rows<NT, N>(a, lds, s2, [&](int o, double s) { if (o < a.C) ch[2 * o + 1] = s; });
    __syncthreads();
    const int lane = threadIdx.x & 63;
    for (int g = threadIdx.x / 64; g < a.G; g += NT / 64) {
        double t1 = 0.0, t2 = 0.0;
        for (int c = lane; c < a.Cg; c += 64) {
            t1 += ch[2 * (g * a.Cg + c)];
            t2 += ch[2 * (g * a.Cg + c) + 1];
        }
        t1 = lanes_sum<64>(t1);
        t2 = lanes_sum<64>(t2);
        if (lane == 0) {
            const GroupStats r(t1, t2, (double)a.V * a.Cg, a.eps);
            st[g] = r;
            if (stats) {
                stats[2 * (n * a.G + g)] = r.mean;
                stats[2 * (n * a.G + g) + 1] = r.rstd;
            }
        }
    }
    __syncthreads();
    if (!col.have) return;
    GnAffine<N> f;
    f.fill(a, col.c, col.have, gamma, beta, [&](int g) { return st[g]; });
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const long long q = col.row + (long long)k * a.rows;
        if (q >= a.V) break;
        float v[N];
        Piece<T>::unpack(raw[k], v);
        f.apply(v, a.act, v);
        store_piece<T>(y + at + q * a.C, col.have, v);
    }
}

// xh and dv of a thread's channels from x and dy.
template <int N> struct GnBack {
    float mean[N], rstd[N], gamma[N], beta[N];
    template <typename T>
    __device__ void fill(const GnArgs &a, long long n, int c, int have, const T *gp, const T *bp, const float *stats)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const bool has = j < have;
            const float *s = stats + 2 * (n * a.G + (has ? (c + j) / a.Cg : 0));
            mean[j] = s[0];
            rstd[j] = has ? s[1] : 0.0f;
            gamma[j] = has ? Store<T>::load(gp, c + j) : 0.0f;
            beta[j] = has ? Store<T>::load(bp, c + j) : 0.0f;
        }
    }
    __device__ void values(int j, int act, float x, float dy, float &xh, float &dv) const
    {
        xh = (x - mean[j]) * rstd[j];
        float silu;
        dv = act ? dy * silu_slope(fmaf(gamma[j], xh, beta[j]), silu) : dy;
    }
};

// part [n slabs + slab][C][2]: sums of dv xh and dv of a slab's rows.
template <typename T>
__global__ void __launch_bounds__(kGnThreads)
k_gn_bwd_sums(GnArgs a, const T *x, const T *gamma, const T *beta, const float *stats, const T *dy, double *part)
{
    constexpr int N = Piece<T>::N, U = 2;
    __shared__ double lds[sum_rows_lds<kGnThreads, N>()];
    const long long n = blockIdx.x / (unsigned)a.slabs, slab = blockIdx.x - n * a.slabs;
    const GnColumn<T> col(a, blockIdx.y);
    const long long end = min(a.V, (slab + 1) * a.slab), at = n * a.V * a.C + col.c;
    double ps[N], qs[N];
#pragma unroll
    for (int j = 0; j < N; ++j) ps[j] = qs[j] = 0.0;
    if (col.have) {
        GnBack<N> f;
        f.fill(a, n, col.c, col.have, gamma, beta, stats);
        for (long long r = slab * a.slab + col.row; r < end; r += U * a.rows) {
            u32x4 rx[U], rd[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long long s = r + u * a.rows;
                rx[u] = load_piece<T>(x + at + s * a.C, s < end ? col.have : 0);
                rd[u] = load_piece<T>(dy + at + s * a.C, s < end ? col.have : 0);
            }
            loads_issued();
            float p[N], q[N];           // of a turn in 32 bits, of turns in 64
#pragma unroll
            for (int j = 0; j < N; ++j) p[j] = q[j] = 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r + u * a.rows >= end) break;
                float v[N], d[N];
                Piece<T>::unpack(rx[u], v);
                Piece<T>::unpack(rd[u], d);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    float xh, dv;
                    f.values(j, a.act, v[j], d[j], xh, dv);
                    p[j] = fmaf(dv, xh, p[j]);
                    q[j] += dv;
                }
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                ps[j] += (double)p[j];
                qs[j] += (double)q[j];
            }
        }
    }
    const int first = blockIdx.y * a.across * N;
    double *to = part + (long long)blockIdx.x * a.C * 2;
    sum_rows<kGnThreads, N>(a, lds, ps, [&](int o, double t) { if (first + o < a.C) to[(first + o) * 2] = t; });
    sum_rows<kGnThreads, N>(a, lds, qs, [&](int o, double t) { if (first + o < a.C) to[(first + o) * 2 + 1] = t; });
}

// The first `groups` workgroups: a group's mean of a and of a xh, from group `first` of all on; the others: dgamma
// and dbeta of 16 channels, 64 lanes each over the parts of all volumes.
template <typename T>
__global__ void __launch_bounds__(1024)
k_gn_bwd_finish(GnArgs a, unsigned first, int groups, const T *gamma, const double *part, float2 *means, float *dgamma, float *dbeta)
{
    __shared__ double2 lds[64][16];
    if ((int)blockIdx.x < groups) {
        const unsigned at = first + blockIdx.x;
        const long long n = at / (unsigned)a.G;
        const int g = (int)(at - n * a.G);
        double s1 = 0.0, s2 = 0.0;
        over_parts(a, part, n, g, [&](int c, double2 v) {
            const double w = (double)Store<T>::load(gamma, c);
            s1 = fma(w, v.y, s1);
            s2 = fma(w, v.x, s2);
        });
        sum1024(s1, s2, (double(*)[2])lds);
        const double inv = 1.0 / ((double)a.V * a.Cg);
        if (threadIdx.x == 0) means[at] = make_float2((float)(s1 * inv), (float)(s2 * inv));
        return;
    }
    const int o = threadIdx.x % 16, lane = threadIdx.x / 16, c = ((int)blockIdx.x - groups) * 16 + o;
    double2 s = make_double2(0.0, 0.0);
    if (c < a.C) {
        const double2 *p = (const double2 *)part + c;
#pragma unroll 8
        for (long long k = lane; k < a.N * a.slabs; k += 64) {
            const double2 v = p[k * a.C];
            s.x += v.x;
            s.y += v.y;
        }
    }
    lds[lane][o] = s;
    __syncthreads();
    if (lane || c >= a.C) return;
    for (int l = 1; l < 64; ++l) {
        s.x += lds[l][o].x;
        s.y += lds[l][o].y;
    }
    dgamma[c] = (float)s.x;
    dbeta[c] = (float)s.y;
}

template <typename T, bool STREAM>
__global__ void __launch_bounds__(kGnThreads)
k_gn_bwd_apply(GnArgs a, const T *x, const T *gamma, const T *beta, const float *stats, const T *dy,
               const float2 *means, T *dx)
{
    constexpr int N = Piece<T>::N, U = 2;
    // from the end, whose rows were read last
    const long long id = gridDim.x - 1 - blockIdx.x, n = id / a.slabs, slab = id - n * a.slabs;
    const GnColumn<T> col(a, blockIdx.y);
    if (!col.have) return;
    GnBack<N> f;
    f.fill(a, n, col.c, col.have, gamma, beta, stats);
    float m1[N], m2[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float2 m = means[n * a.G + (j < col.have ? (col.c + j) / a.Cg : 0)];
        m1[j] = m.x;
        m2[j] = m.y;
    }
    const long long end = min(a.V, (slab + 1) * a.slab), at = n * a.V * a.C + col.c;
    for (long long r = slab * a.slab + col.row; r < end; r += U * a.rows) {
        u32x4 rx[U], rd[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long s = r + u * a.rows;
            rx[u] = load_last<STREAM>(x + at + s * a.C, s < end ? col.have : 0);
            rd[u] = load_last<STREAM>(dy + at + s * a.C, s < end ? col.have : 0);
        }
        loads_issued();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long s = r + u * a.rows;
            if (s >= end) break;
            float v[N], d[N];
            Piece<T>::unpack(rx[u], v);
            Piece<T>::unpack(rd[u], d);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float xh, dv;
                f.values(j, a.act, v[j], d[j], xh, dv);
                d[j] = f.rstd[j] * (fmaf(f.gamma[j], dv, -m1[j]) - xh * m2[j]);
            }
            store_out<STREAM>(dx + at + s * a.C, col.have, d);
        }
    }
}

// A volume in the registers of a workgroup, from volume `first` on; part [n][C][2] as of one slab.
template <typename T, int NT, int K>
__global__ void __launch_bounds__(NT)
k_gn_small_bwd(GnArgs a, unsigned first, const T *x, const T *gamma, const T *beta, const float *stats, const T *dy, T *dx,
               double *part, float *dgamma, float *dbeta)
{
    constexpr int N = Piece<T>::N;
    extern __shared__ double dyn[];
    float *lds = (float *)dyn, *ch = lds + sum_rows_lds<NT, N>(a.across);       // ch [C][2]
    float2 *means = (float2 *)(ch + 2 * a.C);
    const long long n = first + blockIdx.x;
    const GnColumn<T> col(a, 0);
    const long long at = n * a.V * a.C + col.c;
    u32x4 rx[K], rd[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const long long q = col.row + (long long)k * a.rows;
        rx[k] = load_piece<T>(x + at + q * a.C, q < a.V ? col.have : 0);
        rd[k] = load_piece<T>(dy + at + q * a.C, q < a.V ? col.have : 0);
    }
    loads_issued();
    GnBack<N> f;
    f.fill(a, n, col.c, col.have, gamma, beta, stats);
    float p[N], s[N];
#pragma unroll
    for (int j = 0; j < N; ++j) p[j] = s[j] = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (col.row + (long long)k * a.rows >= a.V) break;
        float v[N], d[N];
        Piece<T>::unpack(rx[k], v);
        Piece<T>::unpack(rd[k], d);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float xh, dv;
            f.values(j, a.act, v[j], d[j], xh, dv);
            p[j] = fmaf(dv, xh, p[j]);
            s[j] += dv;
        }
    }
    sum_rows<NT, N>(a, lds, p, [&](int o, float t) { if (o < a.C) ch[2 * o] = t; });
    sum_rows<NT, N>(a, lds, s, [&](int o, float t) { if (o < a.C) ch[2 * o + 1] = t; });
    __syncthreads();
    for (int c = threadIdx.x; c < a.C; c += NT) {
        if (a.N == 1) {
            dgamma[c] = ch[2 * c];
            dbeta[c] = ch[2 * c + 1];
        } else {
            part[(n * a.C + c) * 2] = (double)ch[2 * c];
            part[(n * a.C + c) * 2 + 1] = (double)ch[2 * c + 1];
        }
    }
    const int lane = threadIdx.x & 63;
    const double inv = 1.0 / ((double)a.V * a.Cg);
    for (int g = threadIdx.x / 64; g < a.G; g += NT / 64) {
        double t1 = 0.0, t2 = 0.0;
        for (int c = g * a.Cg + lane; c < (g + 1) * a.Cg; c += 64) {
            const double w = (double)Store<T>::load(gamma, c);
            t1 = fma(w, (double)ch[2 * c + 1], t1);
            t2 = fma(w, (double)ch[2 * c], t2);
        }
        t1 = lanes_sum<64>(t1);
        t2 = lanes_sum<64>(t2);
        if (lane == 0) means[g] = make_float2((float)(t1 * inv), (float)(t2 * inv));
    }
    __syncthreads();
    if (!dx || !col.have) return;
    float m1[N], m2[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float2 m = means[j < col.have ? (col.c + j) / a.Cg : 0];
        m1[j] = m.x;
        m2[j] = m.y;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const long long q = col.row + (long long)k * a.rows;
        if (q >= a.V) break;
        float v[N], d[N];
        Piece<T>::unpack(rx[k], v);
        Piece<T>::unpack(rd[k], d);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float xh, dv;
            f.values(j, a.act, v[j], d[j], xh, dv);
            d[j] = f.rstd[j] * (fmaf(f.gamma[j], dv, -m1[j]) - xh * m2[j]);
        }
        store_piece<T>(dx + at + q * a.C, col.have, d);
    }
}

int check_gn(int64_t N, int64_t V, int32_t C, int32_t G, int32_t dtype)
{
    if (N < 1 || V < 1 || C < 1 || G < 1 || C % G) return PLSTM_EINVAL;
    if (dtype != PLSTM_F32 && dtype != PLSTM_BF16) return PLSTM_EINVAL;
    if (C > kGnMaxC || N > (1LL << 22) || V > (1LL << 36) || N * V > (1LL << 38) / C) return PLSTM_EUNSUPPORTED;
    if (N * G > (1LL << 30)) return PLSTM_EUNSUPPORTED;
    return PLSTM_OK;
}

// How a call is spread.  held: rows a thread of the one workgroup that holds a volume (0: the volume
// is cut into slabs).
struct GnPlan {
    GnArgs a;
    int threads, held, blocks_y;
};

GnPlan gn_plan(int64_t N, int64_t V, int32_t C, int32_t G, int32_t dtype, int32_t act, float eps, int most)
{
    GnPlan p{};
    const int e = dtype == PLSTM_F32 ? 4 : 8;
    GnArgs &a = p.a;
    a.N = N; a.V = V; a.C = C; a.G = G; a.Cg = C / G; a.act = act; a.eps = eps;
    a.pieces = (C + e - 1) / e;
    for (int nt : {kGnThreads, kGnSmall}) {
        if (a.pieces > nt || C > kGnHeldC) continue;
        const int rows = nt / a.pieces;
        const long long held = (V + rows - 1) / rows;
        if (held > (nt == kGnThreads ? min(most, 4) : most)) continue;
        a.across = a.pieces;
        a.rows = rows;
        a.slabs = 1;
        a.slab = V;
        p.threads = nt;
        p.held = 1;
        while (p.held < held) p.held *= 2;
        p.blocks_y = 1;
        return p;
    }
    a.across = min(a.pieces, kGnThreads);
    a.rows = kGnThreads / a.across;
    p.blocks_y = (a.pieces + a.across - 1) / a.across;
    p.threads = kGnThreads;
    // slabs of whole turns of four rows a thread, of one where that would leave most of the card idle
    const long long turn = N * ((V + 4LL * a.rows - 1) / (4LL * a.rows)) * p.blocks_y < 256 ? a.rows : 4LL * a.rows;
    const long long want = kGnBlocks / (N * p.blocks_y) + 1;
    a.slab = ((V + want - 1) / want + turn - 1) / turn * turn;
    a.slabs = (int)((V + a.slab - 1) / a.slab);
    return p;
}

// Rows a thread of a workgroup of 1024 that holds a volume: what fits 128 registers beside the sums.
constexpr int gn_held(int dtype, bool backward)
{
    return (dtype == PLSTM_F32 ? 16 : 8) / (backward ? 2 : 1);
}

template <typename T, int NT, int K>
int launch_small_fwd(const GnPlan &p, const void *x, const void *gamma, const void *beta, void *y, void *stats,
                      hipStream_t st)
{
    const size_t lds = sizeof(double) * (sum_rows_lds<NT, Piece<T>::N>(p.a.across) + 2 * p.a.C) + sizeof(GroupStats) * p.a.G;
    if (lds > 65536)
        (void)hipFuncSetAttribute((const void *)k_gn_small_fwd<T, NT, K>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                  (int)lds);
    return in_launches<NT>(p.a.N, [&](unsigned first, unsigned n) {
        k_gn_small_fwd<T, NT, K><<<n, NT, lds, st>>>(p.a, first, (const T *)x, (const T *)gamma, (const T *)beta,
                                                     (T *)y, (float *)stats);
    });
}

template <typename T, int NT, int K>
int launch_small_bwd(const GnPlan &p, const void *x, const void *gamma, const void *beta, const void *stats,
                      const void *dy, void *dx, double *part, void *dgamma, void *dbeta, hipStream_t st)
{
    const size_t lds = sizeof(float) * (sum_rows_lds<NT, Piece<T>::N>(p.a.across) + 2 * p.a.C) + sizeof(float2) * p.a.G;
    if (lds > 65536)
        (void)hipFuncSetAttribute((const void *)k_gn_small_bwd<T, NT, K>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                  (int)lds);
    return in_launches<NT>(p.a.N, [&](unsigned first, unsigned n) {
        k_gn_small_bwd<T, NT, K><<<n, NT, lds, st>>>(p.a, first, (const T *)x, (const T *)gamma, (const T *)beta,
                                                     (const float *)stats, (const T *)dy, (T *)dx, part,
                                                     (float *)dgamma, (float *)dbeta);
    });
}

template <typename T>
int gn_forward(const GnPlan &p, const void *x, const void *gamma, const void *beta, void *y, void *stats, void *ws,
               hipStream_t st)
{
    const GnArgs &a = p.a;
    if (p.held) {
        int n = 0;
        const auto go = [&](auto fn) { n = fn(p, x, gamma, beta, y, stats, st); };
        if (p.threads == kGnThreads) {
            if (p.held == 1) go(launch_small_fwd<T, kGnThreads, 1>);
            else if (p.held == 2) go(launch_small_fwd<T, kGnThreads, 2>);
            else go(launch_small_fwd<T, kGnThreads, 4>);
        } else {
            if (p.held <= 2) go(launch_small_fwd<T, kGnSmall, 2>);
            else if (p.held == 4) go(launch_small_fwd<T, kGnSmall, 4>);
            else if (p.held == 8) go(launch_small_fwd<T, kGnSmall, 8>);
            else if constexpr (sizeof(T) == 4) go(launch_small_fwd<T, kGnSmall, 16>);
        }
        PLSTM_LAUNCH_CHECK();
        return n;
    }
    Carve cv(ws);
    double *part = cv.take<double>((size_t)a.N * a.slabs * a.C * 2);
    GroupStats *gs = cv.take<GroupStats>((size_t)a.N * a.G);
    const dim3 grid((unsigned)(a.N * a.slabs), p.blocks_y);
    const bool stream = a.N * a.V * a.C * (long long)sizeof(T) >= kStreamBytes;
    k_gn_sums<T><<<grid, kGnThreads, 0, st>>>(a, (const T *)x, part);
    PLSTM_LAUNCH_CHECK();
    // few parts are added by every workgroup for itself (a slab's worth of them: up to 64 of at most 256 channels): 1 x 4096 x 32
    // 13.5 us a call, with a launch between 15.8
    const bool few = a.slabs <= 64 && a.C <= 256;
    int launches = 2;
    if (!few) {
        launches += in_launches<1024>(a.N * a.G, [&](unsigned first, unsigned n) {
            k_gn_stats<<<n, 1024, 0, st>>>(a, first, part, gs, (float *)stats);
        });
        PLSTM_LAUNCH_CHECK();
    }
    const auto apply = few      ? (stream ? k_gn_apply<T, true, true> : k_gn_apply<T, false, true>)
                       : stream ? k_gn_apply<T, true, false>
                                : k_gn_apply<T, false, false>;
    apply<<<grid, kGnThreads, 0, st>>>(a, (const T *)x, (const T *)gamma, (const T *)beta, gs, (T *)y, part,
                                       few ? (float *)stats : nullptr);
    PLSTM_LAUNCH_CHECK();
    return launches;
}

template <typename T>
int gn_backward(const GnPlan &p, const void *x, const void *gamma, const void *beta, const void *stats, const void *dy,
                void *dx, void *dgamma, void *dbeta, void *ws, hipStream_t st)
{
    const GnArgs &a = p.a;
    Carve cv(ws);
    double *part = cv.take<double>((size_t)a.N * a.slabs * a.C * 2);
    float2 *means = cv.take<float2>((size_t)a.N * a.G);
    const int weights = (a.C + 15) / 16;
    if (p.held) {
        int n = 0;
        const auto go = [&](auto fn) { n = fn(p, x, gamma, beta, stats, dy, dx, part, dgamma, dbeta, st); };
        if (p.threads == kGnThreads) {
            if (p.held == 1) go(launch_small_bwd<T, kGnThreads, 1>);
            else if (p.held == 2) go(launch_small_bwd<T, kGnThreads, 2>);
            else go(launch_small_bwd<T, kGnThreads, 4>);
        } else {
            if (p.held <= 2) go(launch_small_bwd<T, kGnSmall, 2>);
            else if (p.held == 4) go(launch_small_bwd<T, kGnSmall, 4>);
            else if constexpr (sizeof(T) == 4) go(launch_small_bwd<T, kGnSmall, 8>);
        }
        PLSTM_LAUNCH_CHECK();
        if (a.N == 1) return n;
        k_gn_bwd_finish<T><<<weights, 1024, 0, st>>>(a, 0, 0, (const T *)gamma, part, means, (float *)dgamma,
                                                     (float *)dbeta);
        PLSTM_LAUNCH_CHECK();
        return n + 1;
    }
    const dim3 grid((unsigned)(a.N * a.slabs), p.blocks_y);
    const bool stream = a.N * a.V * a.C * (long long)sizeof(T) >= kStreamBytes;
    k_gn_bwd_sums<T><<<grid, kGnThreads, 0, st>>>(a, (const T *)x, (const T *)gamma, (const T *)beta,
                                                  (const float *)stats, (const T *)dy, part);
    PLSTM_LAUNCH_CHECK();
    const int launches = 1 + in_launches<1024>(a.N * a.G, [&](unsigned first, unsigned n) {
        // the weights with the last ones
        k_gn_bwd_finish<T><<<n + (first + n == a.N * a.G ? weights : 0), 1024, 0, st>>>(
            a, first, (int)n, (const T *)gamma, part, means, (float *)dgamma, (float *)dbeta);
    });
    PLSTM_LAUNCH_CHECK();
    if (!dx) return launches;
    (stream ? k_gn_bwd_apply<T, true> : k_gn_bwd_apply<T, false>)<<<grid, kGnThreads, 0, st>>>(
        a, (const T *)x, (const T *)gamma, (const T *)beta, (const float *)stats, (const T *)dy, means, (T *)dx);
    PLSTM_LAUNCH_CHECK();
    return launches + 1;
}

}  // namespace
}  // namespace plstm

using namespace plstm;

extern "C" {

size_t pyramid_group_norm_workspace_size(int64_t N, int64_t V, int32_t C, int32_t G)
{
    if (check_gn(N, V, C, G, PLSTM_F32) != PLSTM_OK) return 0;
    size_t most = 256;
    for (int dtype : {PLSTM_F32, PLSTM_BF16})
        for (bool backward : {false, true}) {
            const GnPlan p = gn_plan(N, V, C, G, dtype, 0, 1.0f, gn_held(dtype, backward));
            if (p.held && (!backward || N == 1)) continue;
            Carve cv(nullptr);
            cv.take<double>((size_t)N * p.a.slabs * C * 2);
            cv.take<GroupStats>((size_t)N * G);
            most = max(most, align_up(cv.off, 256));
        }
    return most;
}

int pyramid_group_norm_forward(int64_t N, int64_t V, int32_t C, int32_t G, int32_t dtype, int32_t act,
                               float eps, const void *x, const void *gamma, const void *beta, void *y,
                               void *stats, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = check_gn(N, V, C, G, dtype);
    if (rc != PLSTM_OK) return rc;
    const size_t e = dtype_size(dtype);
    if ((act != 0 && act != 1) || !(eps > 0.0f && eps <= 3.0e38f) || !x || !gamma || !beta || !y || !ws)
        return PLSTM_EINVAL;
    if (!aligned_to(x, e) || !aligned_to(gamma, e) || !aligned_to(beta, e) || !aligned_to(y, e) ||
        !aligned_to(stats, 4) || !aligned_to(ws, 16))
        return PLSTM_EINVAL;
    if (ws_bytes < pyramid_group_norm_workspace_size(N, V, C, G)) return PLSTM_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const GnPlan p = gn_plan(N, V, C, G, dtype, act, eps, gn_held(dtype, false));
    timing_begin("group_norm_fwd", st);
    const int n = (dtype == PLSTM_F32 ? gn_forward<float> : gn_forward<uint16_t>)(p, x, gamma, beta, y, stats, ws, st);
    if (n < 0) return n;
    timing_end(n, st);
    return PLSTM_OK;
}

int pyramid_group_norm_backward(int64_t N, int64_t V, int32_t C, int32_t G, int32_t dtype, int32_t act,
                                const void *x, const void *gamma, const void *beta, const void *stats,
                                const void *dy, void *dx, void *dgamma, void *dbeta, void *ws, size_t ws_bytes,
                                void *stream)
{
    const int rc = check_gn(N, V, C, G, dtype);
    if (rc != PLSTM_OK) return rc;
    const size_t e = dtype_size(dtype);
    if ((act != 0 && act != 1) || !x || !gamma || !beta || !stats || !dy || !dgamma || !dbeta || !ws)
        return PLSTM_EINVAL;
    if (!aligned_to(x, e) || !aligned_to(gamma, e) || !aligned_to(beta, e) || !aligned_to(stats, 4) ||
        !aligned_to(dy, e) || !aligned_to(dx, e) || !aligned_to(dgamma, 4) || !aligned_to(dbeta, 4) ||
        !aligned_to(ws, 16))
        return PLSTM_EINVAL;
    if (ws_bytes < pyramid_group_norm_workspace_size(N, V, C, G)) return PLSTM_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const GnPlan p = gn_plan(N, V, C, G, dtype, act, 1.0f, gn_held(dtype, true));
    timing_begin("group_norm_bwd", st);
    const int n = (dtype == PLSTM_F32 ? gn_backward<float> : gn_backward<uint16_t>)(
        p, x, gamma, beta, stats, dy, dx, dgamma, dbeta, ws, st);
    if (n < 0) return n;
    timing_end(n, st);
    return PLSTM_OK;
}

}  // extern "C"
