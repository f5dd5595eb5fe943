// Selective state space scan along an axis, and its backward pass.  Over sweep positions s
// (sequence.h), for channel i and state k, d = delta + bias (of it the softplus, if asked):
//   a = exp(d A[i][k]),  h_s = a h_{s-1} + d u B_s[k],  p_s = sum_k C_s[k] h_s + D u,  y = p silu(z)
// Backward, dp = dy silu(z) and G_s the gradient of h_s:
//   G_s = C_s dp_s + a_{s+1} G_{s+1}  (the last one takes dhT as well),  dh0 = a_0 G_0
//   dC = sum_i dp h,  dB = sum_i G d u,  q = sum_k G B,  w = sum_k G a h_{s-1} A
//   du = d q + D dp,  dd = u q + w,  dA = sum G a h_{s-1} d,  dD = sum dp u,  dz = dy p silu'(z)
// A workgroup of 8 waves has 16 channels and walks its sequence in tiles.  A lane has one
// channel and a quarter of its states (SR of them), a wave a run of R positions of a tile: it folds its
// run to (P, H), last state = P h + H, keeping the decays in registers; the waves
// exchange these through LDS and run again from the state that reaches them.  So a decay costs one exponential,
// whatever the run's place: the quarter-rate v_exp_f32 (16 of the some 36 cycles that a
// state of a position costs a wave) bounds everything but the smallest S.
// What belongs to an element and not to its states (softplus, d u, the gate) is done once, two
// elements a thread, and passes through LDS.
#include "sequence.h"
#include "timing.h"

namespace plstm {
namespace {

constexpr int kSelMaxS = 64;
constexpr int kSelCh = 16;              // channels of a workgroup, in the lanes of a row of 16
constexpr int kSelW = 8;                // waves
constexpr int kSelThreads = 64 * kSelW;
constexpr float kLog2e = 1.44269504f;

// States a lane and positions of a wave's run, so that SR R decays fit its registers.
inline int sel_sr(int S) { return S <= 4 ? 1 : S <= 8 ? 2 : S <= 16 ? 4 : S <= 32 ? 8 : 16; }
__host__ __device__ constexpr int sel_run(int SR) { return SR <= 4 ? 8 : 32 / SR; }
// Positions of a tile, and between the states that a training forward keeps.
__host__ __device__ constexpr int sel_tile(int SR) { return kSelW * sel_run(SR); }

struct SelArgs {
    long long B, T, I;
    int S, reverse, softplus;
    long long pu, pd, pz, pB, pC;       // elements from one row to the next
    const int32_t *lengths;
    long long tiles;                    // workgroups across the channels
    long long kept;                     // states that a sequence keeps
    int chunks;                         // of a sequence, each with workgroups of its own
    long long chunk;                    // positions of a chunk (whole tiles)
    long long jobs;                     // backward: workgroups down the sequences and chunks
};

// Two elements from any element on, raw.
template <typename T> struct Two;
template <> struct Two<float> {
    uint32_t w[2];
    __device__ void load(const float *p, int have)
    {
        typedef uint32_t V __attribute__((ext_vector_type(2), aligned(4)));
        w[0] = w[1] = 0;
        if (have >= 2) {
            const V r = *(const V *)p;
            w[0] = r[0];
            w[1] = r[1];
        } else if (have == 1) {
            w[0] = float_bits(*p);
        }
    }
    __device__ float lo() const { return bits_float(w[0]); }
    __device__ float hi() const { return bits_float(w[1]); }
    __device__ static void store(float *p, int have, float a, float b)
    {
        typedef uint32_t V __attribute__((ext_vector_type(2), aligned(4)));
        if (have >= 2) *(V *)p = V{float_bits(a), float_bits(b)};
        else if (have == 1) *p = a;
    }
};
template <> struct Two<uint16_t> {
    typedef uint32_t V __attribute__((aligned(2)));
    uint32_t w;
    __device__ void load(const uint16_t *p, int have)
    {
        w = 0;
        if (have >= 2) w = *(const V *)p;
        else if (have == 1) w = *p;
    }
    __device__ float lo() const { return bits_float(w << 16); }
    __device__ float hi() const { return bits_float(w & 0xffff0000u); }
    __device__ static void store(uint16_t *p, int have, float a, float b)
    {
        if (have >= 2) *(V *)p = pack_bf16(a, b);
        else if (have == 1) *p = (uint16_t)pack_bf16(a, a);
    }
};

// log(1 + exp(v)) and its derivative sigmoid(v).  log(1 + e) for e = exp(-|v|): where 1 + e
// rounds, its logarithm is that of another number, by the factor e / ((1 + e) - 1) (Kahan).
__device__ inline float softplus_of(float v)
{
    const float e = __builtin_amdgcn_exp2f(fabsf(v) * -kLog2e);
    const float w = 1.0f + e, x = w - 1.0f;
    const float l = x == 0.0f ? e : __builtin_amdgcn_logf(w) * 0.69314718f * (e * __builtin_amdgcn_rcpf(x));
    return v > 0.0f ? v + l : v == v ? l : v;
}

// Sum over the four rows of 16 lanes (a channel's quarters of states) of R values: lane (row,
// channel) gets that of value sel_row_value(row) + 4 q in v[q]; R = 2: value row / 2.
// Two swaps of half waves and rows and three additions make four sums.
__device__ inline void swap32(float &x, float &y)
{
    const auto r = __builtin_amdgcn_permlane32_swap(float_bits(x), float_bits(y), false, false);
    x = bits_float(r[0]);
    y = bits_float(r[1]);
}
__device__ inline void swap16(float &x, float &y)
{
    const auto r = __builtin_amdgcn_permlane16_swap(float_bits(x), float_bits(y), false, false);
    x = bits_float(r[0]);
    y = bits_float(r[1]);
}
template <int R>
__device__ inline void sum_rows_of_lanes(float *v)
{
    if constexpr (R == 2) {
        swap32(v[0], v[1]);
        float s = v[0] + v[1], t = s;
        swap16(s, t);
        v[0] = s + t;
    } else {
#pragma unroll
        for (int q = 0; q < R / 4; ++q) {
            float *x = v + 4 * q;
            swap32(x[0], x[1]);
            swap32(x[2], x[3]);
            float s = x[0] + x[1], t = x[2] + x[3];
            swap16(s, t);
            v[q] = s + t;
        }
    }
}
template <int R> __device__ inline int row_value(int row) { return R == 2 ? row >> 1 : (row & 1) << 1 | row >> 1; }
// Writes those sums, position first + r of channel ch, to a tile [positions][16].
template <int R>
__device__ inline void put_rows(float (*tile)[kSelCh], int first, int row, int ch, const float *v)
{
    if constexpr (R == 2) {
        if (!(row & 1)) tile[first + (row >> 1)][ch] = v[0];
    } else {
#pragma unroll
        for (int q = 0; q < R / 4; ++q) tile[first + 4 * q + row_value<R>(row)][ch] = v[q];
    }
}

// Sum over the 16 lanes of a row, in every lane.
__device__ inline float sum_channels(float v) { return lanes_sum<16>(v); }

// A thread's two elements of a tile: position `row`, channels 2 pair and the next.
struct Mine {
    int row, pair, have;                // have: channels that there are (0: an idle thread)
    __device__ Mine(int TT, long long i0, long long I)
    {
        row = threadIdx.x / 8;
        pair = threadIdx.x % 8;
        const long long left = I - (i0 + 2 * pair);
        have = row >= TT || left <= 0 ? 0 : left < 2 ? 1 : 2;
    }
};

// One workgroup's place: 16 channels of a sequence, from position `first` on.
struct Place {
    long long b, i0, n, first, last;    // last: end of the chunk
    __device__ Place(const SelArgs &a, long long b_, long long tile, int chunk)
    {
        b = b_;
        i0 = tile * kSelCh;
        n = length_of(a.lengths, b, a.T);
        first = chunk * a.chunk;
        last = min(a.T, first + a.chunk);
    }
    __device__ long long row(const SelArgs &a, long long s) const { return b * a.T + step_of(s, n, a.reverse); }
};

// Workgroups of neighbouring channels of a sequence share lines of its rows: those of an XCD
// (every eighth) are given consecutive numbers.
__device__ inline long long spread(long long id, long long all)
{
    const long long each = all / 8, rest = all - each * 8, x = id & 7;
    return (x < rest ? x * (each + 1) : rest * (each + 1) + (x - rest) * each) + (id >> 3);
}

// The raw inputs of a tile that a thread loads: its elements, and two values each of B and C.
template <typename T, int SR>
struct RawTile {
    static constexpr int SP = 4 * SR, TT = sel_tile(SR), PAIRS = TT * SP / 2;
    static constexpr int NB = (PAIRS + kSelThreads - 1) / kSelThreads;
    Two<T> u, d, z, g, B[NB], C[NB];
    bool live;
    // g: dy, dense
    __device__ void load(const SelArgs &a, const Place &p, const Mine &m, long long s0, const T *pu, const T *pd,
                         const T *pz, const T *pg, const T *pB, const T *pC)
    {
        const long long s = s0 + m.row;
        live = s < p.last && s < p.n;
        const int have = live ? m.have : 0;
        const long long r = live ? p.row(a, s) : 0, i = p.i0 + 2 * m.pair;
        u.load(pu + r * a.pu + i, have);
        d.load(pd + r * a.pd + i, have);
        if (pz) z.load(pz + r * a.pz + i, have);
        if (pg) g.load(pg + r * a.I + i, have);
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            const int e = threadIdx.x + q * kSelThreads, row = e / (SP / 2), k = e % (SP / 2) * 2;
            const long long t = s0 + row;
            const int n = row < TT && t < p.last && t < p.n ? (k + 1 < a.S ? 2 : k < a.S ? 1 : 0) : 0;
            const long long rt = n ? p.row(a, t) : 0;
            B[q].load(pB + rt * a.pB + k, n);
            if (pC) C[q].load(pC + rt * a.pC + k, n);
        }
    }
};

// d and d u of an element.
__device__ inline float step_size(const SelArgs &a, float raw, float bias, bool live)
{
    const float v = raw + bias;
    return live ? (a.softplus ? softplus_of(v) : v) : 0.0f;
}

template <int SR, bool BACK>
struct alignas(16) SelShared {
    static constexpr int SP = 4 * SR, TT = sel_tile(SR), TB = BACK ? TT : 1;
    float2 du[TT][kSelCh];              // d, d u
    float B[TT][SP], C[TT][SP];
    float P[kSelW][SR][64], H[kSelW][SR][64], X[BACK ? kSelW : 1][SR][64];
    float carry[2][SR][64];             // the state (BACK: what the gradient passes on) between tiles, by turns
    float y[TT][kSelCh];                // BACK: p without D u
    float dp[TB][kSelCh], q[TB][kSelCh], w[TB][kSelCh];
    float dB[TB][SP], dC[TB][SP];
};

// The part of a lane in the decays: A log2(e) of its channel's states.
template <int SR>
__device__ inline void lane_A(const SelArgs &a, const Place &p, const float *A, int row, int ch, float scale, float *out)
{
    const long long i = p.i0 + ch;
#pragma unroll
    for (int j = 0; j < SR; ++j) {
        const int k = row * SR + j;
        out[j] = i < a.I && k < a.S ? A[i * a.S + k] * scale : 0.0f;
    }
}
// Element (b, i, row SR + j) of a state [..][I][S]; false where there is none.
template <int SR>
__device__ inline bool state_at(const SelArgs &a, const Place &p, long long outer, int row, int ch, int j, long long &at)
{
    const long long i = p.i0 + ch;
    const int k = row * SR + j;
    at = (outer * a.I + i) * a.S + k;
    return i < a.I && k < a.S;
}

// FOLD: the state after each chunk but the last, for workgroups that have a chunk:
// fold [chunk][b][i][k] (P, H), chunk 0 from h0.
template <typename T, int SR, bool FOLD>
__global__ void __launch_bounds__(kSelThreads, SR < 16 ? 4 : 2)
k_sel_fwd(SelArgs a, const T *u, const T *delta, const float *A, const T *Bm, const T *Cm, const float *D,
          const T *z, const float *dbias, const float *h0, T *y, float *hT, float *saved, float2 *fold)
{
    constexpr int R = sel_run(SR), TT = sel_tile(SR), SP = 4 * SR;
    typedef RawTile<T, SR> Raw;
    __shared__ SelShared<SR, false> sh;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, row = lane >> 4, ch = lane & 15;
    const long long id = spread(blockIdx.x, gridDim.x);
    const int nchunks = FOLD ? a.chunks - 1 : a.chunks;
    const long long bt = id / a.tiles, b = bt / nchunks;
    const int chunk = (int)(bt - b * nchunks);
    const Place p(a, b, id - bt * a.tiles, chunk);
    const Mine m(TT, p.i0, a.I);
    float A2[SR];
    lane_A<SR>(a, p, A, row, ch, kLog2e, A2);
    if (wave == 0) {
#pragma unroll
        for (int j = 0; j < SR; ++j) {
            long long at;
            float h = 0.0f;
            if (state_at<SR>(a, p, b, row, ch, j, at)) {
                if (a.chunks == 1) {
                    h = h0 ? h0[at] : 0.0f;
                } else if (FOLD) {
                    h = chunk == 0 && h0 ? h0[at] : 0.0f;
                    // h0 may be where the state after goes
                    if (chunk == 0) fold[(long long)(a.chunks - 1) * a.B * a.I * a.S + at] = make_float2(0.0f, h);
                } else if (chunk == 0) {
                    h = fold[(long long)(a.chunks - 1) * a.B * a.I * a.S + at].y;
                } else {
                    h = fold[at].y;
                    for (int c = 1; c < chunk; ++c) {
                        const float2 f = fold[(long long)c * a.B * a.I * a.S + at];
                        h = fmaf(f.x, h, f.y);
                    }
                }
            }
            sh.carry[0][j][lane] = h;
        }
    }
    float bias[2], Dv[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const long long i = p.i0 + 2 * m.pair + e;
        bias[e] = dbias && e < m.have ? dbias[i] : 0.0f;
        Dv[e] = D && e < m.have ? D[i] : 0.0f;
    }
    float Pall[SR];
#pragma unroll
    for (int j = 0; j < SR; ++j) Pall[j] = 1.0f;
    Raw raw;
    raw.load(a, p, m, p.first, u, delta, FOLD ? nullptr : z, nullptr, Bm, FOLD ? nullptr : Cm);
    int turn = 0;
    for (long long s0 = p.first; s0 < p.last; s0 += TT, turn ^= 1) {
        const float u0 = raw.u.lo(), u1 = raw.u.hi();
        const Two<T> zz = raw.z;
        const bool live = raw.live;
        if (m.row < TT) {
            const float d0 = step_size(a, raw.d.lo(), bias[0], live), d1 = step_size(a, raw.d.hi(), bias[1], live);
            *(float4 *)&sh.du[m.row][2 * m.pair] = make_float4(d0, d0 * u0, d1, d1 * u1);
        }
#pragma unroll
        for (int q = 0; q < Raw::NB; ++q) {
            const int e = threadIdx.x + q * kSelThreads, r = e / (SP / 2), k = e % (SP / 2) * 2;
            if (r < TT) {
                *(float2 *)&sh.B[r][k] = make_float2(raw.B[q].lo(), raw.B[q].hi());
                if (!FOLD) *(float2 *)&sh.C[r][k] = make_float2(raw.C[q].lo(), raw.C[q].hi());
            }
        }
        __syncthreads();
        if (s0 + TT < p.last)
            raw.load(a, p, m, s0 + TT, u, delta, FOLD ? nullptr : z, nullptr, Bm, FOLD ? nullptr : Cm);
        const int first = wave * R;
        float dec[R][SR], h[SR], sum = 0.0f;
#pragma unroll
        for (int j = 0; j < SR; ++j) h[j] = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float2 v = sh.du[first + r][ch];
            sum += v.x;
#pragma unroll
            for (int j = 0; j < SR; ++j) {
                dec[r][j] = __builtin_amdgcn_exp2f(v.x * A2[j]);
                h[j] = fmaf(dec[r][j], h[j], v.y * sh.B[first + r][row * SR + j]);
            }
        }
#pragma unroll
        for (int j = 0; j < SR; ++j) {
            sh.P[wave][j][lane] = __builtin_amdgcn_exp2f(sum * A2[j]);
            sh.H[wave][j][lane] = h[j];
        }
        __syncthreads();
        const int before = FOLD ? kSelW : wave;
        if (!FOLD || wave == 0) {
#pragma unroll
            for (int j = 0; j < SR; ++j) h[j] = sh.carry[turn][j][lane];
            for (int w = 0; w < before; ++w)
#pragma unroll
                for (int j = 0; j < SR; ++j) {
                    h[j] = fmaf(sh.P[w][j][lane], h[j], sh.H[w][j][lane]);
                    if (FOLD) Pall[j] *= sh.P[w][j][lane];
                }
        }
        if (FOLD) {
            if (wave == 0)
#pragma unroll
                for (int j = 0; j < SR; ++j) sh.carry[turn ^ 1][j][lane] = h[j];
            continue;       // the next tile's first barrier comes before anything that was read is overwritten but du and B
        }
        if (saved && wave == 0)
#pragma unroll
            for (int j = 0; j < SR; ++j) {
                long long at;
                if (state_at<SR>(a, p, b * a.kept + s0 / TT, row, ch, j, at)) saved[at] = h[j];
            }
        float yp[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float v = sh.du[first + r][ch].y;
            yp[r] = 0.0f;
#pragma unroll
            for (int j = 0; j < SR; ++j) {
                h[j] = fmaf(dec[r][j], h[j], v * sh.B[first + r][row * SR + j]);
                yp[r] = fmaf(sh.C[first + r][row * SR + j], h[j], yp[r]);
            }
        }
        sum_rows_of_lanes<R>(yp);
        put_rows<R>(sh.y, first, row, ch, yp);
        if (wave == kSelW - 1)
#pragma unroll
            for (int j = 0; j < SR; ++j) sh.carry[turn ^ 1][j][lane] = h[j];
        __syncthreads();
        const long long s = s0 + m.row;
        if (m.have && s < p.last) {
            const float2 v = *(const float2 *)&sh.y[m.row][2 * m.pair];
            float y0 = fmaf(Dv[0], u0, v.x), y1 = fmaf(Dv[1], u1, v.y);
            if (z) {
                y0 *= silu_of(zz.lo());
                y1 *= silu_of(zz.hi());
            }
            Two<T>::store(y + p.row(a, s) * a.I + p.i0 + 2 * m.pair, m.have, live ? y0 : 0.0f, live ? y1 : 0.0f);
        }
    }
    if (wave == 0 && (FOLD || (hT && chunk == a.chunks - 1)))
#pragma unroll
        for (int j = 0; j < SR; ++j) {
            long long at;
            if (!state_at<SR>(a, p, b, row, ch, j, at)) continue;
            const float v = sh.carry[turn][j][lane];
            if (FOLD) fold[(long long)chunk * a.B * a.I * a.S + at] = make_float2(Pall[j], v);
            else hT[at] = v;
        }
}

// A single step: L lanes of 4 states a channel.
template <typename T, int L>
__global__ void __launch_bounds__(256)
k_sel_step(SelArgs a, const T *u, const T *delta, const float *A, const T *Bm, const T *Cm, const float *D, const T *z,
           const float *dbias, const float *h0, T *y, float *hT)
{
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, col = at / L;
    const int l = (int)(at % L);
    if (col >= a.B * a.I) return;       // whole groups of L lanes
    const long long b = col / a.I, i = col - b * a.I;
    const bool live = length_of(a.lengths, b, 1) > 0;
    const int k0 = 4 * l, have = min(a.S - k0, 4);
    float h[4], Av[4], Bv[4], Cv[4];
    Four<float> rh, rA;
    Four<T> rB, rC;
    rh.zero();
    if (h0) rh.load(h0 + col * a.S + k0, have);
    rA.load(A + i * a.S + k0, have);
    rB.load(Bm + b * a.pB + k0, have);
    rC.load(Cm + b * a.pC + k0, have);
    const float uv = Store<T>::load(u, b * a.pu + i), raw = Store<T>::load(delta, b * a.pd + i);
    const float zv = z ? Store<T>::load(z, b * a.pz + i) : 0.0f;
    rh.get(h);
    rA.get(Av);
    rB.get(Bv);
    rC.get(Cv);
    const float d = step_size(a, raw, dbias ? dbias[i] : 0.0f, true);
    float s = 0.0f;
    if (live) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            h[j] = fmaf(__builtin_amdgcn_exp2f(d * (Av[j] * kLog2e)), h[j], d * uv * Bv[j]);
            s = j < have ? fmaf(Cv[j], h[j], s) : s;
        }
    }
    s = lanes_sum<L>(s);
    if (hT && have > 0) Four<float>::store(hT + col * a.S + k0, have, h);
    if (l == 0) {
        float v = D ? fmaf(D[i], uv, s) : s;
        if (z) v *= silu_of(zv);
        Store<T>::store(y, col, live ? v : 0.0f);
    }
}

// FOLD: what the gradient passes on below each chunk but the first, for workgroups that have
// a chunk: fold [chunk][b][i][k] (P, X), the last one's from dhT.
// Else: parts of the sums over channels (dBp, dCp [tile][b][t][S], where there are several tiles) and of those
// over positions (dAp [job][I][S], dDp [job][I][2]).
template <typename T, int SR, bool FOLD>
__global__ void __launch_bounds__(kSelThreads, 2)
k_sel_bwd(SelArgs a, const T *u, const T *delta, const float *A, const T *Bm, const T *Cm, const float *D, const T *z,
          const float *dbias, const float *saved, const T *dy, const float *dhT, T *du, T *ddelta, T *dz, float *dh0,
          float *dBp, float *dCp, T *dB, T *dC, float *dAp, float *dDp, float2 *fold)
{
    constexpr int R = sel_run(SR), TT = sel_tile(SR), SP = 4 * SR;
    typedef RawTile<T, SR> Raw;
    __shared__ SelShared<SR, !FOLD> sh;
    __shared__ float foldX[FOLD ? kSelW : 1][SR][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, row = lane >> 4, ch = lane & 15;
    const long long id = spread(blockIdx.x, gridDim.x);
    const long long job0 = id / a.tiles, tile = id - job0 * a.tiles;
    const int nchunks = FOLD ? a.chunks - 1 : a.chunks;
    const long long states = a.B * a.I * a.S;
    float Av[SR], dA[SR], dDv[2] = {0.0f, 0.0f}, dbv[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < SR; ++j) dA[j] = 0.0f;
    for (long long job = job0; job < a.B * nchunks; job += a.jobs) {
        const long long b = job / nchunks;
        const int chunk = (int)(job - b * nchunks) + (FOLD ? 1 : 0);
        const Place p(a, b, tile, chunk);
        const Mine m(TT, p.i0, a.I);
        lane_A<SR>(a, p, A, row, ch, 1.0f, Av);
        __syncthreads();                // the job before is done with LDS
        if (wave == 0) {
#pragma unroll
            for (int j = 0; j < SR; ++j) {
                long long at;
                float x = 0.0f;
                if (state_at<SR>(a, p, b, row, ch, j, at)) {
                    if (a.chunks == 1) {
                        x = dhT ? dhT[at] : 0.0f;
                    } else if (FOLD) {
                        x = chunk == a.chunks - 1 && dhT ? dhT[at] : 0.0f;
                        // dhT may be where dh0 goes
                        if (chunk == a.chunks - 1) fold[at] = make_float2(0.0f, x);
                    } else if (chunk == a.chunks - 1) {
                        x = fold[at].y;
                    } else {
                        x = fold[(a.chunks - 1) * states + at].y;
                        for (int c = a.chunks - 2; c > chunk; --c) {
                            const float2 f = fold[c * states + at];
                            x = fmaf(f.x, x, f.y);
                        }
                    }
                }
                sh.carry[0][j][lane] = x;
            }
        }
        float bias[2], Dv[2], Pall[SR];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const long long i = p.i0 + 2 * m.pair + e;
            bias[e] = dbias && e < m.have ? dbias[i] : 0.0f;
            Dv[e] = D && e < m.have ? D[i] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < SR; ++j) Pall[j] = 1.0f;
        int turn = 0;
        const long long tiles = (p.last - p.first + TT - 1) / TT;
        Raw raw;
        raw.load(a, p, m, p.first + (tiles - 1) * TT, u, delta, z, dy, Bm, Cm);
        for (long long tl = tiles - 1; tl >= 0; --tl, turn ^= 1) {
            const long long s0 = p.first + tl * TT;
            const float u0 = raw.u.lo(), u1 = raw.u.hi(), g0 = raw.g.lo(), g1 = raw.g.hi();
            const float z0 = raw.z.lo(), z1 = raw.z.hi(), r0 = raw.d.lo() + bias[0], r1 = raw.d.hi() + bias[1];
            const bool live = raw.live;
            float slope[2] = {0.0f, 0.0f}, dp0 = g0, dp1 = g1, d0 = 0.0f, d1 = 0.0f;
            if (z) {
                float s;
                slope[0] = silu_slope(z0, s);
                dp0 = g0 * s;
                slope[1] = silu_slope(z1, s);
                dp1 = g1 * s;
            }
            if (m.row < TT) {
                d0 = step_size(a, raw.d.lo(), bias[0], live);
                d1 = step_size(a, raw.d.hi(), bias[1], live);
                dp0 = live ? dp0 : 0.0f;
                dp1 = live ? dp1 : 0.0f;
                *(float4 *)&sh.du[m.row][2 * m.pair] = make_float4(d0, d0 * u0, d1, d1 * u1);
                if constexpr (!FOLD) *(float2 *)&sh.dp[m.row][2 * m.pair] = make_float2(dp0, dp1);
                else *(float2 *)&sh.y[m.row][2 * m.pair] = make_float2(dp0, dp1);
            }
            const float (*dpt)[kSelCh];
            if constexpr (FOLD) dpt = sh.y; else dpt = sh.dp;
#pragma unroll
            for (int q = 0; q < Raw::NB; ++q) {
                const int e = threadIdx.x + q * kSelThreads, r = e / (SP / 2), k = e % (SP / 2) * 2;
                if (r < TT) {
                    *(float2 *)&sh.B[r][k] = make_float2(raw.B[q].lo(), raw.B[q].hi());
                    *(float2 *)&sh.C[r][k] = make_float2(raw.C[q].lo(), raw.C[q].hi());
                }
            }
            __syncthreads();
            if (tl > 0) raw.load(a, p, m, s0 - TT, u, delta, z, dy, Bm, Cm);
            const int first = wave * R;
            float dec[R][SR], h[SR], x[SR], sum = 0.0f;
            if constexpr (!FOLD) {
#pragma unroll
                for (int j = 0; j < SR; ++j) h[j] = 0.0f;
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float2 v = sh.du[first + r][ch];
                sum += v.x;
#pragma unroll
                for (int j = 0; j < SR; ++j) {
                    dec[r][j] = __builtin_amdgcn_exp2f(v.x * (Av[j] * kLog2e));
                    if constexpr (!FOLD) h[j] = fmaf(dec[r][j], h[j], v.y * sh.B[first + r][row * SR + j]);
                }
            }
#pragma unroll
            for (int j = 0; j < SR; ++j) x[j] = 0.0f;
#pragma unroll
            for (int r = R - 1; r >= 0; --r) {
                const float g = dpt[first + r][ch];
#pragma unroll
                for (int j = 0; j < SR; ++j) x[j] = dec[r][j] * fmaf(sh.C[first + r][row * SR + j], g, x[j]);
            }
            // the state before the tile
            float hs[SR];
#pragma unroll
            for (int j = 0; j < SR; ++j) {
                sh.P[wave][j][lane] = __builtin_amdgcn_exp2f(sum * (Av[j] * kLog2e));
                if constexpr (FOLD) {
                    foldX[wave][j][lane] = x[j];
                } else {
                    sh.X[wave][j][lane] = x[j];
                    sh.H[wave][j][lane] = h[j];
                    long long at;
                    hs[j] = state_at<SR>(a, p, b * a.kept + s0 / TT, row, ch, j, at) ? saved[at] : 0.0f;
                }
            }
            __syncthreads();
            if constexpr (FOLD) {
                if (wave == 0) {
#pragma unroll
                    for (int j = 0; j < SR; ++j) {
                        float v = sh.carry[turn][j][lane];
                        for (int w = kSelW - 1; w >= 0; --w) {
                            v = fmaf(sh.P[w][j][lane], v, foldX[w][j][lane]);
                            Pall[j] *= sh.P[w][j][lane];
                        }
                        sh.carry[turn ^ 1][j][lane] = v;
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < SR; ++j) {
                    h[j] = hs[j];
                    x[j] = sh.carry[turn][j][lane];
                }
                for (int w = 0; w < wave; ++w)
#pragma unroll
                    for (int j = 0; j < SR; ++j) h[j] = fmaf(sh.P[w][j][lane], h[j], sh.H[w][j][lane]);
                for (int w = kSelW - 1; w > wave; --w)
#pragma unroll
                    for (int j = 0; j < SR; ++j) x[j] = fmaf(sh.P[w][j][lane], x[j], sh.X[w][j][lane]);
                float hb[R][SR], yp[R], qv[R], wv[R];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float v = sh.du[first + r][ch].y;
                    yp[r] = 0.0f;
#pragma unroll
                    for (int j = 0; j < SR; ++j) {
                        hb[r][j] = h[j];
                        h[j] = fmaf(dec[r][j], h[j], v * sh.B[first + r][row * SR + j]);
                        yp[r] = fmaf(sh.C[first + r][row * SR + j], h[j], yp[r]);
                    }
                }
                sum_rows_of_lanes<R>(yp);
                put_rows<R>(sh.y, first, row, ch, yp);
#pragma unroll
                for (int r = R - 1; r >= 0; --r) {
                    const float2 v = sh.du[first + r][ch];
                    const float g = dpt[first + r][ch];
                    float gB[SR], gC[SR];
                    qv[r] = wv[r] = 0.0f;
#pragma unroll
                    for (int j = 0; j < SR; ++j) {
                        const float bv = sh.B[first + r][row * SR + j];
                        const float ah = dec[r][j] * hb[r][j];
                        const float G = fmaf(sh.C[first + r][row * SR + j], g, x[j]);
                        const float t = G * ah;
                        gC[j] = g * fmaf(v.y, bv, ah);
                        gB[j] = G * v.y;
                        qv[r] = fmaf(G, bv, qv[r]);
                        wv[r] = fmaf(t, Av[j], wv[r]);
                        dA[j] = fmaf(t, v.x, dA[j]);
                        x[j] = dec[r][j] * G;
                    }
#pragma unroll
                    for (int j = 0; j < SR; ++j) {
                        gB[j] = sum_channels(gB[j]);
                        gC[j] = sum_channels(gC[j]);
                    }
                    if (ch == 0)
#pragma unroll
                        for (int j = 0; j < SR; ++j) {
                            sh.dB[first + r][row * SR + j] = gB[j];
                            sh.dC[first + r][row * SR + j] = gC[j];
                        }
                }
                sum_rows_of_lanes<R>(qv);
                put_rows<R>(sh.q, first, row, ch, qv);
                sum_rows_of_lanes<R>(wv);
                put_rows<R>(sh.w, first, row, ch, wv);
                if (wave == 0)
#pragma unroll
                    for (int j = 0; j < SR; ++j) sh.carry[turn ^ 1][j][lane] = x[j];
                __syncthreads();
                const long long s = s0 + m.row;
                if (m.have && s < p.last) {
                    const float2 pv = *(const float2 *)&sh.y[m.row][2 * m.pair];
                    const float2 q = *(const float2 *)&sh.q[m.row][2 * m.pair];
                    const float2 w = *(const float2 *)&sh.w[m.row][2 * m.pair];
                    float e0 = fmaf(u0, q.x, w.x), e1 = fmaf(u1, q.y, w.y);
                    if (a.softplus) {
                        e0 *= sigmoid_of(r0);
                        e1 *= sigmoid_of(r1);
                    }
                    e0 = live ? e0 : 0.0f;
                    e1 = live ? e1 : 0.0f;
                    const long long at = p.row(a, s) * a.I + p.i0 + 2 * m.pair;
                    Two<T>::store(du + at, m.have, fmaf(d0, q.x, Dv[0] * dp0), fmaf(d1, q.y, Dv[1] * dp1));
                    Two<T>::store(ddelta + at, m.have, e0, e1);
                    if (z)
                        Two<T>::store(dz + at, m.have, live ? g0 * fmaf(Dv[0], u0, pv.x) * slope[0] : 0.0f,
                                      live ? g1 * fmaf(Dv[1], u1, pv.y) * slope[1] : 0.0f);
                    if (live) {
                        dDv[0] = fmaf(dp0, u0, dDv[0]);
                        dDv[1] = fmaf(dp1, u1, dDv[1]);
                        dbv[0] += e0;
                        dbv[1] += e1;
                    }
                }
                for (int e = threadIdx.x; e < TT * SP; e += kSelThreads) {
                    const int r = e / SP, k = e % SP;
                    if (s0 + r >= p.last || k >= a.S) continue;
                    const long long t = p.row(a, s0 + r);
                    if (a.tiles == 1) {
                        Store<T>::store(dB, t * a.S + k, sh.dB[r][k]);
                        Store<T>::store(dC, t * a.S + k, sh.dC[r][k]);
                    } else {
                        const long long at = (tile * a.B * a.T + t) * a.S + k;
                        dBp[at] = sh.dB[r][k];
                        dCp[at] = sh.dC[r][k];
                    }
                }
            }
        }
        __syncthreads();
        if (wave == 0 && (FOLD || (dh0 && chunk == 0)))
#pragma unroll
            for (int j = 0; j < SR; ++j) {
                long long at;
                if (!state_at<SR>(a, p, b, row, ch, j, at)) continue;
                const float v = sh.carry[turn][j][lane];
                if (FOLD) fold[chunk * states + at] = make_float2(Pall[j], v);
                else dh0[at] = v;
            }
    }
    if constexpr (!FOLD) {
        // the waves' parts of dA, the rows' of dD and dbias, in their order
        __syncthreads();
        const Place p(a, 0, tile, 0);
#pragma unroll
        for (int j = 0; j < SR; ++j) sh.P[wave][j][lane] = dA[j];
        float4 *mine = (float4 *)&sh.du[0][0];
        static_assert(sizeof(sh.du) >= sizeof(float4) * 8 * 16, "");
        // 64 rows of 8 pairs, 16 rows a turn
        __syncthreads();
        if (wave == 0)
#pragma unroll
            for (int j = 0; j < SR; ++j) {
                float s = sh.P[0][j][lane];
                for (int w = 1; w < kSelW; ++w) s += sh.P[w][j][lane];
                long long at;
                if (state_at<SR>(a, p, job0, row, ch, j, at)) dAp[at] = s;
            }
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int t = 0; t < 4; ++t) {
            __syncthreads();
            if (threadIdx.x / 128 == (unsigned)t) mine[threadIdx.x & 127] = make_float4(dDv[0], dDv[1], dbv[0], dbv[1]);
            __syncthreads();
            if (threadIdx.x < 8)
                for (int r = 0; r < 16; ++r) {
                    const float4 v = mine[r * 8 + threadIdx.x];
                    acc.x += v.x;
                    acc.y += v.y;
                    acc.z += v.z;
                    acc.w += v.w;
                }
        }
        const long long i = p.i0 + 2 * threadIdx.x;
        if (threadIdx.x < 8 && i < a.I) {
            float *to = dDp + (job0 * a.I + i) * 2;
            to[0] = acc.x;
            to[1] = acc.z;
            if (i + 1 < a.I) {
                to[2] = acc.y;
                to[3] = acc.w;
            }
        }
    }
}

// dB and dC [n] from the parts of the channel tiles, in their order.
template <typename T>
__global__ void __launch_bounds__(256)
k_sel_rows(long long n, int tiles, const float *dBp, const float *dCp, T *dB, T *dC)
{
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < n; e += (long long)gridDim.x * 256) {
        float b = 0.0f, c = 0.0f;
#pragma unroll 8
        for (int t = 0; t < tiles; ++t) {
            b += dBp[t * n + e];
            c += dCp[t * n + e];
        }
        Store<T>::store(dB, e, b);
        Store<T>::store(dC, e, c);
    }
}

// dA [I S], dD and ddelta_bias [I] from the jobs' parts, in 64 bits: 16 lanes an output.
__global__ void __launch_bounds__(256)
k_sel_weights(long long nA, long long I, int jobs, const float *dAp, const float *dDp, float *dA, float *dD, float *db)
{
    __shared__ double lds[16][16];
    const int o = threadIdx.x % 16, lane = threadIdx.x / 16;
    const long long at = (long long)blockIdx.x * 16 + o, nD = 2 * I;
    double s = 0.0;
    if (at < nA + nD)
        for (int j = lane; j < jobs; j += 16) s += (double)(at < nA ? dAp[j * nA + at] : dDp[j * nD + (at - nA)]);
    lds[lane][o] = s;
    __syncthreads();
    if (lane || at >= nA + nD) return;
    for (int l = 1; l < 16; ++l) s += lds[l][o];
    if (at < nA) {
        dA[at] = (float)s;
    } else {
        const long long i = (at - nA) / 2;
        if ((at - nA) & 1) {
            if (db) db[i] = (float)s;
        } else if (dD) {
            dD[i] = (float)s;
        }
    }
}

int check_sel(int64_t B, int64_t T, int64_t I, int32_t S, int32_t dtype)
{
    if (B < 1 || T < 1 || I < 1 || S < 1) return PLSTM_EINVAL;
    if (dtype != PLSTM_F32 && dtype != PLSTM_BF16) return PLSTM_EINVAL;
    if (S > kSelMaxS || B > (1LL << 30) || T > (1LL << 31) || I > (1LL << 30)) return PLSTM_EUNSUPPORTED;
    if (B > (1LL << 30) / I || T > (1LL << 38) / (B * I) || B * I > (1LL << 34) / S) return PLSTM_EUNSUPPORTED;
    // workgroups of a launch
    if (B * ((I + kSelCh - 1) / kSelCh) > (1LL << 22)) return PLSTM_EUNSUPPORTED;
    return PLSTM_OK;
}

// Workgroups that fill the card, and jobs that a backward call cuts its positions into.
constexpr long long kSelFill = 512, kSelJobs = 1024;

struct SelPlan {
    SelArgs a;
    int SR;
    float2 *fold;
    float *dBp, *dCp, *dAp, *dDp;
    size_t ws;
};

SelPlan sel_plan(int64_t B, int64_t T, int64_t I, int32_t S, int32_t reverse, int32_t softplus, int64_t pu, int64_t pd,
                 int64_t pz, int64_t pB, int64_t pC, const int32_t *lengths, void *ws, bool backward)
{
    SelPlan p{};
    SelArgs &a = p.a;
    p.SR = sel_sr(S);
    const long long tt = sel_tile(p.SR);
    a = SelArgs{B, T, I, S, reverse, softplus, pu ? pu : I, pd ? pd : I, pz ? pz : I, pB ? pB : S, pC ? pC : S, lengths,
                (I + kSelCh - 1) / kSelCh, (T + tt - 1) / tt, 1, a.chunk, 0};
    // Few channels and sequences do not fill the card: chunks of at least 4 tiles run at the same time, at the
    // price of folding all but one first
    const long long groups = B * a.tiles;
    long long chunks = groups * 2 <= kSelFill ? kSelFill / groups : 1;
    if (chunks > a.kept / 4) chunks = a.kept / 4;
    if (chunks < 1) chunks = 1;
    a.chunk = (a.kept + chunks - 1) / chunks * tt;
    a.chunks = (int)((T + a.chunk - 1) / a.chunk);
    const long long jobs = (kSelJobs + a.tiles - 1) / a.tiles;
    a.jobs = jobs < B * a.chunks ? jobs : B * a.chunks;
    Carve cv(ws);
    if (a.chunks > 1) p.fold = cv.take<float2>((size_t)a.chunks * B * I * S);
    if (backward) {
        if (a.tiles > 1) {
            p.dBp = cv.take<float>((size_t)a.tiles * B * T * S);
            p.dCp = cv.take<float>((size_t)a.tiles * B * T * S);
        }
        p.dAp = cv.take<float>((size_t)a.jobs * I * S);
        p.dDp = cv.take<float>((size_t)a.jobs * I * 2);
    }
    p.ws = align_up(cv.off, 256);
    if (p.ws < 256) p.ws = 256;
    return p;
}

bool sel_pitch(int64_t B, int64_t T, int64_t n, int64_t pitch)
{
    return pitch == 0 || (pitch >= n && pitch <= (1LL << 42) / (B * T));
}

template <typename T, int SR>
int sel_forward(const SelPlan &p, const T *u, const T *delta, const float *A, const T *Bm, const T *Cm, const float *D,
                const T *z, const float *dbias, const float *h0, T *y, float *hT, float *saved, hipStream_t st)
{
    const SelArgs &a = p.a;
    int launches = 1;
    if (a.chunks > 1) {
        k_sel_fwd<T, SR, true><<<(unsigned)(a.B * a.tiles * (a.chunks - 1)), kSelThreads, 0, st>>>(
            a, u, delta, A, Bm, Cm, D, z, dbias, h0, y, hT, saved, p.fold);
        PLSTM_LAUNCH_CHECK();
        ++launches;
    }
    k_sel_fwd<T, SR, false><<<(unsigned)(a.B * a.tiles * a.chunks), kSelThreads, 0, st>>>(
        a, u, delta, A, Bm, Cm, D, z, dbias, h0, y, hT, saved, p.fold);
    PLSTM_LAUNCH_CHECK();
    return launches;
}

template <typename T>
int sel_forward_any(const SelPlan &p, const void *u, const void *delta, const void *A, const void *Bm, const void *Cm,
                    const void *D, const void *z, const void *dbias, const void *h0, void *y, void *hT, void *saved,
                    hipStream_t st)
{
    const SelArgs &a = p.a;
    if (a.T == 1 && !saved) {
        const int L = a.S <= 4 ? 1 : a.S <= 8 ? 2 : a.S <= 16 ? 4 : a.S <= 32 ? 8 : 16;
        const unsigned blocks = (unsigned)((a.B * a.I * L + 255) / 256);
        const auto step = [&](auto l) {
            k_sel_step<T, decltype(l)::value><<<blocks, 256, 0, st>>>(
                a, (const T *)u, (const T *)delta, (const float *)A, (const T *)Bm, (const T *)Cm, (const float *)D,
                (const T *)z, (const float *)dbias, (const float *)h0, (T *)y, (float *)hT);
        };
        switch (L) {
        case 1: step(std::integral_constant<int, 1>()); break;
        case 2: step(std::integral_constant<int, 2>()); break;
        case 4: step(std::integral_constant<int, 4>()); break;
        case 8: step(std::integral_constant<int, 8>()); break;
        default: step(std::integral_constant<int, 16>()); break;
        }
        PLSTM_LAUNCH_CHECK();
        return 1;
    }
    const auto go = [&](auto sr) {
        return sel_forward<T, decltype(sr)::value>(p, (const T *)u, (const T *)delta, (const float *)A, (const T *)Bm,
                                                   (const T *)Cm, (const float *)D, (const T *)z, (const float *)dbias,
                                                   (const float *)h0, (T *)y, (float *)hT, (float *)saved, st);
    };
    switch (p.SR) {
    case 1: return go(std::integral_constant<int, 1>());
    case 2: return go(std::integral_constant<int, 2>());
    case 4: return go(std::integral_constant<int, 4>());
    case 8: return go(std::integral_constant<int, 8>());
    default: return go(std::integral_constant<int, 16>());
    }
}

struct SelGrads {
    void *du, *ddelta, *dA, *dB, *dC, *dD, *dz, *db, *dh0;
};

template <typename T, int SR>
int sel_backward(const SelPlan &p, const T *u, const T *delta, const float *A, const T *Bm, const T *Cm, const float *D,
                 const T *z, const float *dbias, const float *saved, const T *dy, const float *dhT, const SelGrads &g,
                 hipStream_t st)
{
    SelArgs a = p.a;
    int launches = 2;
    if (a.chunks > 1) {
        SelArgs f = a;
        f.jobs = a.B * (a.chunks - 1);
        k_sel_bwd<T, SR, true><<<(unsigned)(f.jobs * a.tiles), kSelThreads, 0, st>>>(
            f, u, delta, A, Bm, Cm, D, z, dbias, saved, dy, dhT, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr,
            nullptr, nullptr, nullptr, p.fold);
        PLSTM_LAUNCH_CHECK();
        ++launches;
    }
    k_sel_bwd<T, SR, false><<<(unsigned)(a.jobs * a.tiles), kSelThreads, 0, st>>>(
        a, u, delta, A, Bm, Cm, D, z, dbias, saved, dy, dhT, (T *)g.du, (T *)g.ddelta, (T *)g.dz, (float *)g.dh0, p.dBp,
        p.dCp, (T *)g.dB, (T *)g.dC, p.dAp, p.dDp, p.fold);
    PLSTM_LAUNCH_CHECK();
    if (a.tiles > 1) {
        const long long n = a.B * a.T * a.S;
        k_sel_rows<T><<<(unsigned)min((n + 255) / 256, 8192LL), 256, 0, st>>>(n, (int)a.tiles, p.dBp, p.dCp, (T *)g.dB,
                                                                              (T *)g.dC);
        PLSTM_LAUNCH_CHECK();
        ++launches;
    }
    const long long nA = a.I * a.S;
    k_sel_weights<<<(unsigned)((nA + 2 * a.I + 15) / 16), 256, 0, st>>>(nA, a.I, (int)a.jobs, p.dAp, p.dDp,
                                                                        (float *)g.dA, (float *)g.dD, (float *)g.db);
    PLSTM_LAUNCH_CHECK();
    return launches;
}

template <typename T>
int sel_backward_any(const SelPlan &p, const void *u, const void *delta, const void *A, const void *Bm, const void *Cm,
                     const void *D, const void *z, const void *dbias, const void *saved, const void *dy,
                     const void *dhT, const SelGrads &g, hipStream_t st)
{
    const auto go = [&](auto sr) {
        return sel_backward<T, decltype(sr)::value>(p, (const T *)u, (const T *)delta, (const float *)A, (const T *)Bm,
                                                    (const T *)Cm, (const float *)D, (const T *)z, (const float *)dbias,
                                                    (const float *)saved, (const T *)dy, (const float *)dhT, g, st);
    };
    switch (p.SR) {
    case 1: return go(std::integral_constant<int, 1>());
    case 2: return go(std::integral_constant<int, 2>());
    case 4: return go(std::integral_constant<int, 4>());
    case 8: return go(std::integral_constant<int, 8>());
    default: return go(std::integral_constant<int, 16>());
    }
}

}  // namespace
}  // namespace plstm

using namespace plstm;

extern "C" {

size_t pyramid_selective_scan_saved_size(int64_t B, int64_t T, int64_t I, int32_t S)
{
    if (check_sel(B, T, I, S, PLSTM_F32) != PLSTM_OK) return 0;
    const int64_t tt = sel_tile(sel_sr(S));
    return align_up((size_t)B * ((T + tt - 1) / tt) * I * S * sizeof(float), 256);
}

size_t pyramid_selective_scan_workspace_size(int64_t B, int64_t T, int64_t I, int32_t S, int32_t backward)
{
    if (check_sel(B, T, I, S, PLSTM_F32) != PLSTM_OK || (backward != 0 && backward != 1)) return 0;
    return sel_plan(B, T, I, S, 0, 0, 0, 0, 0, 0, 0, nullptr, nullptr, backward != 0).ws;
}

int pyramid_selective_scan_forward(int64_t B, int64_t T, int64_t I, int32_t S, int32_t dtype,
                                   int32_t reverse, int32_t softplus, const void *u, int64_t u_pitch,
                                   const void *delta, int64_t delta_pitch, const void *A,
                                   const void *Bm, int64_t B_pitch, const void *Cm, int64_t C_pitch,
                                   const void *D, const void *z, int64_t z_pitch,
                                   const void *delta_bias, const int32_t *lengths, const void *h0,
                                   void *y, void *hT, void *saved, void *ws, size_t ws_bytes,
                                   void *stream)
{
    const int rc = check_sel(B, T, I, S, dtype);
    if (rc != PLSTM_OK) return rc;
    if ((reverse != 0 && reverse != 1) || (softplus != 0 && softplus != 1) || !u || !delta || !A || !Bm || !Cm || !y || !ws)
        return PLSTM_EINVAL;
    if (!sel_pitch(B, T, I, u_pitch) || !sel_pitch(B, T, I, delta_pitch) || !sel_pitch(B, T, I, z_pitch) ||
        !sel_pitch(B, T, S, B_pitch) || !sel_pitch(B, T, S, C_pitch))
        return PLSTM_EINVAL;
    const size_t e = dtype_size(dtype);
    if (!aligned_to(u, e) || !aligned_to(delta, e) || !aligned_to(A, 4) || !aligned_to(Bm, e) || !aligned_to(Cm, e) ||
        !aligned_to(D, 4) || !aligned_to(z, e) || !aligned_to(delta_bias, 4) || !aligned_to(lengths, 4) ||
        !aligned_to(h0, 4) || !aligned_to(y, e) || !aligned_to(hT, 4) || !aligned_to(saved, 16) || !aligned_to(ws, 16))
        return PLSTM_EINVAL;
    if (ws_bytes < pyramid_selective_scan_workspace_size(B, T, I, S, 0)) return PLSTM_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const SelPlan p = sel_plan(B, T, I, S, reverse, softplus, u_pitch, delta_pitch, z_pitch, B_pitch, C_pitch, lengths,
                               ws, false);
    timing_begin("selective_fwd", st);
    const int n = (dtype == PLSTM_F32 ? sel_forward_any<float> : sel_forward_any<uint16_t>)(
        p, u, delta, A, Bm, Cm, D, z, delta_bias, h0, y, hT, saved, st);
    if (n < 0) return n;
    timing_end(n, st);
    return PLSTM_OK;
}

int pyramid_selective_scan_backward(int64_t B, int64_t T, int64_t I, int32_t S, int32_t dtype,
                                    int32_t reverse, int32_t softplus, const void *u, int64_t u_pitch,
                                    const void *delta, int64_t delta_pitch, const void *A,
                                    const void *Bm, int64_t B_pitch, const void *Cm, int64_t C_pitch,
                                    const void *D, const void *z, int64_t z_pitch,
                                    const void *delta_bias, const int32_t *lengths, const void *saved,
                                    const void *dy, const void *dhT, void *du, void *ddelta, void *dA,
                                    void *dB, void *dC, void *dD, void *dz, void *ddelta_bias,
                                    void *dh0, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = check_sel(B, T, I, S, dtype);
    if (rc != PLSTM_OK) return rc;
    if ((reverse != 0 && reverse != 1) || (softplus != 0 && softplus != 1) || !u || !delta || !A || !Bm || !Cm ||
        !saved || !dy || !du || !ddelta || !dA || !dB || !dC || !z != !dz || !ws)
        return PLSTM_EINVAL;
    if (!sel_pitch(B, T, I, u_pitch) || !sel_pitch(B, T, I, delta_pitch) || !sel_pitch(B, T, I, z_pitch) ||
        !sel_pitch(B, T, S, B_pitch) || !sel_pitch(B, T, S, C_pitch))
        return PLSTM_EINVAL;
    const size_t e = dtype_size(dtype);
    if (!aligned_to(u, e) || !aligned_to(delta, e) || !aligned_to(A, 4) || !aligned_to(Bm, e) || !aligned_to(Cm, e) ||
        !aligned_to(D, 4) || !aligned_to(z, e) || !aligned_to(delta_bias, 4) || !aligned_to(lengths, 4) ||
        !aligned_to(saved, 16) || !aligned_to(dy, e) || !aligned_to(dhT, 4) || !aligned_to(du, e) ||
        !aligned_to(ddelta, e) || !aligned_to(dA, 4) || !aligned_to(dB, e) || !aligned_to(dC, e) || !aligned_to(dD, 4) ||
        !aligned_to(dz, e) || !aligned_to(ddelta_bias, 4) || !aligned_to(dh0, 4) || !aligned_to(ws, 16))
        return PLSTM_EINVAL;
    if (ws_bytes < pyramid_selective_scan_workspace_size(B, T, I, S, 1)) return PLSTM_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const SelPlan p = sel_plan(B, T, I, S, reverse, softplus, u_pitch, delta_pitch, z_pitch, B_pitch, C_pitch, lengths,
                               ws, true);
    const SelGrads g{du, ddelta, dA, dB, dC, dD, dz, ddelta_bias, dh0};
    timing_begin("selective_bwd", st);
    const int n = (dtype == PLSTM_F32 ? sel_backward_any<float> : sel_backward_any<uint16_t>)(
        p, u, delta, A, Bm, Cm, D, z, delta_bias, saved, dy, dhT, g, st);
    if (n < 0) return n;
    timing_end(n, st);
    return PLSTM_OK;
}

}  // extern "C"
