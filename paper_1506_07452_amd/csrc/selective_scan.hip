// Selective state space scan along an axis, and its backward pass.  Over sweep positions s
// (sequence.h), for channel i and state k, d = delta + bias (of it the softplus, if asked):
//   a = exp(d A[i][k]),  h_s = a h_{s-1} + d u B_s[k],  p_s = sum_k C_s[k] h_s + D u,  y = p silu(z)
// Backward, dp = dy silu(z) and G_s the gradient of h_s:
//   G_s = C_s dp_s + a_{s+1} G_{s+1}  (the last one takes dhT as well),  dh0 = a_0 G_0
//   dC = sum_i dp h,  dB = sum_i G d u,  q = sum_k G B,  w = sum_k G a h_{s-1} A
//   du = d q + D dp,  dd = u q + w,  dA = sum G a h_{s-1} d,  dD = sum dp u,  dz = dy p silu'(z)
// A wave walks a piece of a sequence by itself.  Its four rows of 16 lanes have a quarter of the
// states each (SR of them), the lanes of a row CL channels each, so a lane has CL SR states in registers
// and the rows of B and C that it reads from LDS serve all its channels.  What belongs to an element and
// not to its states (softplus, d u, the gate) is made once, by the lane whose row the element's sum
// over the states comes out in, and passes to the other rows through LDS.
// Few channels and long sequences do not fill the card: a sequence is then cut into chunks whose
// folds (last state = exp(A sum d) h + H) are made first and chained by a small launch.
// Bound by the issue of vector instructions, not by bytes: a state and position take an exponential (the time of 3.2 products),
// 4 products in the forward, 3 in a fold; the backward 29 instructions (11 for the formulas, half of the states again, 5.5 for
// the sums over channels, 3 a state for what belongs to an element).  16 states, bf16, 2 x 4096 x 2048: forward 76 us (its bytes
// 26), folds 51 and 59, backward 289 (bytes 46), the vector units busy 80 to 87%.  The whole MR volume along x (11520 x 240 x 16
// fp32), no folds: forward 231 us, at the rate of its bytes; backward 738.
#include <algorithm>

#include "sequence.h"
#include "timing.h"

namespace plstm {
namespace {

constexpr int kSelMaxS = 64;
// Positions between the states that a training forward keeps: those that a backward wave has in LDS at a time.  Kept states are S / 4 bytes
// an element, written and read: 16 states 4, as much as two bf16 inputs; 64 states 16, more than all of them.
constexpr int kSelKeep = 16;
constexpr int kSelStage = 8;            // positions that a forward wave stages at a time
constexpr float kLog2e = 1.44269504f, kLn2 = 0.69314718f;

inline int sel_sr(int S) { return S <= 4 ? 1 : S <= 8 ? 2 : S <= 16 ? 4 : S <= 32 ? 8 : 16; }
// Channels of a lane in the forward and the folds: two share the rows of B and C that a lane reads (forward and backward, 2 x 4096 x
// 2048 501 us, with one 507; 1 x 16384 x 1024 145, 148; sequences too short to fill the card lose by it, 1 x 1024 x 512 67, 64).
__host__ __device__ constexpr int sel_cl(int SR) { return SR <= 4 ? 2 : 1; }

struct SelArgs {
    long long B, T, I;
    int S, reverse, softplus;
    long long pu, pd, pz, pB, pC;       // elements from one row to the next
    const int32_t *lengths;
    long long tiles;                    // waves across a sequence's channels
    long long groups;                   // waves across all channels and sequences
    long long kept;                     // states that a sequence keeps
    int chunks;                         // of a sequence, each with waves of its own
    long long chunk;                    // positions of a chunk (a multiple of kSelKeep)
    long long jobs;                     // backward: sequences' chunks that run at the same time
};

// One or two elements from any element on, raw.
template <typename T, int N> struct Few;
// A value in the storage type, by the conversion instruction.
__device__ inline void put_one(float *p, float v) { *p = v; }
__device__ inline void put_one(uint16_t *p, float v) { *p = (uint16_t)pack_bf16(v, v); }

template <typename T> struct Few<T, 1> {
    typedef T V;
    T w;
    __device__ void load(const T *p, int have) { w = have > 0 ? *p : (T)0; }
    __device__ void set(V v) { w = v; }
    __device__ float get(int) const { return Store<T>::load(&w, 0); }
    __device__ static void store(T *p, int have, const float *v)
    {
        if (have > 0) put_one(p, *v);
    }
};
template <> struct Few<float, 2> {
    typedef uint32_t V __attribute__((ext_vector_type(2), aligned(4)));
    uint32_t w[2];
    __device__ void set(V v)
    {
        w[0] = v[0];
        w[1] = v[1];
    }
    __device__ void load(const float *p, int have)
    {
        w[0] = w[1] = 0;
        if (have >= 2) {
            const V r = *(const V *)p;
            w[0] = r[0];
            w[1] = r[1];
        } else if (have == 1) {
            w[0] = float_bits(*p);
        }
    }
    __device__ float get(int e) const { return bits_float(w[e]); }
    __device__ static void store(float *p, int have, const float *v)
    {
        if (have >= 2) *(V *)p = V{float_bits(v[0]), float_bits(v[1])};
        else if (have == 1) *p = v[0];
    }
};
template <> struct Few<uint16_t, 2> {
    typedef uint32_t V __attribute__((aligned(2)));
    uint32_t w;
    __device__ void set(V v) { w = v; }
    __device__ void load(const uint16_t *p, int have)
    {
        w = 0;
        if (have >= 2) w = *(const V *)p;
        else if (have == 1) w = *p;
    }
    __device__ float get(int e) const { return bits_float(e ? w & 0xffff0000u : w << 16); }
    __device__ static void store(uint16_t *p, int have, const float *v)
    {
        if (have >= 2) *(V *)p = pack_bf16(v[0], v[1]);
        else if (have == 1) *p = (uint16_t)pack_bf16(v[0], v[0]);
    }
};

// A log2(e), of which a step's exponent is a multiple; within 2^100.  A of minus infinity (a state that forgets at once) times the 0 of
// a step that a sequence does not have is to be 0; so large a number forgets in all steps of over 2^-92, and leaves what a
// gradient times it is a number.
__device__ inline float exponent_of(float A)
{
    const float v = A * kLog2e, most = 1.2676506e30f;
    return v < -most ? -most : v > most ? most : v;         // a NaN stays one
}

// log(1 + exp(v)).  With e = exp(-|v|) and w = 1 + e rounded, log(1 + e) is log(w) and to first order what w has
// lost, e - (w - 1), over w: left out, as what is lost is below 2^-24 and w is 1 where log(w) is small.
__device__ inline float softplus_of(float v)
{
    const float e = __builtin_amdgcn_exp2f(fabsf(v) * -kLog2e), w = 1.0f + e;
    return fmaf(__builtin_amdgcn_logf(w), kLn2, e - (w - 1.0f)) + fmaxf(v, 0.0f);
}

// And its derivative, sigmoid(v), from the same exponential.
__device__ inline float softplus_slope(float v, float &slope)
{
    const float e = __builtin_amdgcn_exp2f(fabsf(v) * -kLog2e), w = 1.0f + e;
    slope = __builtin_amdgcn_rcpf(w) * (v < 0.0f ? e : 1.0f);
    return fmaf(__builtin_amdgcn_logf(w), kLn2, e - (w - 1.0f)) + fmaxf(v, 0.0f);
}

// Sum over the four rows of 16 lanes (a channel's quarters of states) of 4 Q values: lane (row,
// channel) gets that of value 4 q + row_value(row) in v[q].  Two swaps of half waves, one of rows and
// three additions make four sums.
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
template <int Q>
__device__ inline void sum_states(float *v)
{
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        float *x = v + 4 * q;
        swap32(x[0], x[1]);
        swap32(x[2], x[3]);
        float s = x[0] + x[1], t = x[2] + x[3];
        swap16(s, t);
        v[q] = s + t;
    }
}
__device__ inline int row_value(int row) { return (row & 1) << 1 | row >> 1; }

// Sums over the 16 lanes of a row of four values: the lanes of the row's k-th four get that of value
// four_value(k).  Mirrored lanes are added and two sums put into one register by halves, then by quarters.
template <int BANKS>
__device__ inline float banks_of(float a, float b)      // b in those fours of lanes, a in the others
{
    return bits_float((uint32_t)__builtin_amdgcn_update_dpp((int)float_bits(a), (int)float_bits(b), 0xe4, 0xf, BANKS, false));
}
template <int CTRL>
__device__ inline float plus_moved(float v)
{
#pragma clang fp contract(off)          // one addition of a moved lane, not a move and a fused product
    return v + bits_float(moved<CTRL>(float_bits(v)));
}
__device__ inline float sum_four(float a, float b, float c, float d)
{
    const float x = banks_of<0xc>(plus_moved<0x140>(a), plus_moved<0x140>(b));
    const float y = banks_of<0xc>(plus_moved<0x140>(c), plus_moved<0x140>(d));
    float v = banks_of<0xa>(plus_moved<0x141>(x), plus_moved<0x141>(y));
    v = plus_moved<0xb1>(v);
    return plus_moved<0x4e>(v);
}
__device__ inline int four_value(int k) { return (k & 1) << 1 | k >> 1; }

// The value is made here: its operands' registers end here and not where it is used.
__device__ inline void made(float &v) { asm volatile("" : "+v"(v)); }

// LDS that only one wave uses: its accesses are in order, the compiler has to leave them so.
__device__ inline void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The wave's number in its workgroup, in a scalar register: what follows from it is the same for all lanes.
__device__ inline int wave_number() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64); }

// Workgroups of neighbouring channels share lines of their rows: those of an XCD (every
// eighth) are given consecutive numbers.
__device__ inline long long spread(long long id, long long all)
{
    const long long each = all / 8, rest = all - each * 8, x = id & 7;
    return (x < rest ? x * (each + 1) : rest * (each + 1) + (x - rest) * each) + (id >> 3);
}

// A lane's sequence and channels.
struct Lane {
    long long b, n, i;                  // sequence, its length, first channel
    int have;                           // channels that there are (0: an idle lane, which stands on the first)
    // row of position s, the padding's as well
    __device__ long long row(const SelArgs &a, long long s) const { return b * a.T + step_of(s, n, a.reverse); }
};

template <int CL>
__device__ inline Lane lane_of(const SelArgs &a, long long b, long long i)
{
    Lane l;
    l.b = b < a.B ? b : a.B - 1;
    l.n = length_of(a.lengths, l.b, a.T);
    l.i = i < a.I ? i : 0;
    l.have = b < a.B && i < a.I ? (int)min(a.I - i, (long long)CL) : 0;
    return l;
}

// A lane's element of a tensor at position s + r, r < SPAN its own: a scalar address that s decides and the
// lane's 32-bit offset from it (the host keeps rows short enough).
template <typename T, int SPAN>
struct Walk {
    const char *base;                   // of the wave: position 0 of sequence b0 (in reverse the last one's row below)
    long long step;                     // bytes from a position to the next
    uint32_t off;
    __device__ void init(const SelArgs &a, const T *x, long long pitch, long long b0, const Lane &l, int r, long long i)
    {
        const long long n0 = length_of(a.lengths, b0, a.T);
        const long long row = (l.b - b0) * a.T + (a.reverse ? l.n - n0 + SPAN - 1 - r : r);
        base = (const char *)x + (b0 * a.T + (a.reverse ? n0 - SPAN : 0)) * pitch * (long long)sizeof(T);
        step = (a.reverse ? -pitch : pitch) * (long long)sizeof(T);
        off = (uint32_t)((row * pitch + i) * (long long)sizeof(T));
    }
    __device__ char *at(long long s) const { return (char *)base + s * step; }
    // whole: there is no other case for any lane
    template <int N> __device__ void load(Few<T, N> &v, long long s, bool whole, int have) const
    {
        const char *p = at(s);
        if (whole) v.set(*(const typename Few<T, N>::V *)(p + off));
        else v.load((const T *)(p + off), have);
    }
};

// SR states from `row` SR on of a channel in an array [..][S]; have: of them that there are.
template <int SR>
__device__ inline int states_have(const SelArgs &a, int row, bool lane)
{
    const int left = a.S - row * SR;
    return !lane || left <= 0 ? 0 : left < SR ? left : SR;
}
template <int SR>
__device__ inline void load_states(const float *p, int have, float *v)
{
    if constexpr (SR >= 4) {
#pragma unroll
        for (int j = 0; j < SR; j += 4) Piece<float>::unpack(load_piece<float>(p + j, have - j < 4 ? have - j : 4), v + j);
    } else {
#pragma unroll
        for (int j = 0; j < SR; ++j) v[j] = j < have ? p[j] : 0.0f;
    }
}
template <int SR>
__device__ inline void store_states(float *p, int have, const float *v)
{
    if constexpr (SR >= 4) {
#pragma unroll
        for (int j = 0; j < SR; j += 4)
            if (have - j > 0) store_piece<float>(p + j, have - j < 4 ? have - j : 4, v + j);
    } else {
#pragma unroll
        for (int j = 0; j < SR; ++j)
            if (j < have) p[j] = v[j];
    }
}

// A lane's states of a row of B or C in LDS, in one access for each four.
template <int SR>
__device__ inline void row_states(const float *p, float *v)
{
    if constexpr (SR >= 4) {
#pragma unroll
        for (int j = 0; j < SR; j += 4) {
            const float4 w = *(const float4 *)(p + j);
            v[j] = w.x;
            v[j + 1] = w.y;
            v[j + 2] = w.z;
            v[j + 3] = w.w;
        }
    } else if constexpr (SR == 2) {
        const float2 w = *(const float2 *)p;
        v[0] = w.x;
        v[1] = w.y;
    } else {
        v[0] = *p;
    }
}

__device__ inline float step_size(const SelArgs &a, float raw, float bias, bool live)
{
    const float v = raw + bias;
    return live ? (a.softplus ? softplus_of(v) : v) : 0.0f;
}

// Two values each of rows of B or C (4 SR of them, the last ones 0) of R positions of NB sequences,
// by the lanes of a wave, ROWS positions a pass.
template <typename T, int SR, int R, int NB>
struct StateRows {
    static constexpr int SP = 4 * SR, PP = NB * SP / 2;
    static constexpr int ROWS = 64 / PP < R ? 64 / PP : R, Q = R / ROWS;
    static_assert(PP <= 64 && Q * ROWS == R, "a pass takes whole rows");
    Walk<T, ROWS> walk;
    int r, to, want;                    // the lane's position, place in a row of LDS, values that there are
    long long n;
    Few<T, 2> raw[Q];
    __device__ void init(const SelArgs &a, const T *p, long long pitch, long long b0, int lane)
    {
        r = min(lane / PP, ROWS - 1);
        const int at = lane % PP, seq = at / (SP / 2), k = at % (SP / 2) * 2;
        const Lane l = lane_of<1>(a, b0 + seq, 0);
        n = b0 + seq < a.B ? l.n : 0;
        to = seq * SP + k;
        want = k + 1 < a.S ? 2 : k < a.S ? 1 : 0;
        walk.init(a, p, pitch, b0, l, r, want ? k : 0);
    }
    __device__ void load(long long s0, long long last, bool whole)
    {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const long long s = s0 + q * ROWS;
            walk.load(raw[q], s, whole, s + r < last && s + r < n ? want : 0);
        }
    }
    __device__ void put(float (*rows)[NB * SP]) const
    {
#pragma unroll
        for (int q = 0; q < Q; ++q)
            *(float2 *)&rows[q * ROWS + r][to] = make_float2(want > 0 ? raw[q].get(0) : 0.0f, want > 1 ? raw[q].get(1) : 0.0f);
    }
};

// Positions that all sequences of a wave have, and whether its lanes load whole pieces there.
template <int CL, int NB>
__device__ inline long long whole_until(const SelArgs &a, long long b0, long long last)
{
    if ((CL > 1 && a.I % CL) || a.S % 2) return 0;
    long long n = last;
#pragma unroll
    for (int q = 0; q < NB; ++q)
        if (b0 + q < a.B) n = min(n, length_of(a.lengths, b0 + q, a.T));
    return n;
}

// What a wave stages: d and d u (the backward fold: d and dp) of its elements, rows of B and C.
template <int SR, int CL, int NB>
struct alignas(16) ForwardShared {
    float du[kSelStage][16][2 * CL];
    float B[kSelStage][NB * 4 * SR], C[kSelStage][NB * 4 * SR];
};

// Where a wave of the forward or a fold is: NB sequences share it where 16 / NB lanes have all
// their channels.
template <int CL, int NB>
__device__ inline void wave_place(const SelArgs &a, long long id, int lane, Lane &l, long long &b0, int &chunk)
{
    const long long g = id % a.groups;
    chunk = (int)(id / a.groups);
    const int p = lane & 15;
    if (NB == 1) {
        b0 = g / a.tiles;
        l = lane_of<CL>(a, b0, ((g - b0 * a.tiles) * 16 + p) * CL);
    } else {
        b0 = g * NB;
        l = lane_of<CL>(a, b0 + p / (16 / NB), p % (16 / NB) * CL);
    }
}

template <typename T, int SR, int CL, int NB>
__global__ void __launch_bounds__(256)
k_sel_fwd(SelArgs a, const T *u, const T *delta, const float *A, const T *Bm, const T *Cm, const float *D,
          const T *z, const float *dbias, const float *h0, T *y, float *hT, float *saved, const float *start)
{
    constexpr int R = kSelStage, K = R / 4, SP = 4 * SR;
    __shared__ ForwardShared<SR, CL, NB> shared[4];
    const int lane = threadIdx.x & 63, row = lane >> 4, p = lane & 15, rv = row_value(row);
    const int wave = wave_number();
    const long long id = spread(blockIdx.x, gridDim.x) * 4 + wave;
    if (id >= a.groups * a.chunks) return;
    ForwardShared<SR, CL, NB> &sh = shared[wave];
    Lane l;
    long long b0;
    int chunk;
    wave_place<CL, NB>(a, id, lane, l, b0, chunk);
    const long long first = chunk * a.chunk, last = min(a.T, first + a.chunk);
    const int seq = NB == 1 ? 0 : p / (16 / NB);
    float A2[CL][SR], h[CL][SR], bias[CL], Dv[CL];
#pragma unroll
    for (int c = 0; c < CL; ++c) {
        const int have = states_have<SR>(a, row, c < l.have);
        const long long at = (l.b * a.I + l.i + c) * a.S + row * SR;
        load_states<SR>(A + (l.i + c) * a.S + row * SR, have, A2[c]);
        const float *from = a.chunks > 1 ? start + chunk * a.B * a.I * a.S : h0;
        load_states<SR>(from + at, from ? have : 0, h[c]);
#pragma unroll
        for (int j = 0; j < SR; ++j) A2[c][j] = exponent_of(A2[c][j]);
        bias[c] = dbias && c < l.have ? dbias[l.i + c] : 0.0f;
        Dv[c] = D && c < l.have ? D[l.i + c] : 0.0f;
    }
    Walk<T, 4> wu, wd, wz, wy;
    wu.init(a, u, a.pu, b0, l, rv, l.i);
    wd.init(a, delta, a.pd, b0, l, rv, l.i);
    if (z) wz.init(a, z, a.pz, b0, l, rv, l.i);
    wy.init(a, y, a.I, b0, l, rv, l.i);
    StateRows<T, SR, R, NB> rB, rC;
    rB.init(a, Bm, a.pB, b0, lane);
    rC.init(a, Cm, a.pC, b0, lane);
    const long long whole = whole_until<CL, NB>(a, b0, last);
    Few<T, CL> ru[K], rd[K], rz[K];
    const auto fetch_as = [&](long long s0, auto all) {
        constexpr bool W = decltype(all)::value;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const long long s = s0 + 4 * k;
            const int have = !W && s + rv < last && s + rv < l.n ? l.have : 0;
            wu.load(ru[k], s, W, have);
            wd.load(rd[k], s, W, have);
            if (z) wz.load(rz[k], s, W, have);
        }
        rB.load(s0, last, W);
        rC.load(s0, last, W);
    };
    const auto fetch = [&](long long s0) {
        if (s0 + R <= whole) fetch_as(s0, std::true_type());
        else fetch_as(s0, std::false_type());
    };
    fetch(first);
    for (long long s0 = first; s0 < last; s0 += R) {
        float uv[K][CL], zv[K][CL];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool live = s0 + 4 * k + rv < l.n;
            float v[2 * CL];
#pragma unroll
            for (int c = 0; c < CL; ++c) {
                uv[k][c] = ru[k].get(c);
                zv[k][c] = z ? rz[k].get(c) : 0.0f;
                v[2 * c] = step_size(a, rd[k].get(c), bias[c], live);
                v[2 * c + 1] = v[2 * c] * uv[k][c];
            }
            if constexpr (CL == 2) *(float4 *)&sh.du[4 * k + rv][p][0] = make_float4(v[0], v[1], v[2], v[3]);
            else *(float2 *)&sh.du[4 * k + rv][p][0] = make_float2(v[0], v[1]);
        }
        rB.put(sh.B);
        rC.put(sh.C);
        wave_sync();
        if (s0 + R < last) fetch(s0 + R);
        if (saved && s0 % kSelKeep == 0)
#pragma unroll
            for (int c = 0; c < CL; ++c)
                store_states<SR>(saved + ((l.b * a.kept + s0 / kSelKeep) * a.I + l.i + c) * a.S + row * SR,
                                 states_have<SR>(a, row, c < l.have), h[c]);
        float yp[CL][R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float v[2 * CL], Bv[SR], Cv[SR];
#pragma unroll
            for (int e = 0; e < 2 * CL; ++e) v[e] = sh.du[r][p][e];
            row_states<SR>(&sh.B[r][seq * SP + row * SR], Bv);
            row_states<SR>(&sh.C[r][seq * SP + row * SR], Cv);
#pragma unroll
            for (int c = 0; c < CL; ++c) {
                yp[c][r] = 0.0f;
#pragma unroll
                for (int j = 0; j < SR; ++j) {
                    const float dec = __builtin_amdgcn_exp2f(v[2 * c] * A2[c][j]);
                    h[c][j] = fmaf(dec, h[c][j], v[2 * c + 1] * Bv[j]);
                    yp[c][r] = fmaf(Cv[j], h[c][j], yp[c][r]);
                }
            }
        }
#pragma unroll
        for (int c = 0; c < CL; ++c) sum_states<K>(yp[c]);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const long long s = s0 + 4 * k + rv;
            float v[CL];
#pragma unroll
            for (int c = 0; c < CL; ++c) {
                v[c] = fmaf(Dv[c], uv[k][c], yp[c][k]);
                if (z) v[c] *= zv[k][c] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(zv[k][c] * -kLog2e));
                v[c] = s < l.n ? v[c] : 0.0f;
            }
            if (s0 + R <= whole) {
                if (l.have) Few<T, CL>::store((T *)(wy.at(s0 + 4 * k) + wy.off), CL, v);
            } else if (s < last) {
                Few<T, CL>::store(y + l.row(a, s) * a.I + l.i, l.have, v);
            }
        }
        wave_sync();
    }
    if (hT && chunk == a.chunks - 1)
#pragma unroll
        for (int c = 0; c < CL; ++c)
            store_states<SR>(hT + (l.b * a.I + l.i + c) * a.S + row * SR, states_have<SR>(a, row, c < l.have), h[c]);
}

// Folds of chunks: sums of d [chunk][b][i], and what a chunk makes of nothing, its last state or
// (BACK) the gradient that it passes on: H [chunk][b][i][k].
template <typename T, int SR, int CL, int NB, bool BACK>
__global__ void __launch_bounds__(256)
k_sel_fold(SelArgs a, const T *u, const T *delta, const float *A, const T *rows, long long pitch, const T *z,
           const T *dy, const float *dbias, float *H, float *sums)
{
    constexpr int R = kSelStage, K = R / 4, SP = 4 * SR;
    __shared__ ForwardShared<SR, CL, NB> shared[4];
    const int lane = threadIdx.x & 63, row = lane >> 4, p = lane & 15, rv = row_value(row);
    const int wave = wave_number();
    const long long id = spread(blockIdx.x, gridDim.x) * 4 + wave;
    if (id >= a.groups * (a.chunks - 1)) return;
    ForwardShared<SR, CL, NB> &sh = shared[wave];
    Lane l;
    long long b0;
    int chunk;
    wave_place<CL, NB>(a, id, lane, l, b0, chunk);
    chunk += BACK ? 1 : 0;
    const long long first = chunk * a.chunk, last = min(a.T, first + a.chunk);
    const int seq = NB == 1 ? 0 : p / (16 / NB);
    float A2[CL][SR], h[CL][SR], bias[CL], sum[CL];
#pragma unroll
    for (int c = 0; c < CL; ++c) {
        load_states<SR>(A + (l.i + c) * a.S + row * SR, states_have<SR>(a, row, c < l.have), A2[c]);
#pragma unroll
        for (int j = 0; j < SR; ++j) {
            A2[c][j] = exponent_of(A2[c][j]);
            h[c][j] = 0.0f;
        }
        bias[c] = dbias && c < l.have ? dbias[l.i + c] : 0.0f;
        sum[c] = 0.0f;
    }
    Walk<T, 4> wu, wd, wz;              // BACK: dy in the place of u
    wu.init(a, BACK ? dy : u, BACK ? a.I : a.pu, b0, l, rv, l.i);
    wd.init(a, delta, a.pd, b0, l, rv, l.i);
    if (BACK && z) wz.init(a, z, a.pz, b0, l, rv, l.i);
    StateRows<T, SR, R, NB> rB;
    rB.init(a, rows, pitch, b0, lane);
    const long long whole = whole_until<CL, NB>(a, b0, last);
    Few<T, CL> ru[K], rd[K], rz[K];
    const auto fetch_as = [&](long long s0, auto all) {
        constexpr bool W = decltype(all)::value;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const long long s = s0 + 4 * k;
            const int have = !W && s + rv < last && s + rv < l.n ? l.have : 0;
            wu.load(ru[k], s, W, have);
            wd.load(rd[k], s, W, have);
            if (BACK && z) wz.load(rz[k], s, W, have);
        }
        rB.load(s0, last, W);
    };
    const auto fetch = [&](long long s0) {
        if (s0 + R <= whole) fetch_as(s0, std::true_type());
        else fetch_as(s0, std::false_type());
    };
    const long long stages = (last - first + R - 1) / R;
    fetch(BACK ? first + (stages - 1) * R : first);
    for (long long st = 0; st < stages; ++st) {
        const long long s0 = first + (BACK ? stages - 1 - st : st) * R;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool live = s0 + 4 * k + rv < min(l.n, last);
            float v[2 * CL];
#pragma unroll
            for (int c = 0; c < CL; ++c) {
                v[2 * c] = step_size(a, rd[k].get(c), bias[c], live);
                const float x = ru[k].get(c);
                v[2 * c + 1] = BACK ? (z ? x * silu_of(rz[k].get(c)) : x) : v[2 * c] * x;
            }
            if constexpr (CL == 2) *(float4 *)&sh.du[4 * k + rv][p][0] = make_float4(v[0], v[1], v[2], v[3]);
            else *(float2 *)&sh.du[4 * k + rv][p][0] = make_float2(v[0], v[1]);
        }
        rB.put(sh.B);
        wave_sync();
        if (st + 1 < stages) fetch(BACK ? s0 - R : s0 + R);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const int r = BACK ? R - 1 - q : q;
            float v[2 * CL], Bv[SR];
#pragma unroll
            for (int e = 0; e < 2 * CL; ++e) v[e] = sh.du[r][p][e];
            row_states<SR>(&sh.B[r][seq * SP + row * SR], Bv);
#pragma unroll
            for (int c = 0; c < CL; ++c) {
                sum[c] += v[2 * c];
#pragma unroll
                for (int j = 0; j < SR; ++j) {
                    const float dec = __builtin_amdgcn_exp2f(v[2 * c] * A2[c][j]);
                    if (BACK) h[c][j] = dec * fmaf(v[2 * c + 1], Bv[j], h[c][j]);
                    else h[c][j] = fmaf(dec, h[c][j], v[2 * c + 1] * Bv[j]);
                }
            }
        }
        wave_sync();
    }
    const long long cols = a.B * a.I;
#pragma unroll
    for (int c = 0; c < CL; ++c) {
        const long long at = chunk * cols + l.b * a.I + l.i + c;
        store_states<SR>(H + at * a.S + row * SR, states_have<SR>(a, row, c < l.have), h[c]);
        if (row == 0 && c < l.have) sums[at] = sum[c];
    }
}

// The state before each chunk (BACK: the gradient behind each), from h0 (dhT) on, in the place of H.
template <bool BACK>
__global__ void __launch_bounds__(256)
k_sel_chain(long long cols, long long I, int S, int chunks, const float *A, const float *from, float *H, const float *sums)
{
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, col = at / S, states = cols * S;
    if (at >= states) return;
    const float A2 = exponent_of(A[col % I * S + (at - col * S)]);
    float h = from ? from[at] : 0.0f;
    constexpr int U = 16;
    for (int n = 0; n < chunks; n += U) {
        float x[U], s[U];
#pragma unroll
        for (int e = 0; e < U; ++e) {
            const int c = BACK ? chunks - 1 - n - e : n + e;
            const bool has = n + e + 1 < chunks;        // the last one passes nothing on
            x[e] = has ? H[c * states + at] : 0.0f;
            s[e] = has ? sums[c * cols + col] : 0.0f;
        }
        loads_issued();
#pragma unroll
        for (int e = 0; e < U; ++e) {
            if (n + e >= chunks) break;
            H[(BACK ? chunks - 1 - n - e : n + e) * states + at] = h;
            // whole powers of 2 apart: the product may be a number where a chunk's growth alone is none
            const float p = fminf(fmaxf(s[e] * A2, -1e6f), 1e6f), whole = rintf(p);
            h = ldexpf(h * __builtin_amdgcn_exp2f(p - whole), (int)whole) + x[e];
        }
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
            h[j] = fmaf(__builtin_amdgcn_exp2f(d * exponent_of(Av[j])), h[j], d * uv * Bv[j]);
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

// Positions of a run of the backward, whose decays and states a lane has in registers: half of the states are made twice with 8
// of them, three quarters with 4 (2 x 4096 x 2048, 16 states: 310 us, 355).
__host__ __device__ constexpr int sel_run(int SR) { return SR <= 4 ? 8 : 4; }

template <int SR>
struct alignas(16) BackShared {
    static constexpr int SP = 4 * SR, R = sel_run(SR), NR = kSelKeep / R;
    float2 du[kSelKeep][16];            // d, d u
    float2 own[kSelKeep][16];           // u, the derivative of d: what its own lane takes back
    float dp[kSelKeep][16], slope[kSelKeep][16];        // slope: dy silu'(z)
    float B[kSelKeep][SP], C[kSelKeep][SP];
    float start[NR][SR][64];            // the state before each run
    float out[2][2][R][SP];             // a run's dB and dC, by turns
};

// Walks chunks from their ends, kSelKeep positions at a time: the states before the runs from the kept one,
// then run by run, from the last on, the states in it and back.  WIDE: the waves of a workgroup have neighbouring channels of
// the same chunk and add up their dB and dC; else each has the only 16 channels of a sequence of its own.
// dBp, dCp [group of channels][b][t][S] (one group: dB and dC themselves); dAp [job][I][S], dDp [job][I][2].
// Two waves a SIMD; 16 states a lane have the registers of one (64 states, 2 x 2048 x 2048 bf16: 785 us, with two and spills 1202).
template <typename T, int SR, bool WIDE>
__global__ void __launch_bounds__(256, SR <= 8 ? 2 : 1)
k_sel_bwd(SelArgs a, const T *u, const T *delta, const float *A, const T *Bm, const T *Cm, const float *D, const T *z,
          const float *dbias, const float *saved, const T *dy, const float *dhT, const float *behind, T *du, T *ddelta,
          T *dz, float *dh0, float *dBp, float *dCp, T *dB, T *dC, float *dAp, float *dDp)
{
    constexpr int R = sel_run(SR), NR = kSelKeep / R, K = R / 4, SP = 4 * SR;
    extern __shared__ float4 dyn[];
    BackShared<SR> *shared = (BackShared<SR> *)dyn;
    const int wave = wave_number(), waves = blockDim.x / 64;
    const int lane = threadIdx.x & 63, row = lane >> 4, ch = lane & 15, rv = row_value(row), fv = four_value(ch >> 2);
    BackShared<SR> &sh = shared[wave];
    const long long id = spread(blockIdx.x, gridDim.x), wide = (a.tiles + waves - 1) / waves;
    const long long group = WIDE ? id % wide : 0, job0 = WIDE ? id / wide : id * waves + wave;
    const long long i = (WIDE ? group * waves + wave : 0) * 16 + ch;
    const bool has = i < a.I;
    const long long ic = has ? i : 0;
    const int have = states_have<SR>(a, row, has);
    // sums over the steps: of a block in 32 bits, of blocks in 64
    float A2[SR], dA[SR], dDv = 0.0f, dbv = 0.0f;
    double dAs[SR], dDs = 0.0, dbs = 0.0;
    load_states<SR>(A + ic * a.S + row * SR, have, A2);
#pragma unroll
    for (int j = 0; j < SR; ++j) {
        A2[j] = exponent_of(A2[j]);
        dA[j] = 0.0f;
        dAs[j] = 0.0;
    }
    const float bias = dbias && has ? dbias[i] : 0.0f, Dv = D && has ? D[i] : 0.0f;
    if (!WIDE && job0 >= a.jobs) return;
    // element (dB or dC, position, state) of a run's sums that a thread takes where there are no more than threads: from the
    // run's first row, -1 without one
    const int oe = WIDE ? (int)threadIdx.x : lane, orow = oe / SP % R, ok = oe % SP;
    const int out_off = oe < 2 * R * SP && ok < a.S ? (a.reverse ? R - 1 - orow : orow) * a.S + ok : -1;
    for (long long job = job0; job < a.B * a.chunks; job += a.jobs) {
        const long long b = job / a.chunks;
        const int chunk = (int)(job - b * a.chunks);
        const long long first = chunk * a.chunk, last = min(a.T, first + a.chunk);
        Lane l = lane_of<1>(a, b, ic);
        l.have = has;
        const long long at0 = (b * a.I + ic) * a.S + row * SR;
        float x[SR];
        const float *from = a.chunks > 1 ? behind + chunk * a.B * a.I * a.S : dhT;
        load_states<SR>(from + at0, from ? have : 0, x);
        Walk<T, 4> wu, wd, wz, wg;
        wu.init(a, u, a.pu, b, l, rv, ic);
        wd.init(a, delta, a.pd, b, l, rv, ic);
        if (z) wz.init(a, z, a.pz, b, l, rv, ic);
        wg.init(a, dy, a.I, b, l, rv, ic);
        StateRows<T, SR, kSelKeep, 1> rB, rC;
        rB.init(a, Bm, a.pB, b, lane);
        rC.init(a, Cm, a.pC, b, lane);
        // dense outputs are where dy is
        char *const bu = (char *)du + (wg.base - (const char *)dy), *const bd = (char *)ddelta + (wg.base - (const char *)dy);
        char *const bz = (char *)dz + (wg.base - (const char *)dy);
        const long long whole = whole_until<1, 1>(a, b, last);
        Few<T, 1> ru[4], rd[4], rz[4], rg[4];
        float hs[SR];
        const auto fetch_as = [&](long long s0, auto all) {
            constexpr bool W = decltype(all)::value;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const long long s = s0 + 4 * k;
                const int have = !W && has && s + rv < last && s + rv < l.n;
                wu.load(ru[k], s, W, have);
                wd.load(rd[k], s, W, have);
                wg.load(rg[k], s, W, have);
                if (z) wz.load(rz[k], s, W, have);
            }
            rB.load(s0, last, W);
            rC.load(s0, last, W);
        };
        const auto fetch = [&](long long s0) {
            if (s0 + kSelKeep <= whole) fetch_as(s0, std::true_type());
            else fetch_as(s0, std::false_type());
            load_states<SR>(saved + ((b * a.kept + s0 / kSelKeep) * a.I + ic) * a.S + row * SR, have, hs);
        };
        const long long blocks = (last - first + kSelKeep - 1) / kSelKeep;
        fetch(first + (blocks - 1) * kSelKeep);
        int turn = 0;
        for (long long bl = blocks - 1; bl >= 0; --bl) {
            const long long s0 = first + bl * kSelKeep;
            const bool all = s0 + kSelKeep <= whole;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const bool live = has && (all || s0 + 4 * k + rv < l.n);
                const float g = live ? rg[k].get(0) : 0.0f, uv = live ? ru[k].get(0) : 0.0f;
                float dv = rd[k].get(0) + bias, back = 1.0f, dpv = g, slope = 0.0f;
                if (a.softplus) dv = softplus_slope(dv, back);
                dv = live ? dv : 0.0f;
                back = live ? back : 0.0f;
                if (z) {
                    float v;
                    slope = g * silu_slope(rz[k].get(0), v);
                    dpv = g * v;
                    sh.slope[4 * k + rv][ch] = slope;
                }
                sh.du[4 * k + rv][ch] = make_float2(dv, dv * uv);
                sh.own[4 * k + rv][ch] = make_float2(uv, back);
                sh.dp[4 * k + rv][ch] = dpv;
                dDv = fmaf(dpv, uv, dDv);
            }
            rB.put(sh.B);
            rC.put(sh.C);
            float h[SR];
#pragma unroll
            for (int j = 0; j < SR; ++j) h[j] = sh.start[0][j][lane] = hs[j];
            wave_sync();
            if (bl > 0) fetch(s0 - kSelKeep);
#pragma unroll 1
            for (int q = 0; q < NR - 1; ++q) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float2 v = sh.du[q * R + r][ch];
                    float Bv[SR];
                    row_states<SR>(&sh.B[q * R + r][row * SR], Bv);
#pragma unroll
                    for (int j = 0; j < SR; ++j) h[j] = fmaf(__builtin_amdgcn_exp2f(v.x * A2[j]), h[j], v.y * Bv[j]);
                }
#pragma unroll
                for (int j = 0; j < SR; ++j) sh.start[q + 1][j][lane] = h[j];
            }
#pragma unroll 1
            for (int q = NR - 1; q >= 0; --q, turn ^= 1) {
                const int at = q * R;
                float dec[R][SR], hb[R][SR], yp[R], qv[R], wv[R];
                // the registers are for decays and states: rows are read again on the way back, and not ahead of their position
                wave_sync();
#pragma unroll
                for (int j = 0; j < SR; ++j) h[j] = sh.start[q][j][lane];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float2 v = sh.du[at + r][ch];
                    float Bv[SR], Cv[SR];
                    row_states<SR>(&sh.B[at + r][row * SR], Bv);
                    row_states<SR>(&sh.C[at + r][row * SR], Cv);
                    yp[r] = 0.0f;
#pragma unroll
                    for (int j = 0; j < SR; ++j) {
                        dec[r][j] = __builtin_amdgcn_exp2f(v.x * A2[j]);
                        hb[r][j] = h[j];
                        h[j] = fmaf(dec[r][j], h[j], v.y * Bv[j]);
                        yp[r] = fmaf(Cv[j], h[j], yp[r]);
                    }
                    made(yp[r]);
                    if (r % 2) __builtin_amdgcn_sched_barrier(0);
                }
                sum_states<K>(yp);
                wave_sync();
#pragma unroll
                for (int r = R - 1; r >= 0; --r) {
                    const float2 v = sh.du[at + r][ch];
                    const float g = sh.dp[at + r][ch];
                    float gB[SR], gC[SR], Bv[SR], Cv[SR];
                    row_states<SR>(&sh.B[at + r][row * SR], Bv);
                    row_states<SR>(&sh.C[at + r][row * SR], Cv);
                    qv[r] = wv[r] = 0.0f;
#pragma unroll
                    for (int j = 0; j < SR; ++j) {
                        // the gradient that goes on is a G: times the state before, it is that of the exponent
                        const float G = fmaf(Cv[j], g, x[j]);
                        gC[j] = g * (r + 1 < R ? hb[r + 1][j] : h[j]);
                        gB[j] = G * v.y;
                        qv[r] = fmaf(G, Bv[j], qv[r]);
                        x[j] = dec[r][j] * G;
                        const float t = x[j] * hb[r][j];
                        wv[r] = fmaf(t, A2[j], wv[r]);
                        dA[j] = fmaf(t, v.x, dA[j]);
                    }
                    // lanes of a four write the same value
                    if constexpr (SR >= 4) {
#pragma unroll
                        for (int j = 0; j < SR; j += 4) {
                            sh.out[turn][0][r][row * SR + j + fv] = sum_four(gB[j], gB[j + 1], gB[j + 2], gB[j + 3]);
                            sh.out[turn][1][r][row * SR + j + fv] = sum_four(gC[j], gC[j + 1], gC[j + 2], gC[j + 3]);
                        }
                    } else if constexpr (SR == 2) {
                        sh.out[turn][fv >> 1][r][row * SR + (fv & 1)] = sum_four(gB[0], gB[1], gC[0], gC[1]);
                    } else {
                        sh.out[turn][fv & 1][r][row] = sum_four(gB[0], gC[0], gB[0], gC[0]);
                    }
#pragma unroll
                    for (int j = 0; j < SR; ++j) made(dA[j]);
                    made(qv[r]);
                    made(wv[r]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                sum_states<K>(qv);
                sum_states<K>(wv);
#pragma unroll
                for (int m = 0; m < K; ++m) {
                    const int e = at + 4 * m + rv;
                    const long long s = s0 + e;
                    const float2 o = sh.own[e][ch];
                    const float ed = fmaf(o.x, qv[m], wv[m] * kLn2) * o.y;
                    dbv += ed;
                    // from dy's place on, where dense outputs are; padding gets zeros
                    bool write = has, live = true;
                    long long to = (s0 + at + 4 * m) * wg.step + wg.off;
                    if (!all) {
                        live = s < l.n;
                        write = has && s < last;
                        to = (const char *)(dy + l.row(a, s) * a.I + ic) - wg.base;
                    }
                    if (write) {
                        put_one((T *)(bu + to), live ? fmaf(sh.du[e][ch].x, qv[m], Dv * sh.dp[e][ch]) : 0.0f);
                        put_one((T *)(bd + to), live ? ed : 0.0f);
                        if (z) put_one((T *)(bz + to), live ? sh.slope[e][ch] * fmaf(Dv, o.x, yp[m]) : 0.0f);
                    }
                }
                if (WIDE) __syncthreads(); else wave_sync();
                const int step = WIDE ? (int)blockDim.x : 64, e0 = WIDE ? (int)threadIdx.x : lane;
                const auto add_up = [&](int e) {
                    float v = (&(WIDE ? shared[0] : sh).out[turn][0][0][0])[e];
                    if (WIDE)
                        for (int w = 1; w < waves; ++w) v += (&shared[w].out[turn][0][0][0])[e];
                    return v;
                };
                if (all && 2 * R * SP <= step) {
                    // one element a thread, a scalar place and the thread's own part
                    if (out_off >= 0) {
                        const long long row0 = b * a.T + (a.reverse ? l.n - R - (s0 + at) : s0 + at);
                        const float v = add_up(e0);
                        if (!WIDE || wide == 1) put_one((e0 < R * SP ? dB : dC) + row0 * a.S + out_off, v);
                        else ((e0 < R * SP ? dBp : dCp) + group * a.B * a.T * a.S + row0 * a.S)[out_off] = v;
                    }
                } else {
                    for (int e = e0; e < 2 * R * SP; e += step) {
                        const int what = e / (R * SP), r = e / SP % R, k = e % SP;
                        if (k >= a.S || s0 + at + r >= last) continue;
                        const float v = add_up(e);
                        const long long to = l.row(a, s0 + at + r) * a.S + k;
                        if (!WIDE || wide == 1) put_one((what ? dC : dB) + to, v);
                        else (what ? dCp : dBp)[group * a.B * a.T * a.S + to] = v;
                    }
                }
            }
            wave_sync();
#pragma unroll
            for (int j = 0; j < SR; ++j) {
                dAs[j] += (double)dA[j];
                dA[j] = 0.0f;
            }
            dDs += (double)dDv;
            dbs += (double)dbv;
            dDv = dbv = 0.0f;
        }
        if (dh0 && chunk == 0) store_states<SR>(dh0 + at0, have, x);
    }
#pragma unroll
    for (int j = 0; j < SR; ++j) dA[j] = (float)dAs[j];
    store_states<SR>(dAp + (job0 * a.I + ic) * a.S + row * SR, have, dA);
    dDs += __shfl_xor(dDs, 16);
    dDs += __shfl_xor(dDs, 32);
    dbs += __shfl_xor(dbs, 16);
    dbs += __shfl_xor(dbs, 32);
    if (row == 0 && has) {
        dDp[(job0 * a.I + i) * 2] = (float)dDs;
        dDp[(job0 * a.I + i) * 2 + 1] = (float)dbs;
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

// dA [I S], dD and ddelta_bias [I] from the jobs' parts, from workgroup `first` of all on, in 64 bits: L lanes an output.
template <int L>
__global__ void __launch_bounds__(16 * L)
k_sel_weights(unsigned first, long long nA, long long I, int jobs, const float *dAp, const float *dDp, float *dA, float *dD, float *db)
{
    __shared__ double lds[L][16];
    const int o = threadIdx.x % 16, lane = threadIdx.x / 16;
    const long long at = (long long)(first + blockIdx.x) * 16 + o, nD = 2 * I;
    double s = 0.0;
    if (at < nA + nD) {
        const float *p = at < nA ? dAp + at : dDp + (at - nA);
        const long long step = at < nA ? nA : nD;
#pragma unroll 8
        for (int j = lane; j < jobs; j += L) s += (double)p[j * step];
    }
    lds[lane][o] = s;
    __syncthreads();
#pragma unroll
    for (int n = L / 2; n > 0; n /= 2) {
        if (lane < n) lds[lane][o] += lds[lane + n][o];
        __syncthreads();
    }
    if (lane || at >= nA + nD) return;
    s = lds[0][o];
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
    if (S > kSelMaxS || B > (1LL << 30) || T > (1LL << 31) || I > (1LL << 24)) return PLSTM_EUNSUPPORTED;
    if (B > (1LL << 30) / I || T > (1LL << 38) / (B * I) || B * I > (1LL << 34) / S) return PLSTM_EUNSUPPORTED;
    // waves of a launch
    if (B * ((I + 15) / 16) > (1LL << 22)) return PLSTM_EUNSUPPORTED;
    return PLSTM_OK;
}

// Waves that fill the card, and the fewest positions of a chunk.  bf16, forward (and backward): 1 x 16384 x 1024 144 us with 4096 waves, 150
// with 2048, 185 with 1024; 2 x 4096 x 2048 499, 515, 593.  1 x 1024 x 512 in chunks of
// 32 positions 66 us, of 64 90, of 128 147, of 16 65: a chain of 32 chunks.  The chain takes chunks one after another, 14 us for 128 of
// them, and the rule does not weigh that: sequences of few channels have up to 4096.
constexpr long long kSelFill = 4096, kSelChunk = 32;

struct SelPlan {
    SelArgs a;                          // of the forward and the folds
    int SR, CL, NB;
    long long tiles;                    // backward: waves of 16 channels across a sequence's
    int waves;                          // backward: of a workgroup
    float *H, *sums, *dBp, *dCp, *dAp, *dDp;
    size_t ws;
};

SelPlan sel_plan(int64_t B, int64_t T, int64_t I, int32_t S, int32_t reverse, int32_t softplus, int64_t pu, int64_t pd,
                 int64_t pz, int64_t pB, int64_t pC, const int32_t *lengths, void *ws, bool backward)
{
    SelPlan p{};
    SelArgs &a = p.a;
    p.SR = sel_sr(S);
    p.CL = sel_cl(p.SR);
    a.B = B; a.T = T; a.I = I; a.S = S;
    a.reverse = reverse;
    a.softplus = softplus;
    a.pu = pu ? pu : I; a.pd = pd ? pd : I; a.pz = pz ? pz : I; a.pB = pB ? pB : S; a.pC = pC ? pC : S;
    a.lengths = lengths;
    const long long lanes = (I + p.CL - 1) / p.CL;
    // few channels: sequences share a wave (11520 x 240 x 16 forward and backward 981 us, one a wave 1073)
    p.NB = p.CL == 1 || lanes > 8 ? 1 : lanes > 4 ? 2 : 4;
    // sequences that share a wave are within 32-bit offsets of each other
    const long long widest = std::max({a.pu, a.pd, a.pz, a.pB, a.pC});
    if (T > (1LL << 28) / widest / p.NB) p.NB = 1;
    a.tiles = (lanes + 15) / 16;
    a.groups = p.NB == 1 ? B * a.tiles : (B + p.NB - 1) / p.NB;
    a.kept = (T + kSelKeep - 1) / kSelKeep;
    p.tiles = (I + 15) / 16;
    long long chunks = 2 * a.groups <= kSelFill ? kSelFill / a.groups : 1;
    if (chunks > (T + kSelChunk - 1) / kSelChunk) chunks = (T + kSelChunk - 1) / kSelChunk;
    a.chunk = (long long)align_up((size_t)((T + chunks - 1) / chunks), kSelKeep);
    a.chunks = (int)((T + a.chunk - 1) / a.chunk);
    Carve cv(ws);
    if (a.chunks > 1) {
        p.H = cv.take<float>((size_t)a.chunks * B * I * S);
        p.sums = cv.take<float>((size_t)a.chunks * B * I);
    }
    if (backward) {
        p.waves = p.tiles == 1 ? 4 : (int)(p.tiles < 4 ? p.tiles : 4);
        // each of at most 4096 waves takes as many chunks as the others
        const long long all = B * a.chunks, each = (all * p.tiles + 4095) / 4096;
        a.jobs = (all + each - 1) / each;
        const long long groups = (p.tiles + p.waves - 1) / p.waves;
        if (p.tiles > 1 && groups > 1) {
            p.dBp = cv.take<float>((size_t)groups * B * T * S);
            p.dCp = cv.take<float>((size_t)groups * B * T * S);
        }
        p.dAp = cv.take<float>((size_t)a.jobs * I * S);
        p.dDp = cv.take<float>((size_t)a.jobs * I * 2);
    }
    p.ws = align_up(cv.off, 256);
    if (p.ws < 256) p.ws = 256;
    return p;
}

// Rows are at most 2^24 elements apart: lanes' offsets within a stage have 32 bits.
constexpr long long kSelMaxPitch = 1LL << 24;
bool sel_pitch(int64_t n, int64_t pitch) { return pitch == 0 || (pitch >= n && pitch <= kSelMaxPitch); }

// The tensors of a call.
struct SelTensors {
    const void *u, *delta, *A, *Bm, *Cm, *D, *z, *dbias, *h0, *saved, *dy, *dhT;
    void *y, *hT, *keep, *du, *ddelta, *dA, *dB, *dC, *dD, *dz, *db, *dh0;
};

unsigned sel_blocks(long long waves) { return (unsigned)((waves + 3) / 4); }

// Folds all chunks but one, and chains them.
template <typename T, int SR, int NB, bool BACK>
int sel_chain(const SelPlan &p, const SelTensors &t, hipStream_t st)
{
    constexpr int CL = sel_cl(SR);
    const SelArgs &a = p.a;
    k_sel_fold<T, SR, CL, NB, BACK><<<sel_blocks(a.groups * (a.chunks - 1)), 256, 0, st>>>(
        a, (const T *)t.u, (const T *)t.delta, (const float *)t.A, (const T *)(BACK ? t.Cm : t.Bm), BACK ? a.pC : a.pB,
        (const T *)t.z, (const T *)t.dy, (const float *)t.dbias, p.H, p.sums);
    PLSTM_LAUNCH_CHECK();
    const long long cols = a.B * a.I;
    k_sel_chain<BACK><<<(unsigned)((cols * a.S + 255) / 256), 256, 0, st>>>(
        cols, a.I, a.S, a.chunks, (const float *)t.A, (const float *)(BACK ? t.dhT : t.h0), p.H, p.sums);
    PLSTM_LAUNCH_CHECK();
    return 2;
}

template <typename T, int SR, int NB>
int sel_forward(const SelPlan &p, const SelTensors &t, hipStream_t st)
{
    constexpr int CL = sel_cl(SR);
    const SelArgs &a = p.a;
    int launches = 1;
    if (a.chunks > 1) {
        const int n = sel_chain<T, SR, NB, false>(p, t, st);
        if (n < 0) return n;
        launches += n;
    }
    k_sel_fwd<T, SR, CL, NB><<<sel_blocks(a.groups * a.chunks), 256, 0, st>>>(
        a, (const T *)t.u, (const T *)t.delta, (const float *)t.A, (const T *)t.Bm, (const T *)t.Cm, (const float *)t.D,
        (const T *)t.z, (const float *)t.dbias, (const float *)t.h0, (T *)t.y, (float *)t.hT, (float *)t.keep, p.H);
    PLSTM_LAUNCH_CHECK();
    return launches;
}

template <typename T, int SR, bool WIDE>
int sel_backward_walk(const SelPlan &p, const SelTensors &t, hipStream_t st)
{
    SelArgs a = p.a;
    a.tiles = p.tiles;
    const size_t lds = p.waves * sizeof(BackShared<SR>);
    const void *fn = (const void *)k_sel_bwd<T, SR, WIDE>;
    if (lds > 65536 && hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess)
        return PLSTM_EHIP;
    const long long blocks = WIDE ? (p.tiles + p.waves - 1) / p.waves * a.jobs : (a.jobs + p.waves - 1) / p.waves;
    k_sel_bwd<T, SR, WIDE><<<(unsigned)blocks, 64 * p.waves, lds, st>>>(
        a, (const T *)t.u, (const T *)t.delta, (const float *)t.A, (const T *)t.Bm, (const T *)t.Cm, (const float *)t.D,
        (const T *)t.z, (const float *)t.dbias, (const float *)t.saved, (const T *)t.dy, (const float *)t.dhT, p.H,
        (T *)t.du, (T *)t.ddelta, (T *)t.dz, (float *)t.dh0, p.dBp, p.dCp, (T *)t.dB, (T *)t.dC, p.dAp, p.dDp);
    PLSTM_LAUNCH_CHECK();
    return 1;
}

template <typename T, int SR, int NB>
int sel_backward(const SelPlan &p, const SelTensors &t, hipStream_t st)
{
    const SelArgs &a = p.a;
    int launches = 0;
    if (a.chunks > 1) {
        const int n = sel_chain<T, SR, NB, true>(p, t, st);
        if (n < 0) return n;
        launches += n;
    }
    const int n = (p.tiles > 1 ? sel_backward_walk<T, SR, true> : sel_backward_walk<T, SR, false>)(p, t, st);
    if (n < 0) return n;
    launches += n;
    if (p.dBp) {
        const long long n = a.B * a.T * a.S;
        k_sel_rows<T><<<(unsigned)min((n + 255) / 256, 8192LL), 256, 0, st>>>(
            n, (int)((p.tiles + p.waves - 1) / p.waves), p.dBp, p.dCp, (T *)t.dB, (T *)t.dC);
        PLSTM_LAUNCH_CHECK();
        ++launches;
    }
    const long long nA = a.I * a.S;
    const auto weights = [&](auto l) {
        constexpr int L = decltype(l)::value;
        launches += in_launches<16 * L>((nA + 2 * a.I + 15) / 16, [&](unsigned first, unsigned n) {
            k_sel_weights<L><<<n, 16 * L, 0, st>>>(first, nA, a.I, (int)a.jobs, p.dAp, p.dDp, (float *)t.dA, (float *)t.dD,
                                                   (float *)t.db);
        });
    };
    // 3840 parts of 16 x 16 outputs: 64 lanes each 14.6 us, 16 lanes 19.0; 64 parts of 2048 x 16: 8.8, 5.0
    if (a.jobs > 128) weights(std::integral_constant<int, 64>());
    else weights(std::integral_constant<int, 16>());
    PLSTM_LAUNCH_CHECK();
    return launches;
}

template <typename T>
int sel_step(const SelPlan &p, const SelTensors &t, hipStream_t st)
{
    const SelArgs &a = p.a;
    const int L = a.S <= 4 ? 1 : a.S <= 8 ? 2 : a.S <= 16 ? 4 : a.S <= 32 ? 8 : 16;
    const unsigned blocks = (unsigned)((a.B * a.I * L + 255) / 256);
    const auto step = [&](auto l) {
        k_sel_step<T, decltype(l)::value><<<blocks, 256, 0, st>>>(
            a, (const T *)t.u, (const T *)t.delta, (const float *)t.A, (const T *)t.Bm, (const T *)t.Cm,
            (const float *)t.D, (const T *)t.z, (const float *)t.dbias, (const float *)t.h0, (T *)t.y, (float *)t.hT);
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

template <typename T, int SR, int NB>
int sel_run_one(const SelPlan &p, const SelTensors &t, bool backward, hipStream_t st)
{
    return backward ? sel_backward<T, SR, NB>(p, t, st) : sel_forward<T, SR, NB>(p, t, st);
}

template <typename T>
int sel_run_all(const SelPlan &p, const SelTensors &t, bool backward, hipStream_t st)
{
    if (!backward && p.a.T == 1 && !t.keep) return sel_step<T>(p, t, st);
    switch (p.SR * 8 + p.NB) {
    case 9: return sel_run_one<T, 1, 1>(p, t, backward, st);
    case 10: return sel_run_one<T, 1, 2>(p, t, backward, st);
    case 12: return sel_run_one<T, 1, 4>(p, t, backward, st);
    case 17: return sel_run_one<T, 2, 1>(p, t, backward, st);
    case 18: return sel_run_one<T, 2, 2>(p, t, backward, st);
    case 20: return sel_run_one<T, 2, 4>(p, t, backward, st);
    case 33: return sel_run_one<T, 4, 1>(p, t, backward, st);
    case 34: return sel_run_one<T, 4, 2>(p, t, backward, st);
    case 36: return sel_run_one<T, 4, 4>(p, t, backward, st);
    case 65: return sel_run_one<T, 8, 1>(p, t, backward, st);
    default: return sel_run_one<T, 16, 1>(p, t, backward, st);
    }
}

}  // namespace
}  // namespace plstm

using namespace plstm;

extern "C" {

size_t pyramid_selective_scan_saved_size(int64_t B, int64_t T, int64_t I, int32_t S)
{
    if (check_sel(B, T, I, S, PLSTM_F32) != PLSTM_OK) return 0;
    return align_up((size_t)B * ((T + kSelKeep - 1) / kSelKeep) * I * S * sizeof(float), 256);
}

size_t pyramid_selective_scan_workspace_size(int64_t B, int64_t T, int64_t I, int32_t S, int32_t backward)
{
    if (check_sel(B, T, I, S, PLSTM_F32) != PLSTM_OK || (backward != 0 && backward != 1)) return 0;
    // of rows as near and as far apart as they may be: whether sequences share waves decides the chunks
    size_t most = 0;
    for (long long pitch : {0LL, kSelMaxPitch})
        most = std::max(most, sel_plan(B, T, I, S, 0, 0, pitch, pitch, 0, 0, 0, nullptr, nullptr, backward != 0).ws);
    return most;
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
    if (!sel_pitch(I, u_pitch) || !sel_pitch(I, delta_pitch) || !sel_pitch(I, z_pitch) ||
        !sel_pitch(S, B_pitch) || !sel_pitch(S, C_pitch))
        return PLSTM_EINVAL;
    const size_t e = dtype_size(dtype);
    if (!aligned_to(u, e) || !aligned_to(delta, e) || !aligned_to(A, 4) || !aligned_to(Bm, e) || !aligned_to(Cm, e) ||
        !aligned_to(D, 4) || !aligned_to(z, e) || !aligned_to(delta_bias, 4) || !aligned_to(lengths, 4) ||
        !aligned_to(h0, 4) || !aligned_to(y, e) || !aligned_to(hT, 4) || !aligned_to(saved, 16) || !aligned_to(ws, 16))
        return PLSTM_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const SelPlan p = sel_plan(B, T, I, S, reverse, softplus, u_pitch, delta_pitch, z_pitch, B_pitch, C_pitch, lengths,
                               ws, false);
    if (ws_bytes < p.ws) return PLSTM_EWORKSPACE;
    timing_begin("selective_fwd", st);
    SelTensors t{u, delta, A, Bm, Cm, D, z, delta_bias, h0};
    t.y = y;
    t.hT = hT;
    t.keep = saved;
    const int n = (dtype == PLSTM_F32 ? sel_run_all<float> : sel_run_all<uint16_t>)(p, t, false, st);
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
    if (!sel_pitch(I, u_pitch) || !sel_pitch(I, delta_pitch) || !sel_pitch(I, z_pitch) ||
        !sel_pitch(S, B_pitch) || !sel_pitch(S, C_pitch))
        return PLSTM_EINVAL;
    const size_t e = dtype_size(dtype);
    if (!aligned_to(u, e) || !aligned_to(delta, e) || !aligned_to(A, 4) || !aligned_to(Bm, e) || !aligned_to(Cm, e) ||
        !aligned_to(D, 4) || !aligned_to(z, e) || !aligned_to(delta_bias, 4) || !aligned_to(lengths, 4) ||
        !aligned_to(saved, 16) || !aligned_to(dy, e) || !aligned_to(dhT, 4) || !aligned_to(du, e) ||
        !aligned_to(ddelta, e) || !aligned_to(dA, 4) || !aligned_to(dB, e) || !aligned_to(dC, e) || !aligned_to(dD, 4) ||
        !aligned_to(dz, e) || !aligned_to(ddelta_bias, 4) || !aligned_to(dh0, 4) || !aligned_to(ws, 16))
        return PLSTM_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const SelPlan p = sel_plan(B, T, I, S, reverse, softplus, u_pitch, delta_pitch, z_pitch, B_pitch, C_pitch, lengths,
                               ws, true);
    if (ws_bytes < p.ws) return PLSTM_EWORKSPACE;
    const SelTensors t{u, delta, A, Bm, Cm, D, z, delta_bias, nullptr, saved, dy, dhT, nullptr, nullptr, nullptr,
                       du, ddelta, dA, dB, dC, dD, dz, ddelta_bias, dh0};
    timing_begin("selective_bwd", st);
    const int n = (dtype == PLSTM_F32 ? sel_run_all<float> : sel_run_all<uint16_t>)(p, t, true, st);
    if (n < 0) return n;
    timing_end(n, st);
    return PLSTM_OK;
}

}  // extern "C"
