// Gated linear recurrence along an axis, and its backward pass.  Over a
// sequence of T steps and I channels, position s = 0 .. n - 1 of the sweep being
// step t = s, or n - 1 - s in reverse (n the sequence's length):
//   f = sigmoid(g_t),  h_s = f h_{s-1} + (1 - f) u_t,  h_{-1} = h0
// Backward, G_s the gradient of h_s:
//   G_s = dh_t + f_{s+1} G_{s+1}  (the last one takes dhT as well)
//   du_t = (1 - f) G_s,  dg_t = G_s (h_{s-1} - u_t) f (1 - f),  dh0 = f_0 G_0
// States and gradients of states are fp32.  1 - f is sigmoid(-g), not a
// difference: a gate that keeps all but 1e-5 of the state keeps its bits.
// A training forward keeps the state before every 16th position; the backward
// computes the others again from g and u (in the storage type or from 8-bit
// checkpoints), which costs 1/4 byte an element where reading h would cost 2
// or 4.
#include "code8.h"
#include "sweep.h"
#include "timing.h"

namespace plstm {
namespace {

constexpr int kRun = 16;            // positions between kept states, and of a wave's run
constexpr int kGroup = 16;          // chunks between chained states
constexpr uint64_t kEmpty = ~0ull;  // a word that its chunk has not written
constexpr uint32_t kEmptyState = ~0u;

struct ScanArgs {
    long long T, I, cols;           // steps, channels, B I
    int reverse;
    const int32_t *lengths;
    long long runs;                 // ceil(T / kRun)
};

// Chunks of a sequence (kRun positions for each wave of a workgroup) run at the
// same time and hand the state on through memory:
//   agg [chunk][cols]   (A, H) of a chunk: its last state is A (state before) + H
//   state [group][cols] the state before every kGroup-th chunk
// A word is written whole, so whoever finds it other than empty has it all: no
// flag, no fence.  A chunk publishes its aggregate as soon as it has its inputs;
// it then needs its group's state and the aggregates of the chunks before it in
// the group, always folded in the same order, so results do not depend on which
// chunk was faster.  Only the last chunk of a group waits on a chain, one link
// per kGroup chunks.
struct Chain {
    uint64_t *agg;
    uint32_t *state;
    uint32_t *ticket;               // chunks are taken in order: whoever waits, waits on started ones
    int *status;                    // device status word
    int chunks, blocks;             // chunks of a sequence, workgroups across the columns
    int spin, bias;                 // polls before a wait gives up; test mode
};

__global__ void __launch_bounds__(256)
k_scan_chain_init(Chain ch, long long cols, const float *start)
{
    const long long i0 = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long stride = (long long)gridDim.x * 256;
    const long long na = ch.chunks * cols, ns = (ch.chunks + kGroup - 1) / kGroup * cols;
    for (long long i = i0; i < na; i += stride) ch.agg[i] = kEmpty;
    for (long long i = i0; i < ns; i += stride) {
        const float v = i < cols && start ? start[i] : 0.0f;
        ch.state[i] = i >= cols ? kEmptyState : v != v ? 0x7fc00000u : float_bits(v);
    }
    if (i0 == 0) *ch.ticket = 0;
}

// f and 1 - f of sigmoid's argument.
__device__ inline void gate(float g, float &keep, float &take)
{
    const float e = __expf(-fabsf(g));
    const float r = __builtin_amdgcn_rcpf(1.0f + e);
    const float small = e * r;
    keep = g < 0.0f ? small : r;
    take = g < 0.0f ? r : small;
}

template <typename T>
__device__ inline float load_at(const T *x, const uint16_t *, long long i)
{
    return Store<T>::load(x, i);
}
__device__ inline float load_at(const int8_t *x, const uint16_t *scale, long long i)
{
    return (float)x[i] * bf16_to_f32(scale[i >> 6]);
}

// A lane's column: a channel i of sequence b.
struct Column {
    bool has;                       // false past the last column (then a copy of it)
    long long col, base, saved;     // base: element (b, 0, i); saved: state (b, 0, i)
    long long n;                    // the sequence's length
};
__device__ inline Column column_of(const ScanArgs &a, long long col)
{
    Column c;
    c.has = col < a.cols;
    c.col = c.has ? col : a.cols - 1;
    const long long b = c.col / a.I, i = c.col - b * a.I;
    c.base = b * a.T * a.I + i;
    c.saved = b * a.runs * a.I + i;
    c.n = a.T;
    if (a.lengths) {
        const long long n = a.lengths[b];
        c.n = n < 0 ? 0 : n > a.T ? a.T : n;
    }
    return c;
}

// Elements of a run of positions s0 .. s0 + count - 1 (count <= kRun) of a column.
// Positions past the sequence's length stand for the steps of the same number.
template <bool RAGGED>
struct RunAt {
    long long first, step, pad, I;
    int live;                       // positions of the run that the sequence has
    __device__ RunAt(const ScanArgs &a, const Column &c, long long s0)
    {
        I = a.I;
        first = c.base + (a.reverse ? c.n - 1 - s0 : s0) * I;
        step = a.reverse ? -I : I;
        pad = c.base + s0 * I;
        const long long left = c.n - s0;
        live = left < 0 ? 0 : left > kRun ? kRun : (int)left;
    }
    __device__ long long at(int k) const
    {
        if (RAGGED) return k < live ? first + k * step : pad + k * I;
        return first + k * step;
    }
};

// Folds (A, H) pairs lds[0 .. count - 1] over v in order.
__device__ inline float fold(const float2 (*lds)[64], int count, int lane, float v)
{
    for (int w = 0; w < count; ++w) {
        const float2 p = lds[w][lane];
        v = fmaf(p.x, v, p.y);
    }
    return v;
}

// The state before chunk k of the lane's column, and the end state to the next
// group where chunk k is a group's last.  (A, H): the chunk's aggregate.
__device__ inline float chained(const Chain &ch, long long cols, long long col, bool has, int k,
                                float A, float H)
{
    if (has) {
        const uint64_t word = (uint64_t)float_bits(H) << 32 |
                              (A != A ? 0x7fc00000u : float_bits(A));
        __hip_atomic_store(&ch.agg[k * cols + col], word, __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
    }
    const int g = k / kGroup, first = g * kGroup;
    uint64_t w[kGroup];
    uint32_t s = kEmptyState;
    for (int polls = 0;; ++polls) {
        s = __hip_atomic_load(&ch.state[g * cols + col], __ATOMIC_RELAXED,
                              __HIP_MEMORY_SCOPE_AGENT);
        bool all = s != kEmptyState;
#pragma unroll
        for (int j = 0; j < kGroup - 1; ++j)
            if (first + j < k) {
                w[j] = __hip_atomic_load(&ch.agg[(first + j) * cols + col], __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
                all = all && w[j] != kEmpty;
            }
        if (__all(all && ch.bias == 0)) break;
        if (polls >= ch.spin) {
            // gave up: NaN from here on
            if (threadIdx.x == 0)
                __hip_atomic_fetch_or(ch.status, PLSTM_DEVICE_WAIT_GAVE_UP, __ATOMIC_RELAXED,
                                      __HIP_MEMORY_SCOPE_AGENT);
            s = 0x7fc00000u;
            break;
        }
        __builtin_amdgcn_s_sleep(1);
    }
    float v = bits_float(s);
#pragma unroll
    for (int j = 0; j < kGroup - 1; ++j)
        if (first + j < k) v = fmaf(bits_float((uint32_t)w[j]), v, bits_float((uint32_t)(w[j] >> 32)));
    if (k - first == kGroup - 1 && has) {
        const float e = fmaf(A, v, H);
        if (k + 1 < ch.chunks)
            __hip_atomic_store(&ch.state[(g + 1) * cols + col],
                               e != e ? 0x7fc00000u : float_bits(e), __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
    }
    return v;
}

// The next chunk of the chain: its number, and the workgroup's place across the columns.
__device__ inline void take_chunk(const Chain &ch, int &chunk, int &block)
{
    __shared__ uint32_t ticket;
    if (threadIdx.x == 0)
        ticket = __hip_atomic_fetch_add(ch.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    chunk = (int)(ticket / (uint32_t)ch.blocks);
    block = (int)(ticket - (uint32_t)chunk * (uint32_t)ch.blocks);
}

// A workgroup of W waves advances 64 columns by W runs of 16 positions at a
// time, wave w holding run w in registers.  W = 1 walks its runs one after
// another; with more, each wave folds its run to (A, H), and starts it again from
// the state that the waves before it leave.  CHAIN: the workgroup has one chunk
// of W runs and takes the state from the chain.
template <typename T, int W, bool RAGGED, bool CHAIN>
__global__ void __launch_bounds__(64 * W)
k_scan_fwd(ScanArgs a, Chain ch, const T *__restrict__ g, const T *__restrict__ u,
           const float *h0, T *__restrict__ h, float *hT, float *__restrict__ saved)
{
    __shared__ float2 lds[CHAIN ? 1 : 2][W > 1 ? W : 1][64];
    __shared__ float start[64];
    const int lane = threadIdx.x & 63, wave = W > 1 ? threadIdx.x / 64 : 0;
    int chunk = 0, block = blockIdx.x;
    if (CHAIN) take_chunk(ch, chunk, block);
    const Column c = column_of(a, (long long)block * 64 + lane);
    float carry = !CHAIN && h0 ? h0[c.col] : 0.0f;
    int turn = 0;
    for (long long r0 = (long long)chunk * W; r0 < a.runs; r0 += W, turn ^= 1) {
        const long long run = r0 + wave, s0 = run * kRun;
        const int count = run < a.runs ? (int)min((long long)kRun, a.T - s0) : 0;
        const RunAt<RAGGED> at(a, c, s0);
        float f[kRun], v[kRun];
        if (count > 0) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                const long long e = at.at(k < count ? k : count - 1);
                f[k] = Store<T>::load(g, e);
                v[k] = Store<T>::load(u, e);
            }
        }
        float A = 1.0f, H = 0.0f;
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            float keep, take;
            gate(f[k], keep, take);
            const bool in = RAGGED ? k < at.live && k < count : k < count;
            f[k] = in ? keep : 1.0f;
            v[k] = in ? take * v[k] : 0.0f;
            if (W > 1) {
                A *= f[k];
                H = fmaf(f[k], H, v[k]);
            }
        }
        float st = carry;
        if (W > 1) {
            lds[CHAIN ? 0 : turn][wave][lane] = make_float2(A, H);
            __syncthreads();
            const float2 (*parts)[64] = lds[CHAIN ? 0 : turn];
            if (CHAIN) {
                if (wave == 0) {
                    float ca = 1.0f, cb = 0.0f;
                    for (int w = 0; w < W; ++w) {
                        const float2 p = parts[w][lane];
                        ca *= p.x;
                        cb = fmaf(p.x, cb, p.y);
                    }
                    start[lane] = chained(ch, a.cols, c.col, c.has, chunk, ca, cb);
                }
                __syncthreads();
                carry = start[lane];
            }
            st = fold(parts, wave, lane, carry);
        }
        if (count > 0) {
            if (saved && c.has) saved[c.saved + run * a.I] = st;
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                st = fmaf(f[k], st, v[k]);
                const bool in = !RAGGED || k < at.live;
                if (k < count && c.has) Store<T>::store(h, at.at(k), in ? st : 0.0f);
            }
        }
        if (W == 1) carry = st;
        else if (!CHAIN) carry = fold(lds[turn] + wave, W - wave, lane, fold(lds[turn], wave, lane, carry));
        else if (hT && c.has && run == a.runs - 1) hT[c.col] = st;
        if (CHAIN) return;
    }
    if (hT && c.has && wave == 0) hT[c.col] = carry;
}

// As k_scan_fwd from the last run to the first: c, what later positions give a
// position's G, goes through a run as c -> A c + H.  The states inside the run
// come from the one kept before it.
template <typename T, typename X, int W, bool RAGGED, bool CHAIN>
__global__ void __launch_bounds__(64 * W)
k_scan_bwd(ScanArgs a, Chain ch, const X *__restrict__ g, const uint16_t *__restrict__ gscale,
           const X *__restrict__ u, const uint16_t *__restrict__ uscale,
           const float *__restrict__ saved, const T *__restrict__ dh, const float *dhT,
           T *__restrict__ dg, T *__restrict__ du, float *dh0)
{
    __shared__ float2 lds[CHAIN ? 1 : 2][W > 1 ? W : 1][64];
    __shared__ float start[64];
    const int lane = threadIdx.x & 63, wave = W > 1 ? threadIdx.x / 64 : 0;
    int chunk = 0, block = blockIdx.x;
    if (CHAIN) take_chunk(ch, chunk, block);
    const Column c = column_of(a, (long long)block * 64 + lane);
    float carry = !CHAIN && dhT ? dhT[c.col] : 0.0f;
    int turn = 0;
    // wave 0 has the last run of a chunk; a chunk's runs may end before the first
    for (long long r0 = a.runs - 1 - (long long)chunk * W; r0 >= 0; r0 -= W, turn ^= 1) {
        const long long run = r0 - wave, s0 = run * kRun;
        const int count = run >= 0 ? (int)min((long long)kRun, a.T - s0) : 0;
        const RunAt<RAGGED> at(a, c, s0);
        float f[kRun], k1[kRun], d[kRun], v[kRun];      // f, 1 - f, dh, h before - u
        float st = 0.0f;
        if (count > 0) {
            st = saved[c.saved + run * a.I];
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                const long long e = at.at(k < count ? k : count - 1);
                f[k] = load_at(g, gscale, e);
                v[k] = load_at(u, uscale, e);
                d[k] = Store<T>::load(dh, e);
            }
        }
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            const bool in = RAGGED ? k < at.live && k < count : k < count;
            gate(f[k], f[k], k1[k]);
            const float uk = v[k];
            v[k] = st - uk;
            st = in ? fmaf(f[k], st, k1[k] * uk) : st;
            f[k] = in ? f[k] : 1.0f;
            d[k] = in ? d[k] : 0.0f;
        }
        float cin = carry;
        if (W > 1) {
            float A = 1.0f, H = 0.0f;
#pragma unroll
            for (int k = kRun - 1; k >= 0; --k) {
                A *= f[k];
                H = f[k] * (d[k] + H);
            }
            lds[CHAIN ? 0 : turn][wave][lane] = make_float2(A, H);
            __syncthreads();
            const float2 (*parts)[64] = lds[CHAIN ? 0 : turn];
            if (CHAIN) {
                if (wave == 0) {
                    float ca = 1.0f, cb = 0.0f;
                    for (int w = 0; w < W; ++w) {
                        const float2 p = parts[w][lane];
                        ca *= p.x;
                        cb = fmaf(p.x, cb, p.y);
                    }
                    start[lane] = chained(ch, a.cols, c.col, c.has, chunk, ca, cb);
                }
                __syncthreads();
                carry = start[lane];
            }
            cin = fold(parts, wave, lane, carry);
        }
        if (count > 0) {
#pragma unroll
            for (int k = kRun - 1; k >= 0; --k) {
                const bool in = !RAGGED || k < at.live;
                const float G = d[k] + cin;
                const float vu = G * k1[k];
                if (k < count && c.has) {
                    Store<T>::store(dg, at.at(k), in ? vu * f[k] * v[k] : 0.0f);
                    Store<T>::store(du, at.at(k), in ? vu : 0.0f);
                }
                cin = f[k] * G;
            }
        }
        if (W == 1) carry = cin;
        else if (!CHAIN) carry = fold(lds[turn] + wave, W - wave, lane, fold(lds[turn], wave, lane, carry));
        else if (dh0 && c.has && run == 0) dh0[c.col] = cin;
        if (CHAIN) return;
    }
    if (dh0 && c.has && wave == 0) dh0[c.col] = carry;
}

int check_scan(int64_t B, int64_t T, int64_t I, int32_t dtype)
{
    if (B < 1 || T < 1 || I < 1) return PLSTM_EINVAL;
    if (dtype != PLSTM_F32 && dtype != PLSTM_BF16) return PLSTM_EINVAL;
    if (B > (1LL << 30) || T > (1LL << 31) || I > (1LL << 30)) return PLSTM_EUNSUPPORTED;
    if (B > (1LL << 30) / I || T > (1LL << 38) / (B * I)) return PLSTM_EUNSUPPORTED;
    return PLSTM_OK;
}

constexpr int kWaves = 8;           // of a workgroup with more than one

// How a call is spread: waves of a workgroup, and whether chunks are chained.
struct Plan {
    ScanArgs a;
    int waves;
    Chain ch;                       // chunks 0: none
    size_t ws;
};

Plan scan_plan(int64_t B, int64_t T, int64_t I, int32_t reverse, const int32_t *lengths, void *ws)
{
    Plan p{};
    p.a = ScanArgs{T, I, B * I, reverse, lengths, (T + kRun - 1) / kRun};
    const long long blocks = (p.a.cols + 63) / 64;
    const long long chunks = (p.a.runs + kWaves - 1) / kWaves;
    p.waves = blocks >= 1024 || p.a.runs <= 2 ? 1 : kWaves;
    Carve cv(ws);
    if (p.waves > 1 && chunks > 1 && blocks < 256 && chunks * blocks <= (1 << 21)) {
        p.ch.agg = cv.take<uint64_t>(chunks * p.a.cols);
        p.ch.state = cv.take<uint32_t>((chunks + kGroup - 1) / kGroup * p.a.cols);
        p.ch.ticket = cv.take<uint32_t>(1);
        p.ch.chunks = (int)chunks;
        p.ch.blocks = (int)blocks;
        p.ch.spin = g_wait_spin_limit;
        p.ch.bias = g_wait_bias;
    }
    p.ws = align_up(cv.off, 256);
    if (p.ws < 256) p.ws = 256;
    return p;
}

// Empties the chain's words and lays down the state before the first chunk.
int start_chain(Plan &p, const float *start, hipStream_t st)
{
    p.ch.status = device_status_word();
    if (!p.ch.status) return PLSTM_EHIP;
    const long long n = p.ch.chunks * p.a.cols;
    k_scan_chain_init<<<(unsigned)min((n + 255) / 256, 2048LL), 256, 0, st>>>(p.ch, p.a.cols, start);
    PLSTM_LAUNCH_CHECK();
    return PLSTM_OK;
}

template <typename T, int W, bool RAGGED, bool CHAIN>
void launch_fwd(const Plan &p, const void *g, const void *u, const void *h0, void *h, void *hT,
                void *saved, hipStream_t st)
{
    const long long blocks = (p.a.cols + 63) / 64;
    k_scan_fwd<T, W, RAGGED, CHAIN><<<(unsigned)(CHAIN ? blocks * p.ch.chunks : blocks), 64 * W, 0, st>>>(
        p.a, p.ch, (const T *)g, (const T *)u, (const float *)h0, (T *)h, (float *)hT,
        (float *)saved);
}

template <typename T, bool RAGGED>
int scan_forward(Plan &p, const void *g, const void *u, const void *h0, void *h, void *hT,
                 void *saved, hipStream_t st)
{
    if (p.ch.chunks) {
        const int rc = start_chain(p, (const float *)h0, st);
        if (rc != PLSTM_OK) return rc;
        launch_fwd<T, kWaves, RAGGED, true>(p, g, u, h0, h, hT, saved, st);
    } else if (p.waves > 1) {
        launch_fwd<T, kWaves, RAGGED, false>(p, g, u, h0, h, hT, saved, st);
    } else {
        launch_fwd<T, 1, RAGGED, false>(p, g, u, h0, h, hT, saved, st);
    }
    PLSTM_LAUNCH_CHECK();
    return PLSTM_OK;
}

template <typename T, typename X, int W, bool RAGGED, bool CHAIN>
void launch_bwd(const Plan &p, const void *g, const void *gscale, const void *u,
                const void *uscale, const void *saved, const void *dh, const void *dhT, void *dg,
                void *du, void *dh0, hipStream_t st)
{
    const long long blocks = (p.a.cols + 63) / 64;
    k_scan_bwd<T, X, W, RAGGED, CHAIN><<<(unsigned)(CHAIN ? blocks * p.ch.chunks : blocks), 64 * W, 0, st>>>(
        p.a, p.ch, (const X *)g, (const uint16_t *)gscale, (const X *)u, (const uint16_t *)uscale,
        (const float *)saved, (const T *)dh, (const float *)dhT, (T *)dg, (T *)du, (float *)dh0);
}

template <typename T, typename X, bool RAGGED>
int scan_backward(Plan &p, const void *g, const void *gscale, const void *u, const void *uscale,
                  const void *saved, const void *dh, const void *dhT, void *dg, void *du,
                  void *dh0, hipStream_t st)
{
    if (p.ch.chunks) {
        const int rc = start_chain(p, (const float *)dhT, st);
        if (rc != PLSTM_OK) return rc;
        launch_bwd<T, X, kWaves, RAGGED, true>(p, g, gscale, u, uscale, saved, dh, dhT, dg, du, dh0, st);
    } else if (p.waves > 1) {
        launch_bwd<T, X, kWaves, RAGGED, false>(p, g, gscale, u, uscale, saved, dh, dhT, dg, du, dh0, st);
    } else {
        launch_bwd<T, X, 1, RAGGED, false>(p, g, gscale, u, uscale, saved, dh, dhT, dg, du, dh0, st);
    }
    PLSTM_LAUNCH_CHECK();
    return PLSTM_OK;
}

}  // namespace
}  // namespace plstm

using namespace plstm;

extern "C" {

size_t pyramid_scan_saved_size(int64_t B, int64_t T, int64_t I)
{
    if (check_scan(B, T, I, PLSTM_F32) != PLSTM_OK) return 0;
    return align_up((size_t)B * ((T + kRun - 1) / kRun) * I * sizeof(float), 256);
}

size_t pyramid_scan_workspace_size(int64_t B, int64_t T, int64_t I)
{
    if (check_scan(B, T, I, PLSTM_F32) != PLSTM_OK) return 0;
    return scan_plan(B, T, I, 0, nullptr, nullptr).ws;
}

int pyramid_scan_forward(int64_t B, int64_t T, int64_t I, int32_t dtype, int32_t reverse,
                         const void *g, const void *u, const int32_t *lengths, const void *h0,
                         void *h, void *hT, void *saved, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_scan(B, T, I, dtype);
    if (rc != PLSTM_OK) return rc;
    if ((reverse != 0 && reverse != 1) || !g || !u || !h || !ws) return PLSTM_EINVAL;
    const size_t e = dtype_size(dtype);
    if (!aligned_to(g, e) || !aligned_to(u, e) || !aligned_to(lengths, 4) || !aligned_to(h0, 4) ||
        !aligned_to(h, e) || !aligned_to(hT, 4) || !aligned_to(saved, 16) || !aligned_to(ws, 16))
        return PLSTM_EINVAL;
    if (ws_bytes < pyramid_scan_workspace_size(B, T, I)) return PLSTM_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    Plan p = scan_plan(B, T, I, reverse, lengths, ws);
    timing_begin("scan_fwd", st);
    rc = dtype == PLSTM_F32
             ? (lengths ? scan_forward<float, true> : scan_forward<float, false>)(p, g, u, h0, h, hT,
                                                                                  saved, st)
             : (lengths ? scan_forward<uint16_t, true> : scan_forward<uint16_t, false>)(
                   p, g, u, h0, h, hT, saved, st);
    if (rc == PLSTM_OK) timing_end(p.ch.chunks ? 2 : 1, st);
    return rc;
}

int pyramid_scan_backward(int64_t B, int64_t T, int64_t I, int32_t dtype, int32_t reverse,
                          const void *g, const void *gscale, const void *u, const void *uscale,
                          const int32_t *lengths, const void *saved, const void *dh,
                          const void *dhT, void *dg, void *du, void *dh0, void *ws,
                          size_t ws_bytes, void *stream)
{
    int rc = check_scan(B, T, I, dtype);
    if (rc != PLSTM_OK) return rc;
    if ((reverse != 0 && reverse != 1) || !g || !u || !saved || !dh || !dg || !du || !ws ||
        !gscale != !uscale)
        return PLSTM_EINVAL;
    const size_t e = dtype_size(dtype), in = gscale ? 16 : e;
    if (!aligned_to(g, in) || !aligned_to(gscale, 16) || !aligned_to(u, in) ||
        !aligned_to(uscale, 16) || !aligned_to(lengths, 4) || !aligned_to(saved, 16) ||
        !aligned_to(dh, e) || !aligned_to(dhT, 4) || !aligned_to(dg, e) || !aligned_to(du, e) ||
        !aligned_to(dh0, 4) || !aligned_to(ws, 16))
        return PLSTM_EINVAL;
    if (ws_bytes < pyramid_scan_workspace_size(B, T, I)) return PLSTM_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    Plan p = scan_plan(B, T, I, reverse, lengths, ws);
    timing_begin("scan_bwd", st);
    const auto run = [&](auto fn) {
        return fn(p, g, gscale, u, uscale, saved, dh, dhT, dg, du, dh0, st);
    };
    if (dtype == PLSTM_F32) {
        if (gscale) rc = run(lengths ? scan_backward<float, int8_t, true> : scan_backward<float, int8_t, false>);
        else rc = run(lengths ? scan_backward<float, float, true> : scan_backward<float, float, false>);
    } else {
        if (gscale) rc = run(lengths ? scan_backward<uint16_t, int8_t, true> : scan_backward<uint16_t, int8_t, false>);
        else rc = run(lengths ? scan_backward<uint16_t, uint16_t, true> : scan_backward<uint16_t, uint16_t, false>);
    }
    if (rc == PLSTM_OK) timing_end(p.ch.chunks ? 2 : 1, st);
    return rc;
}

}  // extern "C"
