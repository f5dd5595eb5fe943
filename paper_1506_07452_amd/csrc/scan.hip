// Gated linear recurrence along an axis, and its backward pass.  Over a
// sequence of T steps and I channels, position s = 0 .. n - 1 of the sweep being
// step t = s, or n - 1 - s in reverse (n the sequence's length):
//   f = sigmoid(g_t),  h_s = f h_{s-1} + (1 - f) u_t,  h_{-1} = h0
// Backward, G_s the gradient of h_s:
//   G_s = dh_t + f_{s+1} G_{s+1}  (the last one takes dhT as well)
//   du_t = (1 - f) G_s,  dg_t = G_s (h_{s-1} - u_t) f (1 - f),  dh0 = f_0 G_0
// States and gradients of states are fp32.  1 - f is sigmoid(-g), not a
// difference: what a gate takes keeps its bits however little it is.  f itself is rounded
// next to 1, so a step that keeps the state is off by up to 2^-23 of it, always the same
// way under a constant gate (g = 15: a state of 1 fed with 1 is 0.996 after 65536 steps).
// Folding 1 - f instead would mend that and lose states that are infinite (0 times infinity
// where f = 1).
// A training forward keeps the state before every 16th position; the backward
// computes the others again from g and u (in the storage type or from 8-bit
// checkpoints), which costs 1/4 byte an element where reading h would cost 2
// or 4.
#include "rows.h"
#include "sweep.h"
#include "timing.h"

namespace plstm {
namespace {

constexpr int kChainWaves = 16;     // waves of a chained workgroup, at most
constexpr int kRun = 16;            // positions between kept states, and of a wave's run
constexpr int kGroup = 16;          // chunks between chained states, at least
constexpr uint64_t kEmpty = ~0ull;  // a word that its chunk has not written
constexpr uint32_t kEmptyState = ~0u;

struct ScanArgs {
    long long T, I, cols;           // steps, channels, B I
    int reverse;
    const int32_t *lengths;
    long long runs;                 // ceil(T / kRun)
    long long across;               // workgroups across a sequence's channels; 0: 64 columns
                                    // each, whatever sequences they belong to
};

// Chunks of a sequence (kRun positions for each wave of a workgroup) run at the
// same time and hand the state on through memory:
//   agg [chunk][cols]   (A, H) of a chunk: its last state is A (state before) + H
//   state [group][cols] the state before every group of chunks
// A word is written whole, so whoever finds it other than empty has it all: no
// flag, no fence.  A chunk publishes its aggregate as soon as it has its inputs;
// it then needs its group's state and the aggregates of the chunks before it in
// the group, always folded in the same order, so results do not depend on which
// chunk was faster.  Only the last chunk of a group waits on a chain, whose links
// take about 2 us each.
struct Chain {
    uint64_t *agg;
    uint32_t *state;
    uint32_t *ticket;               // chunks are taken in order: whoever waits, waits on started ones
    int *status;                    // device status word
    int chunks, blocks;             // chunks of a sequence, workgroups across the columns
    int group;                      // chunks of a group
    int spin, bias;                 // polls before a wait gives up; test mode
};

// Empties the words before each chained launch: 2.5 to 5 us.
__global__ void __launch_bounds__(256)
k_scan_chain_init(Chain ch, long long cols, const float *start)
{
    const long long i0 = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long stride = (long long)gridDim.x * 256;
    const long long na = ch.chunks * cols, ns = (ch.chunks + ch.group - 1) / ch.group * cols;
    for (long long i = i0; i < na; i += stride) ch.agg[i] = kEmpty;
    for (long long i = i0; i < ns; i += stride) {
        const float v = i < cols && start ? start[i] : 0.0f;
        ch.state[i] = i >= cols ? kEmptyState : v != v ? 0x7fc00000u : float_bits(v);
    }
    if (i0 == 0) *ch.ticket = 0;
}

// f and 1 - f of sigmoid's argument.  exp(-|g|) <= 1: nothing overflows, and
// neither is a difference (their sum is 1 to 2^-23).
__device__ inline void gate(float g, float &keep, float &take)
{
    const float e = __builtin_amdgcn_exp2f(fabsf(g) * -1.44269504f);
    const float r = __builtin_amdgcn_rcpf(1.0f + e);
    const float small = e * r;
    keep = g < 0.0f ? small : r;
    take = g < 0.0f ? r : small;
}

// A workgroup's 64 columns (channels of sequences) and a lane's among them.
// Element (b, t, i) of the lane is element `base` + off + t I: base is the same
// for the workgroup, so that addresses are a scalar pointer and a lane's 32-bit
// offset (the host keeps offsets below 2^32 bytes, scan_plan).
struct Column {
    bool has;                       // false past the last column (then a copy of it)
    bool one;                       // all columns of the workgroup are of one sequence
    long long base, saved, first;   // of the first column: element (b, 0, i), state (b, 0, i), column
    uint32_t off, soff, coff;       // the lane's, from those
    long long n;                    // the sequence's length
};
__device__ inline Column column_of(const ScanArgs &a, int block, int lane)
{
    Column c;
    long long b;
    uint32_t i, last;
    if (a.across) {
        b = (uint32_t)block / (uint32_t)a.across;
        i = (uint32_t)(block - b * a.across) * 64;
        last = (uint32_t)a.I - 1 - i;
        c.first = b * a.I + i;
    } else {
        c.first = (long long)block * 64;
        b = (uint32_t)c.first / (uint32_t)a.I;
        i = (uint32_t)(c.first - b * a.I);
        last = (uint32_t)min(a.cols - 1 - c.first, 63LL);
    }
    c.has = lane <= (int)min(last, 63u);
    c.one = i + min(last, 63u) < (uint32_t)a.I;
    c.coff = min((uint32_t)lane, last);
    const uint32_t at = i + c.coff, I = (uint32_t)a.I;
    const uint32_t db = a.across ? 0 : at / I, di = at - db * I - i;
    c.base = b * a.T * a.I + i;
    c.saved = b * a.runs * a.I + i;
    c.off = db * (uint32_t)(a.T * a.I) + di;
    c.soff = db * (uint32_t)(a.runs * a.I) + di;
    c.n = a.T;
    if (a.lengths) {
        const long long n = a.lengths[b + db];
        c.n = n < 0 ? 0 : n > a.T ? a.T : n;
    }
    return c;
}

// Element offset of a lane from a uniform one: 32 bits where all sequences have
// the same length, else 64 (positions count from each sequence's end).
template <bool RAGGED> struct Offset { typedef uint32_t type; };
template <> struct Offset<true> { typedef long long type; };

// Loads give raw bits.
template <typename O>
__device__ inline uint32_t get(const float *p, long long base, O off)
{
    return *(const uint32_t *)((const char *)(p + base) + (O)(off * 4));
}
template <typename O>
__device__ inline uint32_t get(const uint16_t *p, long long base, O off)
{
    return *(const uint16_t *)((const char *)(p + base) + (O)(off * 2));
}
template <typename O>
__device__ inline uint32_t get(const int8_t *p, long long base, O off)
{
    return (uint32_t)(int)*(const int8_t *)((const char *)(p + base) + off);
}
template <typename X> __device__ inline float value(uint32_t raw);
template <> __device__ inline float value<float>(uint32_t raw) { return bits_float(raw); }
template <> __device__ inline float value<uint16_t>(uint32_t raw) { return bits_float(raw << 16); }
template <> __device__ inline float value<int8_t>(uint32_t raw) { return (float)(int)raw; }
// Raw scale of a code.
template <typename O>
__device__ inline uint32_t get_scale(const uint16_t *scale, long long base, O off)
{
    const O block = ((O)(base & (kCodeBlock - 1)) + off) >> 6;
    return *(const uint16_t *)((const char *)(scale + (base >> 6)) + (O)(block * 2));
}

// Scales of a run of a coded tensor where a workgroup's columns are of one
// sequence: a position's 64 elements, consecutive from `first` + k step, lie in two blocks
// at most.  Lane k has the scale of the first one of position k, lane 16 + k of
// the second: one load instead of one a position.
struct RunScales {
    uint32_t s;
    long long first, step;
    __device__ RunScales(const uint16_t *scale, long long blocks, long long first_, long long step_,
                         int lane)
        : first(first_), step(step_)
    {
        const long long b = ((first + (lane & 15) * step) >> 6) + (lane >> 4 & 1);
        s = scale[b < blocks ? b : blocks - 1];
    }
    __device__ float of(int k, int lane) const
    {
        const uint32_t s0 = (uint32_t)__builtin_amdgcn_readlane((int)s, k);
        const uint32_t s1 = (uint32_t)__builtin_amdgcn_readlane((int)s, 16 + k);
        const int turn = kCodeBlock - (int)((first + k * step) & (kCodeBlock - 1));
        return bits_float((lane < turn ? s0 : s1) << 16);
    }
};

template <typename O>
__device__ inline void put(float *p, long long base, O off, float v)
{
    *(float *)((char *)(p + base) + (O)(off * 4)) = v;
}
template <typename O>
__device__ inline void put(uint16_t *p, long long base, O off, float v)
{
    *(uint16_t *)((char *)(p + base) + (O)(off * 2)) = (uint16_t)pack_bf16(v, v);
}

// The elements of a run of positions s0 .. s0 + count - 1 of a column.  Positions
// past a sequence's length stand for the steps of the same number.
template <bool RAGGED>
struct RunAt {
    typedef typename Offset<RAGGED>::type O;
    long long base, step;           // position k: base + k step, from the lane's `off`
    O off;
    long long pbase, pstep;         // the same for positions past the length
    O poff;
    int live;                       // positions of the run that the sequence has
    __device__ RunAt(const ScanArgs &a, const Column &c, long long s0)
    {
        const long long end = RAGGED ? 0 : a.T - 1;
        base = c.base + (a.reverse ? end - s0 : s0) * a.I;
        step = a.reverse ? -a.I : a.I;
        off = RAGGED && a.reverse ? (O)(c.off + (c.n - 1) * a.I) : (O)c.off;
        pbase = c.base + s0 * a.I;
        pstep = a.I;
        poff = (O)c.off;
        const long long left = c.n - s0;
        live = left < 0 ? 0 : left > kRun ? kRun : (int)left;
    }
    // Where position k is, and how far the lane from there: of a run that every lane
    // has in full, and of any (`count` > 0 positions are the tensor's, `live` of
    // them the sequence's; others stand for some place that there is).
    __device__ long long from(int k) const { return base + k * step; }
    __device__ void any(int k, int count, long long &b, O &o) const
    {
        const int j = k < count ? k : count - 1;
        if (RAGGED) {
            b = 0;
            o = (O)(j < live ? base + j * step + off : pbase + j * pstep + poff);
        } else {
            b = base + j * step;
            o = off;
        }
    }
    __device__ bool has(int k, int count) const { return k < count && k < live; }
    template <typename T> __device__ void store(T *x, int k, float v) const
    {
        put(x, base + k * step, off, v);
    }
    // 0 where the sequence has no position k
    template <typename T> __device__ void store(T *x, int k, int count, float v) const
    {
        if (k >= count) return;
        long long b;
        O o;
        any(k, count, b, o);
        put(x, b, o, k < live ? v : 0.0f);
    }
};

// Waits for a word of the chain to be written; false when it gave up.
template <typename V>
__device__ inline bool wait_word(const Chain &ch, const V *p, V empty, V &v)
{
    for (int polls = 0;; ++polls) {
        v = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (__all(v != empty && ch.bias == 0)) return true;
        if (polls >= ch.spin) {
            if ((threadIdx.x & 63) == 0)
                __hip_atomic_fetch_or(ch.status, PLSTM_DEVICE_WAIT_GAVE_UP, __ATOMIC_RELAXED,
                                      __HIP_MEMORY_SCOPE_AGENT);
            return false;
        }
        __builtin_amdgcn_s_sleep(1);
    }
}

// The next chunk of the chain: its number, and the workgroup's place across the columns.
__device__ inline void take_chunk(const Chain &ch, int &chunk, int &block)
{
    __shared__ uint32_t ticket;
    if (threadIdx.x == 0)
        ticket = __hip_atomic_fetch_add(ch.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const uint32_t t = (uint32_t)__builtin_amdgcn_readfirstlane((int)ticket);
    chunk = (int)(t / (uint32_t)ch.blocks);
    block = (int)(t - (uint32_t)chunk * (uint32_t)ch.blocks);
}

// What the waves of a workgroup give each other: (A, H) of their runs, and
// (CHAIN) of the chunks before it in its group and the group's state.
template <int W, bool CHAIN>
struct Shared {
    float2 part[CHAIN ? 1 : 2][W][64];      // two turns: one barrier a turn
    float2 prev[CHAIN ? W : 1][64];
    float start[64];
};

// The state before the wave's run, `carry` being the one before the workgroup's
// first (CHAIN: taken from the chain); carry becomes the one after its last.
// Every wave of the workgroup is here at once.  U: steps of the folds at a time, which
// decides the registers.
template <int W, bool CHAIN, int U>
__device__ inline float before_run(Shared<W, CHAIN> &sh, int turn, const Chain &ch, long long cols,
                                   const Column &c, int chunk, int wave, int lane, float A, float H,
                                   float &carry)
{
    const float2 (*part)[64] = sh.part[CHAIN ? 0 : turn];
    sh.part[CHAIN ? 0 : turn][wave][lane] = make_float2(A, H);
    __syncthreads();
    if (CHAIN) {
        const int g = chunk / ch.group, first = g * ch.group, share = ch.group / W;
        if (wave == 0 && chunk + 1 < ch.chunks) {
            float a = 1.0f, h = 0.0f;
#pragma unroll U
            for (int w = 0; w < W; ++w) {
                const float2 p = part[w][lane];
                a *= p.x;
                h = fmaf(p.x, h, p.y);
            }
            const uint64_t word = (uint64_t)float_bits(h) << 32 |
                                  (a != a ? 0x7fc00000u : float_bits(a));
            if (c.has)
                __hip_atomic_store(ch.agg + (chunk * cols + c.first) + c.coff, word,
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        // each wave takes its share of the chunks before
        float a = 1.0f, h = 0.0f;
        for (int k = first + wave * share; k < min(first + (wave + 1) * share, chunk); ++k) {
            uint64_t w;
            const bool ok = wait_word(ch, ch.agg + (k * cols + c.first) + c.coff, kEmpty, w);
            const float wa = ok ? bits_float((uint32_t)w) : __builtin_nanf("");
            a *= wa;
            h = fmaf(wa, h, bits_float((uint32_t)(w >> 32)));
        }
        sh.prev[wave][lane] = make_float2(a, h);
        if (wave == W - 1) {
            uint32_t s;
            const bool ok = wait_word(ch, ch.state + (g * cols + c.first) + c.coff, kEmptyState, s);
            sh.start[lane] = ok ? bits_float(s) : __builtin_nanf("");
        }
        __syncthreads();
        carry = sh.start[lane];
#pragma unroll U
        for (int w = 0; w < W; ++w) {
            const float2 p = sh.prev[w][lane];
            carry = fmaf(p.x, carry, p.y);
        }
    }
    float v = carry, at = carry;
#pragma unroll U
    for (int w = 0; w < W; ++w) {
        const float2 p = part[w][lane];
        at = w == wave ? v : at;
        v = fmaf(p.x, v, p.y);
    }
    carry = v;
    if (CHAIN && wave == 0 && (chunk + 1) % ch.group == 0 && chunk + 1 < ch.chunks && c.has)
        __hip_atomic_store(ch.state + ((chunk + 1) / ch.group * cols + c.first) + c.coff,
                           v != v ? 0x7fc00000u : float_bits(v), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
    return at;
}

// Bound by bytes where columns fill the card (11520 x 240 x 16 fp32 in 110 us, 4.8 TB/s; 64 x 512
// x 512 bf16 in 20 us, 5.1 TB/s), in chains by their phases (2 x 8192 x 2048 fp32 in 88 us, 4.6 TB/s;
// 65536 x 1024 bf16 in 95 to 100 us, 4.0 to 4.2 TB/s; 4096 x 512 in about 10 us with the clearing launch).
// A workgroup of W waves advances 64 columns by W runs of 16 positions at a
// time, wave w holding run w in registers.  W = 1 walks its runs one after
// another; with more, each wave folds its run to (A, H), and starts it again from
// the state that the waves before it leave.  CHAIN: the workgroup has one chunk
// of W runs and takes the state from the chain.  Runs that every lane has in full
// are loaded and stored without a condition.
template <typename T, int W, bool RAGGED, bool CHAIN>
__global__ void __launch_bounds__(64 * W)
k_scan_fwd(ScanArgs a, Chain ch, const T *__restrict__ g, const T *__restrict__ u,
           const float *h0, T *__restrict__ h, float *hT, float *__restrict__ saved)
{
    // bf16: folds by four keep a chained chunk to 64 registers, two workgroups a CU
    // (65536 steps of 1024 channels 116 -> 101 us); fp32 has as many bytes on the
    // way with one (16384 steps of 1024 channels 48 us, with two 54)
    constexpr int folds = CHAIN && sizeof(T) == 2 ? 4 : W;
    __shared__ Shared<W, CHAIN> sh;
    const int lane = threadIdx.x & 63;
    const int wave = W > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0;
    int chunk = 0, block = blockIdx.x, turn = 0;
    if (CHAIN) take_chunk(ch, chunk, block);
    const Column c = column_of(a, block, lane);
    float carry = !CHAIN && h0 ? h0[c.first + c.coff] : 0.0f;
    for (long long r0 = (long long)chunk * W; r0 < a.runs; r0 += W, turn ^= 1) {
        const long long run = r0 + wave, s0 = run * kRun;
        const int count = run < a.runs ? (int)min((long long)kRun, a.T - s0) : 0;
        const RunAt<RAGGED> at(a, c, s0);
        const bool full = count == kRun && (!RAGGED || __all(at.live == kRun));
        const bool any = count > 0 && (!RAGGED || !__all(at.live == 0));
        float f[kRun], v[kRun];
        if (full) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                f[k] = value<T>(get(g, at.from(k), at.off));
                v[k] = value<T>(get(u, at.from(k), at.off));
            }
        } else {
            // a position that is not there keeps the state: f = 1, nothing taken
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                f[k] = __builtin_inff();
                v[k] = 0.0f;
            }
            if (any) {
#pragma unroll
                for (int k = 0; k < kRun; ++k) {
                    long long b;
                    typename RunAt<RAGGED>::O o;
                    at.any(k, count, b, o);
                    const float fk = value<T>(get(g, b, o)), vk = value<T>(get(u, b, o));
                    f[k] = at.has(k, count) ? fk : __builtin_inff();
                    v[k] = at.has(k, count) ? vk : 0.0f;
                }
            }
        }
        float A = 1.0f, H = 0.0f;
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            float take;
            gate(f[k], f[k], take);
            v[k] *= take;
            if (W > 1) {
                A *= f[k];
                H = fmaf(f[k], H, v[k]);
            }
        }
        float st = carry;
        if constexpr (W > 1)
            st = before_run<W, CHAIN, folds>(sh, turn, ch, a.cols, c, chunk, wave, lane, A, H, carry);
        if (saved && count > 0 && c.has) put(saved, c.saved + run * a.I, c.soff, st);
        if (full && c.has) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                st = fmaf(f[k], st, v[k]);
                at.store(h, k, st);
            }
        } else if (c.has) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                st = fmaf(f[k], st, v[k]);
                at.store(h, k, count, st);
            }
        }
        if (W == 1) carry = st;
        if (CHAIN) break;
    }
    if (hT && c.has && wave == 0 && (!CHAIN || chunk == ch.chunks - 1)) hT[c.first + c.coff] = carry;
}

// g and u of a full run from their codes.
template <bool RAGGED>
__device__ inline void coded_run(const ScanArgs &a, const RunAt<RAGGED> &at, const Column &c,
                                 int lane, const int8_t *g, const uint16_t *gscale,
                                 const int8_t *u, const uint16_t *uscale, float *f, float *v)
{
    uint32_t rg[kRun], ru[kRun];
    if (c.one) {
        // the lanes of a sequence are as far from its end
        const long long first =
            at.base + (RAGGED ? (long long)__builtin_amdgcn_readfirstlane((int)((long long)at.off >> 32)) << 32 |
                                    (uint32_t)__builtin_amdgcn_readfirstlane((int)at.off)
                              : 0);
        const long long blocks = (a.cols * a.T + kCodeBlock - 1) / kCodeBlock;
        const RunScales sg(gscale, blocks, first, at.step, lane);
        const RunScales su(uscale, blocks, first, at.step, lane);
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            rg[k] = get(g, at.from(k), at.off);
            ru[k] = get(u, at.from(k), at.off);
        }
        loads_issued();
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            f[k] = value<int8_t>(rg[k]) * sg.of(k, lane);
            v[k] = value<int8_t>(ru[k]) * su.of(k, lane);
        }
    } else {
        uint32_t sg[kRun], su[kRun];
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            rg[k] = get(g, at.from(k), at.off);
            ru[k] = get(u, at.from(k), at.off);
            sg[k] = get_scale(gscale, at.from(k), at.off);
            su[k] = get_scale(uscale, at.from(k), at.off);
        }
        loads_issued();
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            f[k] = value<int8_t>(rg[k]) * value<uint16_t>(sg[k]);
            v[k] = value<int8_t>(ru[k]) * value<uint16_t>(su[k]);
        }
    }
}

// Bound by bytes: 11520 x 240 x 16 fp32 in 175 us (5.1 TB/s), 2 x 8192 x 2048 fp32, chained, in 124
// us (5.5 TB/s), 65536 x 1024 bf16, chained, in 160 us (4.3 TB/s).
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
    constexpr bool coded = sizeof(X) == 1;
    __shared__ Shared<W, CHAIN> sh;
    const int lane = threadIdx.x & 63;
    const int wave = W > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0;
    int chunk = 0, block = blockIdx.x, turn = 0;
    if (CHAIN) take_chunk(ch, chunk, block);
    const Column c = column_of(a, block, lane);
    float carry = !CHAIN && dhT ? dhT[c.first + c.coff] : 0.0f;
    // wave 0 has the last run of a chunk; a chunk's runs may end before the first
    for (long long r0 = a.runs - 1 - (long long)chunk * W; r0 >= 0; r0 -= W, turn ^= 1) {
        const long long run = r0 - wave, s0 = run * kRun;
        const int count = run >= 0 ? (int)min((long long)kRun, a.T - s0) : 0;
        const RunAt<RAGGED> at(a, c, s0);
        const bool full = count == kRun && (!RAGGED || __all(at.live == kRun));
        const bool any = count > 0 && (!RAGGED || !__all(at.live == 0));
        float f[kRun], k1[kRun], d[kRun], v[kRun];      // f, 1 - f, dh, h before - u
        float st = 0.0f;
        if (count > 0) st = value<float>(get(saved, c.saved + run * a.I, c.soff));
        if (full) {
            if constexpr (coded) {
                coded_run(a, at, c, lane, g, gscale, u, uscale, f, v);
            } else {
#pragma unroll
                for (int k = 0; k < kRun; ++k) {
                    f[k] = value<X>(get(g, at.from(k), at.off));
                    v[k] = value<X>(get(u, at.from(k), at.off));
                }
            }
#pragma unroll
            for (int k = 0; k < kRun; ++k) d[k] = value<T>(get(dh, at.from(k), at.off));
        } else {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                f[k] = __builtin_inff();
                v[k] = d[k] = 0.0f;
            }
            if (any) {
#pragma unroll
                for (int k = 0; k < kRun; ++k) {
                    long long b;
                    typename RunAt<RAGGED>::O o;
                    at.any(k, count, b, o);
                    float fk = value<X>(get(g, b, o)), vk = value<X>(get(u, b, o));
                    const float dk = value<T>(get(dh, b, o));
                    if constexpr (coded) {
                        fk *= value<uint16_t>(get_scale(gscale, b, o));
                        vk *= value<uint16_t>(get_scale(uscale, b, o));
                    }
                    f[k] = at.has(k, count) ? fk : __builtin_inff();
                    v[k] = at.has(k, count) ? vk : 0.0f;
                    d[k] = at.has(k, count) ? dk : 0.0f;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            gate(f[k], f[k], k1[k]);
            const float uk = v[k];
            v[k] = st - uk;
            st = fmaf(f[k], st, k1[k] * uk);
        }
        float cin = carry;
        if constexpr (W > 1) {
            float A = 1.0f, H = 0.0f;
#pragma unroll
            for (int k = kRun - 1; k >= 0; --k) {
                A *= f[k];
                H = f[k] * (d[k] + H);
            }
            cin = before_run<W, CHAIN, CHAIN && W == kChainWaves ? 4 : W>(sh, turn, ch, a.cols, c, chunk, wave, lane, A, H, carry);
        }
        if (full && c.has) {
#pragma unroll
            for (int k = kRun - 1; k >= 0; --k) {
                const float G = d[k] + cin, vu = G * k1[k];
                cin = f[k] * G;
                at.store(dg, k, vu * f[k] * v[k]);
                at.store(du, k, vu);
            }
        } else if (c.has) {
#pragma unroll
            for (int k = kRun - 1; k >= 0; --k) {
                const float G = d[k] + cin, vu = G * k1[k];
                cin = f[k] * G;
                at.store(dg, k, count, vu * f[k] * v[k]);
                at.store(du, k, count, vu);
            }
        }
        if (W == 1) carry = cin;
        if (CHAIN) break;
    }
    if (dh0 && c.has && wave == 0 && (!CHAIN || chunk == ch.chunks - 1))
        dh0[c.first + c.coff] = carry;
}

int check_scan(int64_t B, int64_t T, int64_t I, int32_t dtype)
{
    if (B < 1 || T < 1 || I < 1) return PLSTM_EINVAL;
    if (dtype != PLSTM_F32 && dtype != PLSTM_BF16) return PLSTM_EINVAL;
    if (B > (1LL << 30) || T > (1LL << 31) || I > (1LL << 30)) return PLSTM_EUNSUPPORTED;
    if (B > (1LL << 30) / I || T > (1LL << 38) / (B * I)) return PLSTM_EUNSUPPORTED;
    return PLSTM_OK;
}

// Waves of a workgroup by the runs of a sequence: one for a single run, four up to
// four, else eight (training along x of a 48 x 240 x 240 volume, fp32, 15 runs: 305 us with
// one, 286 with eight; 256 sequences of 4 runs of 2048 channels 257 with one, 212 with four).
constexpr int kWaves = 8, kFewWaves = 4;
// Waves of a chained chunk of the forward: sixteen, so half the links, and one
// workgroup a CU (bf16, 16384 steps of 1024 channels: 31 us; with eight, four
// workgroups a CU, 39).  The backward's registers leave room for one such workgroup a
// CU, or two of eight: sixteen while that is at most two rounds of the card (bf16, 4096
// steps of 2048 channels 28 -> 25 us), else eight (two sequences of 8192 steps 88 and 80).
constexpr long long kShortChain = 512;
// Columns from which a card is filled without chains: at 16384 (fp32, eight sequences of
// 2048 steps of 2048 channels) 88 us, 97 chained; at 4096 189 and 93.
constexpr long long kChainCols = 16384;

// How a call is spread: waves of a workgroup, and whether chunks are chained.
struct Plan {
    ScanArgs a;
    long long blocks;               // workgroups across the columns
    int waves, chain_waves;
    Chain ch;                       // chunks 0: none
    size_t ws;
};

Plan scan_plan(int64_t B, int64_t T, int64_t I, int32_t reverse, const int32_t *lengths, void *ws,
               bool backward)
{
    Plan p{};
    p.a = ScanArgs{T, I, B * I, reverse, lengths, (T + kRun - 1) / kRun, 0};
    p.blocks = (p.a.cols + 63) / 64;
    // a lane's offset from its workgroup's first column, in bytes of fp32: the
    // sequences that 64 columns touch.  Past 32 bits columns do not share workgroups
    // across sequences.
    if (B > 1 && (double)(63 / I + 1) * T * I >= (double)(1 << 30)) {
        p.a.across = (I + 63) / 64;
        p.blocks = B * p.a.across;
    }
    const long long few = (p.a.runs + kChainWaves - 1) / kChainWaves;
    p.chain_waves = backward && few * p.blocks > kShortChain ? kWaves : kChainWaves;
    const long long chunks = (p.a.runs + p.chain_waves - 1) / p.chain_waves;
    p.waves = p.a.runs == 1 ? 1 : p.a.runs <= kFewWaves ? kFewWaves : kWaves;
    // a launch has fewer than 2^32 work items: columns past that (2^29 of over 64 steps)
    // fill the card many times over with one wave each
    if (p.blocks * 64 * p.waves >= (1LL << 32)) p.waves = 1;
    Carve cv(ws);
    if (chunks > 1 && p.a.cols < kChainCols && chunks * p.blocks <= (1 << 21)) {
        p.ch.agg = cv.take<uint64_t>(chunks * p.a.cols);
        p.ch.state = cv.take<uint32_t>((chunks + kGroup - 1) / kGroup * p.a.cols);
        p.ch.ticket = cv.take<uint32_t>(1);
        p.ch.chunks = (int)chunks;
        p.ch.blocks = (int)p.blocks;
        // where links would take longer than the data, twice as many chunks a link
        // (bf16, 65536 steps of 256 channels, eight waves: 72 -> 50 us)
        p.ch.group = p.a.cols <= 512 ? 2 * kGroup : kGroup;
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
    k_scan_fwd<T, W, RAGGED, CHAIN><<<(unsigned)(CHAIN ? p.blocks * p.ch.chunks : p.blocks), 64 * W, 0, st>>>(
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
        launch_fwd<T, kChainWaves, RAGGED, true>(p, g, u, h0, h, hT, saved, st);
    } else if (p.waves == kWaves) {
        launch_fwd<T, kWaves, RAGGED, false>(p, g, u, h0, h, hT, saved, st);
    } else if (p.waves == kFewWaves) {
        launch_fwd<T, kFewWaves, RAGGED, false>(p, g, u, h0, h, hT, saved, st);
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
    k_scan_bwd<T, X, W, RAGGED, CHAIN><<<(unsigned)(CHAIN ? p.blocks * p.ch.chunks : p.blocks), 64 * W, 0, st>>>(
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
        if (p.chain_waves == kChainWaves)
            launch_bwd<T, X, kChainWaves, RAGGED, true>(p, g, gscale, u, uscale, saved, dh, dhT, dg, du, dh0, st);
        else
            launch_bwd<T, X, kWaves, RAGGED, true>(p, g, gscale, u, uscale, saved, dh, dhT, dg, du, dh0, st);
    } else if (p.waves == kWaves) {
        launch_bwd<T, X, kWaves, RAGGED, false>(p, g, gscale, u, uscale, saved, dh, dhT, dg, du, dh0, st);
    } else if (p.waves == kFewWaves) {
        launch_bwd<T, X, kFewWaves, RAGGED, false>(p, g, gscale, u, uscale, saved, dh, dhT, dg, du, dh0, st);
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
    const size_t f = scan_plan(B, T, I, 0, nullptr, nullptr, false).ws;
    const size_t b = scan_plan(B, T, I, 0, nullptr, nullptr, true).ws;
    return f > b ? f : b;
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
    Plan p = scan_plan(B, T, I, reverse, lengths, ws, false);
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
    Plan p = scan_plan(B, T, I, reverse, lengths, ws, true);
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
