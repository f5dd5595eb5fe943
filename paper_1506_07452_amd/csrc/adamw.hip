// AdamW over many tensors in one launch, moments in 32 bits or in 8.
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2          (rounded to fp32)
//   theta -= lr (m c1 / (sqrt(v c2) + eps) + decay theta),   c = 1 / (1 - b^t)
// 8-bit moments: blocks of 256 elements of a tensor share an fp32 scale, the block's
// largest |m| or v, and an element is the code of its ratio r to that:
//   m: sign, 4 bits of exponent, 3 of mantissa;  v: 5 and 3, no sign.  Codes from 8 on are
//   2^(k/8 - E) (1 + (k mod 8) / 8) with E = 15 or 31 (so 2^0 is the last one used, 120 or 248),
//   codes below 8 linear: k / 8 of the least of those.
// A moment moves by 1 - b of itself in a step, by far less than a code, so rounding to
// the nearest would hold it where it is.  16 random bits an element decide instead, the upper code with the
// probability of how near it is: the held moment is right on the average.  They are a hash of
// (seed, step, tensor, element), so a run is repeated bit for bit.  v is never rounded to
// 0 where it is not 0: m / sqrt(v) would explode.
// m and v are made in 64 bits (as fast as 32 here), each product and the sum rounded, and then
// rounded to fp32; ratios are 64-bit quotients: codes are a well-defined function of the inputs.
// Bound by bytes: 66 million bf16 gradients with 8-bit moments and bf16 copies, 16 bytes an element, 203 us (5.2 TB/s; with one
// block a wave 241), their moments as fp32 numbers, 10 bytes, 109 us (6.1 TB/s); 69 million fp32 gradients with 32-bit moments, 28 bytes,
// 355 us (5.5 TB/s).
#include <math.h>

#include "sequence.h"
#include "timing.h"

namespace plstm {
namespace {

constexpr int kAdamSegs = 48;               // tensors a launch: their pointers travel in its arguments
constexpr int kAdamBlock = 256;             // elements that share scales: 4 a lane of a wave
constexpr int kAdamTile = 8 * kAdamBlock;   // elements of a workgroup, two blocks a wave
constexpr long long kAdamMaxN = 1LL << 34;
constexpr long long kAdamMaxTiles = 1LL << 23;

struct AdamSeg {
    float *theta;
    const void *grad;
    void *m, *v;
    float *mscale, *vscale;
    uint16_t *copy;
    long long n;
    float decay;
    uint32_t id;                            // number of the tensor in the call
};

// What a step's number decides, on the device for steps in a captured graph.
struct Clock {
    long long t;
    float c1, c2;
    uint32_t key;
};

struct AdamArgs {
    int count;
    int start[kAdamSegs + 1];               // first tile of each tensor
    AdamSeg seg[kAdamSegs];
    double b1, b2;
    float lr, eps;
    Clock now;
    const Clock *clock;                     // instead of `now` where not NULL
    const float *lr_at;                     // instead of lr where not NULL
    const float *grad_scale;                // NULL: 1
};

// A published 32-bit integer hash, two rounds of xorshift and multiply (Wellons,
// "lowbias32").
__host__ __device__ inline uint32_t mix32(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x7feb352du;
    x = (x ^ (x >> 15)) * 0x846ca68bu;
    return x ^ (x >> 16);
}

__host__ __device__ inline Clock clock_at(long long t, double b1, double b2, uint32_t seed)
{
    Clock c;
    c.t = t;
    c.c1 = (float)(1.0 / (1.0 - pow(b1, (double)t)));
    c.c2 = (float)(1.0 / (1.0 - pow(b2, (double)t)));
    c.key = mix32(mix32(seed) + (uint32_t)t);
    return c;
}

__global__ void k_adamw_clock(Clock *c, double b1, double b2, uint32_t seed)
{
    *c = clock_at(c->t + 1, b1, b2, seed);
}

// The ratio of code k, its bits at 20 .. 27 of `code`: those of an fp32 number 2^(E - 127) times the
// ratio, whose subnormal numbers are the linear codes.
template <int E> __device__ inline float code_ratio(uint32_t code)
{
    return bits_float(code) * bits_float((uint32_t)(254 - E) << 23);
}

// Scale of a block from the bits of its largest magnitude (a NaN the largest of all): a block
// with an infinity or a NaN becomes NaN, so that moments never hide a divergence.
struct Narrow {
    double scale, inv;
    float stored;
    uint32_t keep;                          // of codes: none of a block of zeros or NaNs
    __device__ explicit Narrow(uint32_t top)
    {
        const bool none = top == 0 || top >= kInfBits;
        stored = top >= kInfBits ? __builtin_nanf("") : bits_float(top);
        scale = none ? 0.0 : (double)stored;
        inv = none ? 0.0 : 1.0 / scale;
        keep = none ? 0u : 255u;
    }
    // Code of |x| <= scale.  The quotient: a correctly rounded reciprocal, and a step of
    // Markstein's, which makes the correctly rounded quotient.
    template <int E> __device__ uint32_t code(float x, uint32_t random) const
    {
        const double a = fabs((double)x), q = a * inv;
        const double r = fma(fma(-q, scale, a), inv, q);
        // exponent, three bits of mantissa and 16 more of the ratio, those before code 8 in equal steps
        const uint64_t bits = __builtin_bit_cast(uint64_t, r);
        const uint32_t hi = (uint32_t)(bits >> 33);
        const uint32_t fine = hi - ((uint32_t)(1023 - E) << 19);
        const uint32_t low = (uint32_t)(r * (double)(1ull << (18 + E)));
        return ((hi < ((uint32_t)(1024 - E) << 19) ? low : fine) + random) >> 16 & keep;
    }
};

// b m + k g.  No fused product: 0.9 and 0.1 make (9 m + g) / 10, which falls next to the middle between two
// fp32 numbers for one element in some hundred, and there the last bit of 64 decides.
__device__ inline float blend(double b, float m, double k, double g)
{
#pragma clang fp contract(off)
    const double x = b * (double)m, y = k * g;
    return (float)(x + y);
}

// Elements 4 lane .. of a block: pointers start at any element (codes at 16 bytes).
template <typename T>
__device__ inline void load4(const T *p, int have, float *v)
{
    Four<T> w;
    w.load(p, have);
    w.get(v);
}
__device__ inline uint32_t load4_codes(const uint8_t *p, int have)
{
    if (have >= 4) return *(const uint32_t *)p;
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if (j < have) w |= (uint32_t)p[j] << (8 * j);
    return w;
}
template <bool STREAM>
__device__ inline void store4_codes(uint8_t *p, int have, const uint32_t *k)
{
    if (have >= 4) {
        const uint32_t w = k[0] | k[1] << 8 | k[2] << 16 | k[3] << 24;
        if (STREAM) __builtin_nontemporal_store(w, (uint32_t *)p);
        else *(uint32_t *)p = w;
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < have) p[j] = (uint8_t)k[j];
    }
}

__device__ inline void wide_m(uint32_t w, float scale, float *v)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t k = w << (24 - 8 * j);       // the code at the top, its sign in the sign's place
        const float f = code_ratio<15>(k >> 4 & 0x07f00000u) * scale;
        v[j] = bits_float((float_bits(f) & 0x7fffffffu) | (k & 0x80000000u));
    }
}
__device__ inline void wide_v(uint32_t w, float scale, float *v)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = code_ratio<31>((w >> (8 * j) & 255u) << 20) * scale;
}

// The tensor of a workgroup's tile, and the tile's first element in it.
__device__ inline int seg_of(const AdamArgs &a, long long &first)
{
    int lo = 0, hi = a.count - 1;           // last tensor with start <= tile
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.start[mid] <= (int)blockIdx.x) lo = mid; else hi = mid - 1;
    }
    first = (long long)((int)blockIdx.x - a.start[lo]) * kAdamTile;
    return lo;
}

// Elements of a lane's four from `at` on that a tensor of n has; WHOLE: the tile is inside it.
template <bool WHOLE>
__device__ inline int have_of(long long n, long long at)
{
    const long long left = n - at;
    return WHOLE ? 4 : left < 0 ? 0 : left > 4 ? 4 : (int)left;
}

template <int BITS, typename G, bool ROOT, bool STREAM, bool WHOLE>
__device__ inline void adamw_tile(const AdamArgs &a, const AdamSeg &s, long long first)
{
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const Clock now = a.clock ? *a.clock : a.now;
    const float lr = a.lr_at ? *a.lr_at : a.lr;
    const double gs = a.grad_scale ? (double)*a.grad_scale : 1.0;
    const uint32_t key = mix32(now.key + s.id);
    const double k1 = 1.0 - a.b1, k2 = 1.0 - a.b2;
    float p[2][4], g[2][4], m[2][4], v[2][4];
    uint32_t cm[2], cv[2];
    float sm[2], sv[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const long long at = first + (2 * wave + u) * kAdamBlock + 4 * lane;
        const int have = have_of<WHOLE>(s.n, at);
        load4(s.theta + at, have, p[u]);
        load4((const G *)s.grad + at, have, g[u]);
        if constexpr (BITS == 32) {
            load4((const float *)s.m + at, have, m[u]);
            load4((const float *)s.v + at, have, v[u]);
        } else {
            cm[u] = load4_codes((const uint8_t *)s.m + at, have);
            cv[u] = load4_codes((const uint8_t *)s.v + at, have);
            const long long block = (first + (2 * wave + u) * kAdamBlock) / kAdamBlock;
            const bool any = WHOLE || block * kAdamBlock < s.n;
            sm[u] = any ? s.mscale[block] : 0.0f;
            sv[u] = any ? s.vscale[block] : 0.0f;
        }
    }
    loads_issued();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const long long at0 = first + (2 * wave + u) * kAdamBlock, at = at0 + 4 * lane;
        if (!WHOLE && at0 >= s.n) break;
        const int have = have_of<WHOLE>(s.n, at);
        if constexpr (BITS == 8) {
            wide_m(cm[u], sm[u], m[u]);
            wide_v(cv[u], sv[u], v[u]);
        }
        float q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const double gd = (double)g[u][j] * gs;
            m[u][j] = blend(a.b1, m[u][j], k1, gd);
            v[u][j] = blend(a.b2, v[u][j], k2, gd * gd);
            // off by 8 steps of fp32 at most; the root's instruction takes subnormal numbers for 0, which only an
            // eps of their roots' size would show (ROOT: there a whole root, and a quotient, as 1 / eps need not be a number)
            const float root = ROOT ? sqrtf(v[u][j] * now.c2) : __builtin_amdgcn_sqrtf(v[u][j] * now.c2);
            const float step = ROOT ? m[u][j] * now.c1 / (root + a.eps)
                                    : m[u][j] * now.c1 * __builtin_amdgcn_rcpf(root + a.eps);
            q[j] = fmaf(-lr, fmaf(s.decay, p[u][j], step), p[u][j]);
        }
        store_out<STREAM>(s.theta + at, have, q);
        if (s.copy) Four<uint16_t>::store<STREAM>(s.copy + at, have, q);
        if constexpr (BITS == 32) {
            store_out<STREAM>((float *)s.m + at, have, m[u]);
            store_out<STREAM>((float *)s.v + at, have, v[u]);
        } else {
            if (!WHOLE)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    m[u][j] = j < have ? m[u][j] : 0.0f;
                    v[u][j] = j < have ? v[u][j] : 0.0f;
                }
            const Narrow nm(lanes_max<64>(top_bits<4>(m[u]))), nv(lanes_max<64>(top_bits<4>(v[u])));
            const uint32_t kb = key ^ mix32((uint32_t)(at0 >> 32));
            uint32_t km[4], kv[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t random = mix32((uint32_t)(at + j) ^ kb);
                km[j] = nm.code<15>(m[u][j], random & 0xffffu);
                km[j] |= km[j] ? float_bits(m[u][j]) >> 24 & 128u : 0u;
                kv[j] = nv.code<31>(v[u][j], random >> 16);
                kv[j] = max(kv[j], v[u][j] > 0.0f ? nv.keep & 1u : 0u);
            }
            store4_codes<STREAM>((uint8_t *)s.m + at, have, km);
            store4_codes<STREAM>((uint8_t *)s.v + at, have, kv);
            if (lane == 0) {
                s.mscale[at0 / kAdamBlock] = nm.stored;
                s.vscale[at0 / kAdamBlock] = nv.stored;
            }
        }
    }
}

template <int BITS, typename G, bool ROOT, bool STREAM>
__global__ void __launch_bounds__(256)
k_adamw(AdamArgs a)
{
    long long first;
    const AdamSeg &s = a.seg[seg_of(a, first)];
    if (first + kAdamTile <= s.n) adamw_tile<BITS, G, ROOT, STREAM, true>(a, s, first);
    else adamw_tile<BITS, G, ROOT, STREAM, false>(a, s, first);
}

// The fp32 numbers that 8-bit moments stand for: theta takes m's, copy v's.
template <bool STREAM>
__global__ void __launch_bounds__(256)
k_adamw_moments(AdamArgs a)
{
    long long first;
    const AdamSeg &s = a.seg[seg_of(a, first)];
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const long long at0 = first + (2 * wave + u) * kAdamBlock, at = at0 + 4 * lane;
        if (at0 >= s.n) break;
        const long long left = s.n - at;
        const int have = left < 0 ? 0 : left > 4 ? 4 : (int)left;
        float m[4], v[4];
        wide_m(load4_codes((const uint8_t *)s.m + at, have), s.mscale[at0 / kAdamBlock], m);
        wide_v(load4_codes((const uint8_t *)s.v + at, have), s.vscale[at0 / kAdamBlock], v);
        store_out<STREAM>(s.theta + at, have, m);
        store_out<STREAM>((float *)s.copy + at, have, v);
    }
}

// Launches `fn` over the tensors, kAdamSegs and 2^23 tiles at a time; returns the number of
// launches or a negative status.
template <typename F>
int for_tiles(AdamArgs &a, int32_t count, F segment, const void *fn, hipStream_t st)
{
    int launches = 0;
    a.count = 0;
    long long tiles = 0;
    for (int32_t k = 0; k <= count; ++k) {
        AdamSeg s{};
        if (k < count) {
            s = segment(k);
            if (s.n == 0) continue;
            s.id = (uint32_t)k;
        }
        const long long t = (s.n + kAdamTile - 1) / kAdamTile;
        if (a.count > 0 && (k == count || a.count == kAdamSegs || tiles + t > kAdamMaxTiles)) {
            a.start[a.count] = (int)tiles;
            void *args[] = {&a};
            if (hipLaunchKernel(fn, dim3((unsigned)tiles), dim3(256), args, 0, st) != hipSuccess)
                return PLSTM_EHIP;
            ++launches;
            a.count = 0;
            tiles = 0;
        }
        if (k == count) break;
        a.start[a.count] = (int)tiles;
        a.seg[a.count++] = s;
        tiles += t;
    }
    return launches;
}

// Parameters that the caches do not hold until they are read again.
bool large(int32_t count, const plstm_adamw_segment *segs)
{
    long long n = 0;
    for (int32_t k = 0; k < count; ++k) n += segs[k].n;
    return n * 4 >= kStreamBytes;
}

int check_segments(int32_t count, const plstm_adamw_segment *segs, int32_t bits)
{
    if (count < 1 || !segs || (bits != 8 && bits != 32)) return PLSTM_EINVAL;
    for (int32_t k = 0; k < count; ++k) {
        const plstm_adamw_segment &s = segs[k];
        if (s.n < 0) return PLSTM_EINVAL;
        if (s.n > kAdamMaxN) return PLSTM_EUNSUPPORTED;
        if (s.n == 0) continue;
        const size_t e = bits == 8 ? 16 : 4;
        if (!s.m || !s.v || !aligned_to(s.m, e) || !aligned_to(s.v, e)) return PLSTM_EINVAL;
        if (bits == 8 && (!s.mscale || !s.vscale || !aligned_to(s.mscale, 4) || !aligned_to(s.vscale, 4)))
            return PLSTM_EINVAL;
    }
    return PLSTM_OK;
}

}  // namespace
}  // namespace plstm

using namespace plstm;

extern "C" {

int64_t pyramid_adamw_scales(int64_t n)
{
    return n < 1 || n > kAdamMaxN ? 0 : (n + kAdamBlock - 1) / kAdamBlock;
}

int pyramid_adamw_step(int32_t count, const plstm_adamw_segment *segs, int32_t bits,
                       int32_t grad_dtype, double lr, double beta1, double beta2, double eps,
                       int64_t step, uint32_t seed, void *clock, const void *lr_dev,
                       const void *grad_scale, void *stream)
{
    const int rc = check_segments(count, segs, bits);
    if (rc != PLSTM_OK) return rc;
    if (grad_dtype != PLSTM_F32 && grad_dtype != PLSTM_BF16) return PLSTM_EINVAL;
    if (!(lr >= 0.0 && lr <= 3.0e38) || !(beta1 >= 0.0 && beta1 < 1.0) ||
        !(beta2 >= 0.0 && beta2 < 1.0) || !((float)eps > 0.0f && eps <= 3.0e38) ||
        (!clock && step < 1))
        return PLSTM_EINVAL;
    if (!aligned_to(clock, 8) || !aligned_to(lr_dev, 4) || !aligned_to(grad_scale, 4))
        return PLSTM_EINVAL;
    const size_t e = dtype_size(grad_dtype);
    for (int32_t k = 0; k < count; ++k) {
        const plstm_adamw_segment &s = segs[k];
        if (!(s.weight_decay >= 0.0f && s.weight_decay <= 3.0e38f)) return PLSTM_EINVAL;
        if (s.n == 0) continue;
        if (!s.theta || !s.grad || !aligned_to(s.theta, 4) || !aligned_to(s.grad, e) ||
            !aligned_to(s.copy, 2))
            return PLSTM_EINVAL;
    }
    hipStream_t st = (hipStream_t)stream;
    AdamArgs a;
    a.b1 = beta1;
    a.b2 = beta2;
    a.lr = (float)lr;
    a.eps = (float)eps;
    a.now = clock ? Clock{} : clock_at(step, beta1, beta2, seed);
    a.clock = (const Clock *)clock;
    a.lr_at = (const float *)lr_dev;
    a.grad_scale = (const float *)grad_scale;
    timing_begin("adamw", st);
    if (clock) {
        k_adamw_clock<<<1, 1, 0, st>>>((Clock *)clock, beta1, beta2, seed);
        PLSTM_LAUNCH_CHECK();
    }
    const auto pick = [&](auto root, auto stream) {
        constexpr bool ROOT = decltype(root)::value, STREAM = decltype(stream)::value;
        if (bits == 32)
            return grad_dtype == PLSTM_F32 ? (const void *)k_adamw<32, float, ROOT, STREAM>
                                           : (const void *)k_adamw<32, uint16_t, ROOT, STREAM>;
        return grad_dtype == PLSTM_F32 ? (const void *)k_adamw<8, float, ROOT, STREAM>
                                       : (const void *)k_adamw<8, uint16_t, ROOT, STREAM>;
    };
    const void *fn = eps < 1e-15               ? pick(std::true_type(), std::false_type())
                     : large(count, segs)      ? pick(std::false_type(), std::true_type())
                                               : pick(std::false_type(), std::false_type());
    const int n = for_tiles(a, count, [&](int32_t k) {
        const plstm_adamw_segment &s = segs[k];
        return AdamSeg{s.theta, s.grad, s.m, s.v, s.mscale, s.vscale, (uint16_t *)s.copy, s.n,
                       s.weight_decay, 0};
    }, fn, st);
    if (n < 0) return n;
    timing_end(n + (clock ? 1 : 0), st);
    return PLSTM_OK;
}

int pyramid_adamw_moments(int32_t count, const plstm_adamw_segment *segs, void *const *m,
                          void *const *v, void *stream)
{
    const int rc = check_segments(count, segs, 8);
    if (rc != PLSTM_OK) return rc;
    if (!m || !v) return PLSTM_EINVAL;
    for (int32_t k = 0; k < count; ++k)
        if (segs[k].n > 0 && (!m[k] || !v[k] || !aligned_to(m[k], 4) || !aligned_to(v[k], 4)))
            return PLSTM_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    AdamArgs a{};
    timing_begin("adamw_moments", st);
    const int n = for_tiles(a, count, [&](int32_t k) {
        const plstm_adamw_segment &s = segs[k];
        return AdamSeg{(float *)m[k], nullptr, s.m, s.v, s.mscale, s.vscale, (uint16_t *)v[k], s.n,
                       0.0f, 0};
    }, large(count, segs) ? (const void *)k_adamw_moments<true> : (const void *)k_adamw_moments<false>, st);
    if (n < 0) return n;
    timing_end(n, st);
    return PLSTM_OK;
}

}  // extern "C"
