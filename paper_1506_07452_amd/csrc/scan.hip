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
#include "timing.h"

namespace plstm {
namespace {

constexpr int kScanThreads = 256;
constexpr int kRun = 16;            // positions between kept states

struct ScanArgs {
    long long B, T, I;
    int reverse;
    const int32_t *lengths;
    long long runs;                 // ceil(T / kRun)
};

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

__device__ inline long long length_of(const ScanArgs &a, long long b)
{
    if (!a.lengths) return a.T;
    const long long n = a.lengths[b];
    return n < 0 ? 0 : n > a.T ? a.T : n;
}

// A thread per channel of a sequence.
template <typename T>
__global__ void __launch_bounds__(kScanThreads)
k_scan_fwd(ScanArgs a, const T *__restrict__ g, const T *__restrict__ u, const float *h0,
           T *__restrict__ h, float *hT, float *__restrict__ saved)
{
    const long long col = (long long)blockIdx.x * kScanThreads + threadIdx.x;
    if (col >= a.B * a.I) return;
    const long long b = col / a.I, i = col - b * a.I;
    const long long n = length_of(a, b);
    float st = h0 ? h0[col] : 0.0f;
    for (long long s = 0; s < a.T; ++s) {
        if (saved && s % kRun == 0) saved[(b * a.runs + s / kRun) * a.I + i] = st;
        const long long t = a.reverse && s < n ? n - 1 - s : s;
        const long long at = (b * a.T + t) * a.I + i;
        if (s < n) {
            float keep, take;
            gate(Store<T>::load(g, at), keep, take);
            st = keep * st + take * Store<T>::load(u, at);
        }
        Store<T>::store(h, at, s < n ? st : 0.0f);
    }
    if (hT) hT[col] = st;
}

template <typename T, typename X>
__global__ void __launch_bounds__(kScanThreads)
k_scan_bwd(ScanArgs a, const X *__restrict__ g, const uint16_t *__restrict__ gscale,
           const X *__restrict__ u, const uint16_t *__restrict__ uscale,
           const float *__restrict__ saved, const T *__restrict__ dh, const float *dhT,
           T *__restrict__ dg, T *__restrict__ du, float *dh0)
{
    const long long col = (long long)blockIdx.x * kScanThreads + threadIdx.x;
    if (col >= a.B * a.I) return;
    const long long b = col / a.I, i = col - b * a.I;
    const long long n = length_of(a, b);
    float G = dhT ? dhT[col] : 0.0f;
    for (long long run = a.runs - 1; run >= 0; --run) {
        const long long s0 = run * kRun;
        float before[kRun];
        float st = saved[(b * a.runs + run) * a.I + i];
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            const long long s = s0 + k;
            before[k] = st;
            if (s < n) {
                const long long at = (b * a.T + (a.reverse ? n - 1 - s : s)) * a.I + i;
                float keep, take;
                gate(load_at(g, gscale, at), keep, take);
                st = keep * st + take * load_at(u, uscale, at);
            }
        }
#pragma unroll
        for (int k = kRun - 1; k >= 0; --k) {
            const long long s = s0 + k;
            if (s >= a.T) continue;
            const long long at = (b * a.T + (a.reverse && s < n ? n - 1 - s : s)) * a.I + i;
            float vg = 0.0f, vu = 0.0f;
            if (s < n) {
                float keep, take;
                gate(load_at(g, gscale, at), keep, take);
                G += Store<T>::load(dh, at);
                vg = G * (before[k] - load_at(u, uscale, at)) * keep * take;
                vu = G * take;
                G *= keep;
            }
            Store<T>::store(dg, at, vg);
            Store<T>::store(du, at, vu);
        }
    }
    if (dh0) dh0[col] = G;
}

int check_scan(int64_t B, int64_t T, int64_t I, int32_t dtype)
{
    if (B < 1 || T < 1 || I < 1) return PLSTM_EINVAL;
    if (dtype != PLSTM_F32 && dtype != PLSTM_BF16) return PLSTM_EINVAL;
    if (B > (1LL << 31) || T > (1LL << 31) || I > (1LL << 31)) return PLSTM_EUNSUPPORTED;
    if (B > (1LL << 38) / I || T > (1LL << 38) / (B * I)) return PLSTM_EUNSUPPORTED;
    return PLSTM_OK;
}

ScanArgs scan_args(int64_t B, int64_t T, int64_t I, int32_t reverse, const int32_t *lengths)
{
    return ScanArgs{B, T, I, reverse, lengths, (T + kRun - 1) / kRun};
}

template <typename T, typename X>
int scan_backward(const ScanArgs &a, const void *g, const void *gscale, const void *u,
                  const void *uscale, const void *saved, const void *dh, const void *dhT,
                  void *dg, void *du, void *dh0, hipStream_t st)
{
    const unsigned grid = (unsigned)((a.B * a.I + kScanThreads - 1) / kScanThreads);
    k_scan_bwd<T, X><<<grid, kScanThreads, 0, st>>>(
        a, (const X *)g, (const uint16_t *)gscale, (const X *)u, (const uint16_t *)uscale,
        (const float *)saved, (const T *)dh, (const float *)dhT, (T *)dg, (T *)du, (float *)dh0);
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
    return 256;
}

int pyramid_scan_forward(int64_t B, int64_t T, int64_t I, int32_t dtype, int32_t reverse,
                         const void *g, const void *u, const int32_t *lengths, const void *h0,
                         void *h, void *hT, void *saved, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = check_scan(B, T, I, dtype);
    if (rc != PLSTM_OK) return rc;
    if ((reverse != 0 && reverse != 1) || !g || !u || !h || !ws) return PLSTM_EINVAL;
    const size_t e = dtype_size(dtype);
    if (!aligned_to(g, e) || !aligned_to(u, e) || !aligned_to(lengths, 4) || !aligned_to(h0, 4) ||
        !aligned_to(h, e) || !aligned_to(hT, 4) || !aligned_to(saved, 16) || !aligned_to(ws, 16))
        return PLSTM_EINVAL;
    if (ws_bytes < pyramid_scan_workspace_size(B, T, I)) return PLSTM_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const ScanArgs a = scan_args(B, T, I, reverse, lengths);
    const unsigned grid = (unsigned)((B * I + kScanThreads - 1) / kScanThreads);
    timing_begin("scan_fwd", st);
    if (dtype == PLSTM_F32)
        k_scan_fwd<<<grid, kScanThreads, 0, st>>>(a, (const float *)g, (const float *)u,
                                                  (const float *)h0, (float *)h, (float *)hT,
                                                  (float *)saved);
    else
        k_scan_fwd<<<grid, kScanThreads, 0, st>>>(a, (const uint16_t *)g, (const uint16_t *)u,
                                                  (const float *)h0, (uint16_t *)h, (float *)hT,
                                                  (float *)saved);
    PLSTM_LAUNCH_CHECK();
    timing_end(1, st);
    return PLSTM_OK;
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
    const ScanArgs a = scan_args(B, T, I, reverse, lengths);
    timing_begin("scan_bwd", st);
    rc = dtype == PLSTM_F32
             ? (gscale ? scan_backward<float, int8_t> : scan_backward<float, float>)(
                   a, g, gscale, u, uscale, saved, dh, dhT, dg, du, dh0, st)
             : (gscale ? scan_backward<uint16_t, int8_t> : scan_backward<uint16_t, uint16_t>)(
                   a, g, gscale, u, uscale, saved, dh, dhT, dg, du, dh0, st);
    if (rc == PLSTM_OK) timing_end(1, st);
    return rc;
}

}  // extern "C"
