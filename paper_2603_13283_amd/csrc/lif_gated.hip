// lif_gated.hip -- the gated leaky integrator over sequences of binned input
// (lif_gated_scan), its gradient (lif_gated_scan_backward) and its single
// step on a pool of states (lif_gated_step).
//
// Each channel runs the affine recurrence h -> a h + u with
//   a = sigmoid(f),  u = (1 - a) x (coupled) or x.
#include "lif_host.hpp"
#include "lif_types.hpp"

namespace lif {
namespace {

// a = sigmoid(f) and 1 - a, each to a few units in its last place.
// e = e^{-|f|} is the square of a power of two, so that it keeps values below
// the smallest normal number, which the hardware's power of two drops.
__device__ __forceinline__ void gate(float f, float& a, float& na)
{
    const float r = __builtin_amdgcn_exp2f(-0.5f * 1.44269504088896341f * fabsf(f));
    const float e = r * r;
    const float s = __builtin_amdgcn_rcpf(1.0f + e);
    a = f >= 0.0f ? s : e * s;
    na = f >= 0.0f ? e * s : s;
}

__device__ __forceinline__ int steps_of(const int32_t* __restrict__ length, int b, int T)
{
    return length ? min(max(length[b], 0), T) : T;
}

template <typename E>
__global__ __launch_bounds__(64) void k_gated_scan(const E* __restrict__ x, const E* __restrict__ f,
                                                   const int32_t* __restrict__ length,
                                                   const float* __restrict__ h_first, lif_gated_params p,
                                                   E* __restrict__ h_out, float* __restrict__ h_last,
                                                   float* __restrict__ marks)
{
    const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (c >= (int64_t)p.B * p.D) return;
    const int b = (int)(c / p.D), d = (int)(c % p.D);
    const int n = steps_of(length, b, p.T);
    const int nm = (p.T + LIF_GATED_MARK - 1) / LIF_GATED_MARK;
    const bool coupled = p.flags & LIF_GATED_COUPLED;
    float h = h_first ? h_first[c] : 0.0f;
    for (int t = 0; t < p.T; ++t) {
        if (marks && t % LIF_GATED_MARK == 0) marks[((int64_t)b * nm + t / LIF_GATED_MARK) * p.D + d] = h;
        float y = 0.0f;
        if (t < n) {
            float a, na;
            gate(to_f32(f[b * p.f_batch + t * p.f_time + d]), a, na);
            const float xv = to_f32(x[b * p.x_batch + t * p.x_time + d]);
            h = fmaf(a, h, coupled ? na * xv : xv);
            y = h;
        }
        if (h_out) h_out[((int64_t)b * p.T + t) * p.D + d] = from_f32<E>(y);
    }
    if (h_last) h_last[c] = h;
}

template <typename E>
__global__ __launch_bounds__(64) void k_gated_back(const E* __restrict__ x, const E* __restrict__ f,
                                                   const int32_t* __restrict__ length,
                                                   const float* __restrict__ marks, const E* __restrict__ grad_h,
                                                   const float* __restrict__ grad_last, lif_gated_params p,
                                                   E* __restrict__ grad_x, E* __restrict__ grad_f,
                                                   float* __restrict__ grad_first)
{
    __shared__ float hs[LIF_GATED_MARK][64];          // the state entering each step of a block
    const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (c >= (int64_t)p.B * p.D) return;
    const int b = (int)(c / p.D), d = (int)(c % p.D);
    const int n = steps_of(length, b, p.T);
    const int nm = (p.T + LIF_GATED_MARK - 1) / LIF_GATED_MARK;
    const bool coupled = p.flags & LIF_GATED_COUPLED;
    float lam = grad_last ? grad_last[c] : 0.0f;
    for (int j = nm - 1; j >= 0; --j) {
        const int t0 = j * LIF_GATED_MARK, t1 = min(t0 + LIF_GATED_MARK, p.T);
        float h = marks[((int64_t)b * nm + j) * p.D + d];
        for (int t = t0; t < min(t1, n); ++t) {
            hs[t - t0][threadIdx.x] = h;
            float a, na;
            gate(to_f32(f[b * p.f_batch + t * p.f_time + d]), a, na);
            const float xv = to_f32(x[b * p.x_batch + t * p.x_time + d]);
            h = fmaf(a, h, coupled ? na * xv : xv);
        }
        for (int t = t1 - 1; t >= t0; --t) {
            float gx = 0.0f, gf = 0.0f;
            if (t < n) {
                float a, na;
                gate(to_f32(f[b * p.f_batch + t * p.f_time + d]), a, na);
                const float xv = to_f32(x[b * p.x_batch + t * p.x_time + d]);
                if (grad_h) lam += to_f32(grad_h[b * p.g_batch + t * p.g_time + d]);
                const float before = hs[t - t0][threadIdx.x];
                gx = coupled ? lam * na : lam;
                gf = lam * (coupled ? before - xv : before) * (a * na);
                lam *= a;
            }
            grad_x[((int64_t)b * p.T + t) * p.D + d] = from_f32<E>(gx);
            grad_f[((int64_t)b * p.T + t) * p.D + d] = from_f32<E>(gf);
        }
    }
    if (grad_first) grad_first[c] = lam;
}

template <typename E>
__global__ __launch_bounds__(256) void k_gated_step(const E* __restrict__ x, const E* __restrict__ f,
                                                    const int32_t* __restrict__ slot, float* __restrict__ state,
                                                    int n_slots, lif_gated_params p, E* __restrict__ h_out)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= (int64_t)p.B * p.D) return;
    const int b = (int)(c / p.D), d = (int)(c % p.D);
    const int s = slot ? slot[b] : b;
    float h = 0.0f;
    if (s >= 0 && s < n_slots) {
        float a, na;
        gate(to_f32(f[b * p.f_batch + d]), a, na);
        const float xv = to_f32(x[b * p.x_batch + d]);
        float* at = state + (int64_t)s * p.D + d;
        h = fmaf(a, *at, (p.flags & LIF_GATED_COUPLED) ? na * xv : xv);
        *at = h;
    }
    h_out[c] = from_f32<E>(h);
}

int check_gated(const lif_gated_params* p)
{
    if (!p || p->B < 0 || p->T < 0 || p->D < 1 || p->reserved != 0 || (p->flags & ~LIF_GATED_COUPLED))
        return LIF_ERR_ARG;
    if (p->dtype != LIF_F32 && p->dtype != LIF_BF16 && p->dtype != LIF_F16) return LIF_ERR_ARG;
    if (p->x_batch < 0 || p->x_time < 0 || p->f_batch < 0 || p->f_time < 0 || p->g_batch < 0 || p->g_time < 0)
        return LIF_ERR_ARG;
    if ((int64_t)p->B * p->D >= ((int64_t)1 << 31)) return LIF_ERR_SIZE;
    if ((int64_t)p->B * p->D * p->T >= ((int64_t)1 << 48)) return LIF_ERR_SIZE;
    return LIF_OK;
}

}  // namespace
}  // namespace lif

extern "C" size_t lif_gated_scan_workspace_size(const lif_gated_params* p)
{
    if (lif::check_gated(p) != LIF_OK) return 0;
    return 0;
}

extern "C" int lif_gated_scan(const void* x, const void* f, const int32_t* length, const float* h_first,
                              const lif_gated_params* p, void* h, float* h_last, float* marks, void* ws,
                              size_t ws_bytes, lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_gated(p);
    if (rc) return rc;
    const int64_t chans = (int64_t)p->B * p->D;
    if (chans * p->T > 0 && (!x || !f)) return LIF_ERR_ARG;
    if (chans > 0 && !h && !h_last && !marks) return LIF_ERR_ARG;
    const size_t need = lif_gated_scan_workspace_size(p);
    if (need > 0 && !ws) return LIF_ERR_ARG;
    if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    if (chans == 0) return LIF_OK;
    with_dtype(p->dtype, [&](auto tag) {
        using E = decltype(tag);
        TIMED_LAUNCH("gated_scan", k_gated_scan<E>, dim3((unsigned)((chans + 63) / 64)), dim3(64), 0,
                     (hipStream_t)stream, (const E*)x, (const E*)f, length, h_first, *p, (E*)h, h_last, marks);
    });
    return check_launch();
}

extern "C" int lif_gated_scan_backward(const void* x, const void* f, const int32_t* length, const float* marks,
                                       const void* grad_h, const float* grad_last, const lif_gated_params* p,
                                       void* grad_x, void* grad_f, float* grad_h_first, void* ws, size_t ws_bytes,
                                       lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_gated(p);
    if (rc) return rc;
    const int64_t chans = (int64_t)p->B * p->D;
    if (chans * p->T > 0 && (!x || !f || !marks || !grad_x || !grad_f)) return LIF_ERR_ARG;
    const size_t need = lif_gated_scan_workspace_size(p);
    if (need > 0 && !ws) return LIF_ERR_ARG;
    if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    if (chans == 0) return LIF_OK;
    with_dtype(p->dtype, [&](auto tag) {
        using E = decltype(tag);
        TIMED_LAUNCH("gated_back", k_gated_back<E>, dim3((unsigned)((chans + 63) / 64)), dim3(64), 0,
                     (hipStream_t)stream, (const E*)x, (const E*)f, length, marks, (const E*)grad_h, grad_last, *p,
                     (E*)grad_x, (E*)grad_f, grad_h_first);
    });
    return check_launch();
}

extern "C" int lif_gated_step(const void* x, const void* f, const int32_t* slot, float* state, int n_slots,
                              const lif_gated_params* p, void* h, lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_gated(p);
    if (rc) return rc;
    const int64_t chans = (int64_t)p->B * p->D;
    if (p->T != 1 || n_slots < 0 || (!slot && n_slots < p->B)) return LIF_ERR_ARG;
    if (chans == 0) return LIF_OK;
    if (!x || !f || !h || (n_slots > 0 && !state)) return LIF_ERR_ARG;
    with_dtype(p->dtype, [&](auto tag) {
        using E = decltype(tag);
        TIMED_LAUNCH("gated_step", k_gated_step<E>, dim3((unsigned)((chans + 255) / 256)), dim3(256), 0,
                     (hipStream_t)stream, (const E*)x, (const E*)f, slot, state, n_slots, *p, (E*)h);
    });
    return check_launch();
}
