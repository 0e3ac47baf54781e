// lif_conv.hip -- the short causal convolution along time (lif_causal_conv),
// its gradient (lif_causal_conv_backward) and its single step on a pool of last
// inputs (lif_causal_conv_step).
//
// A lane holds VEC adjacent channels and walks a strip of the time axis; the
// last K inputs (backward: and the last K gradients of c) stay in its
// registers, so that every element is read once, but for K - 1 steps at a
// strip's edge.  All three are bound by memory.
#include "lif_host.hpp"
#include "lif_types.hpp"
#include "lif_walk.hpp"

namespace lif {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kAhead = 8;             // steps of a batch, whose loads are in flight at once
// Steps of a strip: kMaxStrip, halved down to kMinStrip while a launch has fewer
// than kStripLanes lanes.  In us, training: 16 x 1000 x 512 f32 52 by the rule, 69
// with strips of 64; 4 x 8192 x 1001 f16 104 by the rule, 115 with twice the lanes,
// 147 with strips of 128.
constexpr int kMaxStrip = 64, kMinStrip = 16, kStripLanes = 1 << 16;

struct Geometry {
    int B, T, D, groups, S, strip;    // channel groups, strips of the time axis and their steps
    uint32_t flags;
    int64_t x_batch, x_time, g_batch, g_time;
};

// A lane's strip of steps [t0, t1) of sample b and its channels from d on.
// Where VEC does not divide D, the last group starts at D - VEC: the channels
// that it shares with the group before get the same bits twice.
struct Place {
    int b, s, d, n, t0, t1;
};

template <int VEC>
__device__ __forceinline__ bool place_of(const Geometry& q, const int32_t* __restrict__ length, Place& p)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t strip = at / q.groups;
    if (strip >= (int64_t)q.B * q.S) return false;
    p.b = (int)(strip / q.S);
    p.s = (int)(strip - (int64_t)p.b * q.S);
    p.d = min((int)(at - strip * q.groups) * VEC, q.D - VEC);
    p.n = length ? min(max(length[p.b], 0), q.T) : q.T;
    p.t0 = p.s * q.strip;
    p.t1 = min(p.t0 + q.strip, q.T);
    return true;
}

template <typename E, int VEC> struct Vec {
    E v[VEC];
};

// STEPS steps of x or grad_y from t >= 0 on; those past the sample's end as 0.
// The loads of a batch are issued together.
template <typename E, int VEC, int STEPS>
__device__ __forceinline__ void load_batch(Vec<E, VEC> (&to)[STEPS], const E* __restrict__ in, int64_t time, int t,
                                           int n)
{
    const E* at = in + t * time;
    if (t + STEPS <= n) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i, at += time) load_elems<E, VEC>(at, to[i].v);
    } else {
#pragma unroll
        for (int i = 0; i < STEPS; ++i, at += time) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) to[i].v[k] = from_f32<E>(0.0f);
            if (t + i < n) load_elems<E, VEC>(at, to[i].v);
        }
    }
}

// The input at step t < n, from x_first (or 0) where t < 0.
template <typename E, int K, int VEC>
__device__ __forceinline__ Vec<E, VEC> input_at(const E* __restrict__ x, const E* __restrict__ first,
                                                const Geometry& q, const Place& p, int t)
{
    Vec<E, VEC> v;
#pragma unroll
    for (int k = 0; k < VEC; ++k) v.v[k] = from_f32<E>(0.0f);
    if (t >= 0) {
        if (t < p.n) load_elems<E, VEC>(x + p.b * q.x_batch + t * q.x_time + p.d, v.v);
    } else if (first) {
        load_elems<E, VEC>(first + ((int64_t)p.b * (K - 1) + t + K - 1) * q.D + p.d, v.v);
    }
    return v;
}

template <typename E, int VEC> __device__ __forceinline__ void to_floats(const Vec<E, VEC>& r, float (&v)[VEC])
{
#pragma unroll
    for (int k = 0; k < VEC; ++k) v[k] = to_f32(r.v[k]);
}

template <int K, int VEC>
__device__ __forceinline__ void load_taps(const float* __restrict__ w, const float* __restrict__ bias, int d,
                                          float (&tap)[K][VEC], float (&b)[VEC])
{
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
#pragma unroll
        for (int j = 0; j < K; ++j) tap[j][k] = w[(int64_t)(d + k) * K + j];
        b[k] = bias ? bias[d + k] : 0.0f;
    }
}

// c / (1 + e^-c) and its derivative.
__device__ __forceinline__ float silu(float c, float& slope)
{
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * c));
    slope = s * fmaf(c, 1.0f - s, 1.0f);
    return c * s;
}

// Bound by memory with the vector units half busy (8 x 2048 x 2048 bf16, ragged,
// 26 us, 100 MB at 3.9 TB/s; 4 x 8192 x 1001 f16 32 us, 131 MB at 4.1).
template <typename E, int K, int VEC>
__global__ __launch_bounds__(256) void k_conv(const E* __restrict__ x, const float* __restrict__ w,
                                              const float* __restrict__ bias, const int32_t* __restrict__ length,
                                              const E* __restrict__ first, Geometry q, E* __restrict__ y,
                                              E* __restrict__ last)
{
    Place p;
    if (!place_of<VEC>(q, length, p)) return;
    if (last && p.s == 0)
        for (int j = 0; j < K - 1; ++j) {
            const Vec<E, VEC> v = input_at<E, K, VEC>(x, first, q, p, p.n - (K - 1) + j);
            store_elems<E, VEC>(last + ((int64_t)p.b * (K - 1) + j) * q.D + p.d, v.v);
        }
    if (!y) return;
    float tap[K][VEC], b[VEC], win[K - 1 + kAhead][VEC];
    Vec<E, VEC> raw[kAhead];
    const E* in = x + p.b * q.x_batch + p.d;
    load_batch<E, VEC, kAhead>(raw, in, q.x_time, p.t0, p.n);
    load_taps<K, VEC>(w, bias, p.d, tap, b);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) to_floats(input_at<E, K, VEC>(x, first, q, p, p.t0 - (K - 1) + j), win[j]);
    E* out = y + ((int64_t)p.b * q.T + p.t0) * q.D + p.d;
    for (int t = p.t0; t < p.t1; t += kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) to_floats(raw[i], win[K - 1 + i]);
        if (t + kAhead < p.t1) load_batch<E, VEC, kAhead>(raw, in, q.x_time, t + kAhead, p.n);
        const bool whole = t + kAhead <= min(p.n, p.t1);
#pragma unroll
        for (int i = 0; i < kAhead; ++i, out += q.D) {
            E o[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                float c = b[k], slope;
#pragma unroll
                for (int j = 0; j < K; ++j) c = fmaf(tap[j][k], win[i + j][k], c);
                if (q.flags & LIF_CONV_SILU) c = silu(c, slope);
                o[k] = from_f32<E>(whole || t + i < p.n ? c : 0.0f);
            }
            if (whole || t + i < p.t1) store_elems<E, VEC>(out, o);
        }
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
#pragma unroll
            for (int k = 0; k < VEC; ++k) win[j][k] = win[kAhead + j][k];
    }
}

// At step t the gradients gc_{t-K+1} .. gc_t give that of the input K - 1 steps
// before, sum_j w[j] gc_{t-j}: a strip walks K - 1 steps past its end.  The sums
// for w and bias go over the strip's own steps.  Eight steps of two inputs in
// flight hide the loads where the taps leave room for them in registers (K <= 4:
// 114 -> 107 us, training 4 x 8192 x 1001 f16; K = 8: 140 -> 172, 8 x 2048 x 2048
// bf16).  4 x 8192 x 1001 f16 62 us, 205 MB at 3.3 TB/s; vector units 47 % busy.
template <typename E, int K, int VEC>
__global__ __launch_bounds__(256) void k_conv_back(const E* __restrict__ x, const float* __restrict__ w,
                                                   const float* __restrict__ bias, const int32_t* __restrict__ length,
                                                   const E* __restrict__ first, const E* __restrict__ gy,
                                                   const float* __restrict__ grad_last, Geometry q,
                                                   E* __restrict__ gx, float* __restrict__ g_first,
                                                   float* __restrict__ part)
{
    constexpr int U = K <= 4 ? 8 : 4;
    Place p;
    if (!place_of<VEC>(q, length, p)) return;
    float tap[K][VEC], b[VEC], win[K - 1 + U][VEC], gc[K - 1 + U][VEC], gw[K][VEC], gb[VEC];
    Vec<E, VEC> rx[U], rg[U];
    const E* in = x + p.b * q.x_batch + p.d;
    const E* gin = gy ? gy + p.b * q.g_batch + p.d : nullptr;
    const int gn = gy ? p.n : 0;                              // steps that have a gradient
    load_batch<E, VEC, U>(rx, in, q.x_time, p.t0, p.n);
    load_batch<E, VEC, U>(rg, gin, q.g_time, p.t0, gn);
    load_taps<K, VEC>(w, bias, p.d, tap, b);
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        gb[k] = 0.0f;
#pragma unroll
        for (int j = 0; j < K; ++j) gw[j][k] = 0.0f;
#pragma unroll
        for (int j = 0; j < K - 1; ++j) gc[j][k] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < K - 1; ++j) to_floats(input_at<E, K, VEC>(x, first, q, p, p.t0 - (K - 1) + j), win[j]);
    const int from = p.s == 0 ? -(K - 1) : p.t0, end = p.t1 + K - 1;
    for (int t = p.t0; t < end; t += U) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            to_floats(rx[i], win[K - 1 + i]);
            to_floats(rg[i], gc[K - 1 + i]);
        }
        if (t + U < end) {
            load_batch<E, VEC, U>(rx, in, q.x_time, t + U, p.n);
            load_batch<E, VEC, U>(rg, gin, q.g_time, t + U, gn);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const bool on = t + i < p.n, own = on && t + i < p.t1;
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                float c = b[k], slope = 1.0f;
#pragma unroll
                for (int j = 0; j < K; ++j) c = fmaf(tap[j][k], win[i + j][k], c);
                if (q.flags & LIF_CONV_SILU) silu(c, slope);
                const float g = on ? gc[K - 1 + i][k] * slope : 0.0f;
                gc[K - 1 + i][k] = g;
                if (own) {
#pragma unroll
                    for (int j = 0; j < K; ++j) gw[j][k] = fmaf(g, win[i + j][k], gw[j][k]);
                    gb[k] += g;
                }
            }
            const int at = t + i - (K - 1);
            if (at < from || at >= p.t1) continue;
            float v[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                v[k] = 0.0f;
#pragma unroll
                for (int j = 0; j < K; ++j) v[k] = fmaf(tap[j][k], gc[K - 1 + i - j][k], v[k]);
            }
            const int j = at - (p.n - (K - 1));
            if (grad_last && j >= 0 && j < K - 1) {
                float l[VEC];
                load_elems<float, VEC>(grad_last + ((int64_t)p.b * (K - 1) + j) * q.D + p.d, l);
#pragma unroll
                for (int k = 0; k < VEC; ++k) v[k] += l[k];
            }
            if (at >= 0) {
                E o[VEC];
#pragma unroll
                for (int k = 0; k < VEC; ++k) o[k] = from_f32<E>(at < p.n ? v[k] : 0.0f);
                store_elems<E, VEC>(gx + ((int64_t)p.b * q.T + at) * q.D + p.d, o);
            } else if (g_first) {
                store_elems<float, VEC>(g_first + ((int64_t)p.b * (K - 1) + at + K - 1) * q.D + p.d, v);
            }
        }
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
#pragma unroll
            for (int k = 0; k < VEC; ++k) win[j][k] = win[U + j][k], gc[j][k] = gc[U + j][k];
    }
    if (part) {
        float* to = part + ((int64_t)p.b * q.S + p.s) * (K + 1) * q.D + p.d;
#pragma unroll
        for (int j = 0; j < K; ++j) store_elems<float, VEC>(to + (int64_t)j * q.D, gw[j]);
        store_elems<float, VEC>(to + (int64_t)K * q.D, gb);
    }
}

// Adds up the strips' parts [strips][K + 1][D]: 64 of the (K + 1) D sums to a
// workgroup at a time, whose 16 waves each take a contiguous range of strips.
__global__ __launch_bounds__(1024) void k_conv_sums(const float* __restrict__ part, int64_t strips, int K, int D,
                                                    float* __restrict__ gw, float* __restrict__ gb)
{
    __shared__ float sh[16][64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t sums = (int64_t)(K + 1) * D;
    for (int64_t at0 = (int64_t)blockIdx.x * 64; at0 < sums; at0 += (int64_t)gridDim.x * 64) {
        const int64_t at = at0 + lane;
        sh[w][lane] = at < sums ? sum_rows(part + at, sums, strips * w / 16, strips * (w + 1) / 16) : 0.0f;
        __syncthreads();
        if (w == 0 && at < sums) {
            float s = 0.0f;
            for (int j = 0; j < 16; ++j) s += sh[j][lane];
            const int j = (int)(at / D), d = (int)(at - (int64_t)j * D);
            if (j < K) {
                if (gw) gw[(int64_t)d * K + j] = s;
            } else if (gb) {
                gb[d] = s;
            }
        }
        __syncthreads();
    }
}

// One step of VEC channels from d on of stream b.
template <typename E, int K, int VEC>
__device__ __forceinline__ void step_at(const E* __restrict__ x, const float* __restrict__ w,
                                        const float* __restrict__ bias, E* __restrict__ state, int row, bool on,
                                        const Geometry& q, int b, int d, E* __restrict__ y)
{
    E o[VEC];
    if (on) {
        E win[K][VEC];
        E* st = state + (int64_t)row * (K - 1) * q.D + d;
#pragma unroll
        for (int j = 0; j < K - 1; ++j) load_elems<E, VEC>(st + (int64_t)j * q.D, win[j]);
        load_elems<E, VEC>(x + b * q.x_batch + d, win[K - 1]);
        float tap[K][VEC], bs[VEC];
        load_taps<K, VEC>(w, bias, d, tap, bs);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            float c = bs[k], slope;
#pragma unroll
            for (int j = 0; j < K; ++j) c = fmaf(tap[j][k], to_f32(win[j][k]), c);
            o[k] = from_f32<E>((q.flags & LIF_CONV_SILU) ? silu(c, slope) : c);
        }
#pragma unroll
        for (int j = 0; j < K - 1; ++j) store_elems<E, VEC>(st + (int64_t)j * q.D, win[j + 1]);
    } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k) o[k] = from_f32<E>(0.0f);
    }
    store_elems<E, VEC>(y + (int64_t)b * q.D + d, o);
}

// The state is read and written in place, so every channel has one lane: the
// first D / VEC lanes of a stream take VEC channels each, the D % VEC after them
// one each.  Bound by the launch: 64 x 2048 bf16 3.7 us.
template <typename E, int K, int VEC>
__global__ __launch_bounds__(256) void k_conv_step(const E* __restrict__ x, const float* __restrict__ w,
                                                   const float* __restrict__ bias, const int32_t* __restrict__ slot,
                                                   E* __restrict__ state, int n_slots, Geometry q, E* __restrict__ y)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= (int64_t)q.B * q.groups) return;
    const int b = (int)(at / q.groups), i = (int)(at - (int64_t)b * q.groups), wide = q.D / VEC;
    const int row = slot ? slot[b] : b;
    const bool on = row >= 0 && row < n_slots;
    if (i < wide) step_at<E, K, VEC>(x, w, bias, state, row, on, q, b, i * VEC, y);
    else if constexpr (VEC > 1) step_at<E, K, 1>(x, w, bias, state, row, on, q, b, wide * VEC + i - wide, y);
}

int check_conv(const lif_conv_params* p)
{
    if (!p || p->B < 0 || p->T < 0 || p->D < 1 || p->K < 2 || (p->flags & ~LIF_CONV_SILU)) return LIF_ERR_ARG;
    if (p->dtype != LIF_F32 && p->dtype != LIF_BF16 && p->dtype != LIF_F16) return LIF_ERR_ARG;
    if (p->x_batch < 0 || p->x_time < 0 || p->g_batch < 0 || p->g_time < 0) return LIF_ERR_ARG;
    if (p->K > LIF_CONV_MAX || (int64_t)p->B * p->D >= ((int64_t)1 << 28) || p->T > (1 << 30)) return LIF_ERR_SIZE;
    if ((int64_t)p->B * p->D * p->T >= ((int64_t)1 << 40)) return LIF_ERR_SIZE;
    return LIF_OK;
}

int vec_of(const lif_conv_params& p) { return p.D >= 4 ? 4 : 1; }

Geometry geometry_of(const lif_conv_params& p, int strip)
{
    Geometry q;
    q.B = p.B, q.T = p.T, q.D = p.D;
    q.groups = (p.D + vec_of(p) - 1) / vec_of(p);
    q.strip = strip;
    q.S = p.T > 0 ? (p.T + strip - 1) / strip : 1;
    q.flags = p.flags;
    q.x_batch = p.x_batch, q.x_time = p.x_time, q.g_batch = p.g_batch, q.g_time = p.g_time;
    return q;
}

// Steps of a strip: shorter ones where there would be few lanes.  A launch has
// fewer than 2^32 threads.
int strip_of(const lif_conv_params& p)
{
    const int64_t lanes = (int64_t)p.B * ((p.D + vec_of(p) - 1) / vec_of(p));
    int strip = kMaxStrip;
    while (strip > kMinStrip && lanes * ((p.T + strip - 1) / strip) < kStripLanes) strip /= 2;
    while (lanes * ((p.T + strip - 1) / strip) >= ((int64_t)1 << 31)) strip *= 2;
    return strip;
}

template <int V> struct Int { static constexpr int value = V; };

template <typename Fn> void with_shape(const lif_conv_params& p, Fn&& fn)
{
    with_dtype(p.dtype, [&](auto e) {
        auto with = [&](auto k) {
            if (vec_of(p) == 4) fn(e, k, Int<4>());
            else fn(e, k, Int<1>());
        };
        switch (p.K) {
            case 2: return with(Int<2>());
            case 3: return with(Int<3>());
            case 4: return with(Int<4>());
            case 5: return with(Int<5>());
            case 6: return with(Int<6>());
            case 7: return with(Int<7>());
            default: return with(Int<8>());
        }
    });
}

}  // namespace
}  // namespace lif

extern "C" size_t lif_causal_conv_workspace_size(const lif_conv_params* p)
{
    using namespace lif;
    if (check_conv(p) != LIF_OK) return 0;
    const Geometry q = geometry_of(*p, strip_of(*p));
    return sizeof(float) * (size_t)q.B * q.S * (p->K + 1) * q.D;
}

extern "C" int lif_causal_conv(const void* x, const float* w, const float* bias, const int32_t* length,
                               const void* x_first, const lif_conv_params* p, void* y, void* x_last,
                               lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_conv(p);
    if (rc) return rc;
    if (p->B > 0 && ((p->T > 0 && !x) || !w || (!y && !x_last))) return LIF_ERR_ARG;
    if (p->B == 0) return LIF_OK;
    const Geometry q = geometry_of(*p, strip_of(*p));
    const int64_t lanes = (int64_t)q.B * q.S * q.groups;
    with_shape(*p, [&](auto e, auto taps, auto vec) {
        using E = decltype(e);
        constexpr int K = decltype(taps)::value, VEC = decltype(vec)::value;
        TIMED_LAUNCH("conv", (k_conv<E, K, VEC>), dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0,
                     (hipStream_t)stream, (const E*)x, w, bias, length, (const E*)x_first, q, (E*)y, (E*)x_last);
    });
    return check_launch();
}

extern "C" int lif_causal_conv_backward(const void* x, const float* w, const float* bias, const int32_t* length,
                                        const void* x_first, const void* grad_y, const float* grad_last,
                                        const lif_conv_params* p, void* grad_x, float* grad_w, float* grad_bias,
                                        float* grad_x_first, void* ws, size_t ws_bytes, lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_conv(p);
    if (rc) return rc;
    if (p->B > 0 && ((p->T > 0 && (!x || !grad_x)) || !w)) return LIF_ERR_ARG;
    const size_t need = lif_causal_conv_workspace_size(p);
    const bool sums = grad_w || grad_bias;
    if (sums && need > 0) {
        if (!ws || (uintptr_t)ws % 16) return LIF_ERR_ARG;
        if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    }
    const Geometry q = geometry_of(*p, strip_of(*p));
    const int64_t lanes = (int64_t)q.B * q.S * q.groups;
    if (p->B > 0)
        with_shape(*p, [&](auto e, auto taps, auto vec) {
            using E = decltype(e);
            constexpr int K = decltype(taps)::value, VEC = decltype(vec)::value;
            TIMED_LAUNCH("conv_back", (k_conv_back<E, K, VEC>), dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0,
                         (hipStream_t)stream, (const E*)x, w, bias, length, (const E*)x_first, (const E*)grad_y,
                         grad_last, q, (E*)grad_x, grad_x_first, sums ? (float*)ws : nullptr);
        });
    const int64_t blocks = min(((int64_t)(p->K + 1) * q.D + 63) / 64, (int64_t)1 << 20);
    if (sums)
        TIMED_LAUNCH("conv_sums", k_conv_sums, dim3((unsigned)blocks), dim3(1024), 0, (hipStream_t)stream,
                     (const float*)ws, (int64_t)q.B * q.S, p->K, q.D, grad_w, grad_bias);
    return check_launch();
}

extern "C" int lif_causal_conv_step(const void* x, const float* w, const float* bias, const int32_t* slot,
                                    void* state, int n_slots, const lif_conv_params* p, void* y, lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_conv(p);
    if (rc) return rc;
    if (p->T != 1 || n_slots < 0 || (!slot && n_slots < p->B)) return LIF_ERR_ARG;
    if (p->B == 0) return LIF_OK;
    if (!x || !w || !y || (n_slots > 0 && !state)) return LIF_ERR_ARG;
    Geometry q = geometry_of(*p, 1);
    q.groups = p->D / vec_of(*p) + p->D % vec_of(*p);
    const int64_t lanes = (int64_t)q.B * q.groups;
    with_shape(*p, [&](auto e, auto taps, auto vec) {
        using E = decltype(e);
        constexpr int K = decltype(taps)::value, VEC = decltype(vec)::value;
        TIMED_LAUNCH("conv_step", (k_conv_step<E, K, VEC>), dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0,
                     (hipStream_t)stream, (const E*)x, w, bias, slot, (E*)state, n_slots, q, (E*)y);
    });
    return check_launch();
}
