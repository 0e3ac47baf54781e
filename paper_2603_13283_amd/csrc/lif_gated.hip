// lif_gated.hip -- the gated leaky integrator over sequences of binned input
// (lif_gated_scan), its gradient (lif_gated_scan_backward) and its single
// step on a pool of states (lif_gated_step).
//
// Each channel runs the affine recurrence h -> a h + u with
//   a = sigmoid(f),  u = (1 - a) x (coupled) or x,
// and affine maps compose: (A2, H2) after (A1, H1) is (A2 A1, A2 H1 + H2).
// The adjoint mu that enters a step from the later side obeys the same kind
// of map, mu -> a mu + a g (lambda = g + mu, g = dL/dh), in reverse order.
//
// A lane holds CPL adjacent channels; consecutive lanes hold consecutive
// channel groups of the flattened (sample, channel) axis, so that narrow
// layers still fill a wave.  A workgroup of NW waves takes a tile of NW * TS
// steps of its 64 lanes' channels: each wave composes the maps of its TS
// steps in registers, the waves' maps meet in LDS (one barrier per tile, two
// buffers), every wave folds them onto the state carried from the tile before
// and runs its steps once more from its own entering state.  x and f are read
// once, the next tile's loads are in flight while a tile is worked on.
// Rerunning the steps (one FMA each) instead of applying the composed prefix
// products keeps a state's rounding that of the recurrence.
#include "lif_host.hpp"
#include "lif_types.hpp"

namespace lif {
namespace {

constexpr int kTS = 8;            // steps of a wave in a tile
constexpr int kMaxWaves = 8;      // waves of a workgroup
static_assert(LIF_GATED_MARK % kTS == 0 && kTS * kMaxWaves == LIF_GATED_MARK,
              "a mark is the state entering some wave's first step, and a backward tile starts at one");

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

// What a launch works on: `groups` = B * D / CPL lanes in all, `S` segments of
// `seg_len` steps (a multiple of LIF_GATED_MARK) of the time axis.
struct Geometry {
    int B, T, D, groups, per_sample, S, seg_len;
    int64_t x_batch, x_time, f_batch, f_time, g_batch, g_time;
};

// A lane's place: sample b, first channel d, flat channel c = b * D + d, the
// sample's steps n and the smallest and largest n of the wave.  Lanes past
// the last group repeat it and store nothing.
struct Place {
    int b, d, n, n_min, n_max;
    int64_t c;
    bool live;
};

template <int CPL>
__device__ __forceinline__ Place place_of(const Geometry& g, const int32_t* __restrict__ length, int lane)
{
    Place p;
    const int64_t at = (int64_t)blockIdx.x * kWave + lane;
    p.live = at < g.groups;
    const int cg = p.live ? (int)at : g.groups - 1;
    p.b = cg / g.per_sample;
    p.d = (cg - p.b * g.per_sample) * CPL;
    p.c = (int64_t)p.b * g.D + p.d;
    p.n = steps_of(length, p.b, g.T);
    p.n_min = p.n_max = p.n;
    for (int o = 32; o; o >>= 1) {
        p.n_min = min(p.n_min, __shfl_xor(p.n_min, o));
        p.n_max = max(p.n_max, __shfl_xor(p.n_max, o));
    }
    p.n_min = __builtin_amdgcn_readfirstlane(p.n_min);
    p.n_max = __builtin_amdgcn_readfirstlane(p.n_max);
    return p;
}

// The raw elements of a wave's TS steps of two or three inputs.
template <typename E, int CPL, int N>
struct Raw {
    E v[N][kTS][CPL];
};

// Loads steps t .. t + TS - 1 (those below the lane's n) of one input.
template <typename E, int CPL>
__device__ __forceinline__ void load_steps(E (&v)[kTS][CPL], const E* __restrict__ base, int64_t stride, int t,
                                           const Place& p)
{
    const E* at = base + (int64_t)t * stride;
    if (t + kTS <= p.n_min) {
#pragma unroll
        for (int i = 0; i < kTS; ++i) load_elems<E, CPL>(at + i * stride, v[i]);
    } else if (t < p.n_max) {
#pragma unroll
        for (int i = 0; i < kTS; ++i)
            if (t + i < p.n) load_elems<E, CPL>(at + i * stride, v[i]);
    }
}

// The state that enters a segment: h_first (or grad_last) carried through the
// maps of the segments before it in the direction of the walk, `count` of
// them from `from` on, one every `step`.
template <int CPL>
__device__ __forceinline__ void fold_segments(float (&c)[CPL], const float2* __restrict__ maps, int64_t chans,
                                              int64_t at, int from, int count, int step)
{
#pragma unroll 4
    for (int s = 0; s < count; ++s) {
        const float2* q = maps + (int64_t)(from + s * step) * chans + at;
#pragma unroll
        for (int k = 0; k < CPL; ++k) c[k] = fmaf(q[k].x, c[k], q[k].y);
    }
}

// Composed maps of whole segments, where the time axis is shared out over
// workgroups: segment blockIdx.y's map of h (forward: inputs f and x) or of mu
// (REVERSE: inputs f and grad_h).  Each wave takes a contiguous part of the
// segment with no barrier; the waves' maps meet once at the end.
template <typename E, int CPL, bool COUPLED, bool REVERSE>
__global__ __launch_bounds__(kMaxWaves* kWave) void k_segment_maps(const E* __restrict__ in, const E* __restrict__ f,
                                                                   const int32_t* __restrict__ length, Geometry g,
                                                                   float2* __restrict__ maps)
{
    __shared__ float2 sh[kMaxWaves][CPL][kWave];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
    const int seg = REVERSE ? blockIdx.y + 1 : blockIdx.y;       // the walk's last segment needs no map
    const Place p = place_of<CPL>(g, length, lane);
    const int64_t in_batch = REVERSE ? g.g_batch : g.x_batch, in_time = REVERSE ? g.g_time : g.x_time;
    const E* in0 = in ? in + p.b * in_batch + p.d : nullptr;     // no grad_h: 0
    const E* f0 = f + p.b * g.f_batch + p.d;
    const int part = g.seg_len / nw;                             // a multiple of TS
    const int t0 = seg * g.seg_len + w * part;
    const int t1 = min(t0 + part, g.T);
    float A[CPL], H[CPL];
#pragma unroll
    for (int k = 0; k < CPL; ++k) A[k] = 1.0f, H[k] = 0.0f;
    const int blocks = t1 > t0 ? (min(t1, p.n_max) - t0 + kTS - 1) / kTS : 0;
    Raw<E, CPL, 2> cur, nxt;
    auto at = [&](int j) { return REVERSE ? t0 + (blocks - 1 - j) * kTS : t0 + j * kTS; };
    auto load = [&](Raw<E, CPL, 2>& r, int j) {
        load_steps<E, CPL>(r.v[0], f0, g.f_time, at(j), p);
        if (in0) load_steps<E, CPL>(r.v[1], in0, in_time, at(j), p);
    };
    if (blocks > 0) load(cur, 0);
    for (int j = 0; j < blocks; ++j) {
        if (j + 1 < blocks) load(nxt, j + 1);
        const int t = at(j);
#pragma unroll
        for (int q = 0; q < kTS; ++q) {
            const int i = REVERSE ? kTS - 1 - q : q;
            if (t + i < p.n) {
#pragma unroll
                for (int k = 0; k < CPL; ++k) {
                    float a, na;
                    gate(to_f32(cur.v[0][i][k]), a, na);
                    const float v = in0 ? to_f32(cur.v[1][i][k]) : 0.0f;
                    H[k] = REVERSE ? a * (H[k] + v) : fmaf(a, H[k], COUPLED ? na * v : v);
                    A[k] *= a;
                }
            }
        }
        cur = nxt;
    }
#pragma unroll
    for (int k = 0; k < CPL; ++k) sh[w][k][lane] = make_float2(A[k], H[k]);
    __syncthreads();
    if (w == 0 && p.live) {
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
            float a = 1.0f, h = 0.0f;
            for (int q = 0; q < nw; ++q) {
                const float2 m = sh[REVERSE ? nw - 1 - q : q][k][lane];
                h = fmaf(m.x, h, m.y);
                a *= m.x;
            }
            maps[(int64_t)seg * ((int64_t)g.B * g.D) + p.c + k] = make_float2(a, h);
        }
    }
}

template <typename E, int CPL, bool COUPLED>
__global__ __launch_bounds__(kMaxWaves* kWave) void k_scan(const E* __restrict__ x, const E* __restrict__ f,
                                                           const int32_t* __restrict__ length,
                                                           const float* __restrict__ h_first, Geometry g,
                                                           const float2* __restrict__ maps, E* __restrict__ h_out,
                                                           float* __restrict__ h_last, float* __restrict__ marks)
{
    __shared__ float2 sh[2][kMaxWaves][CPL][kWave];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
    const int seg = blockIdx.y, tile = nw * kTS;
    const int64_t chans = (int64_t)g.B * g.D;
    const Place p = place_of<CPL>(g, length, lane);
    const int t0 = seg * g.seg_len, t1 = min(t0 + g.seg_len, g.T);
    const E* x0 = x + p.b * g.x_batch + p.d;
    const E* f0 = f + p.b * g.f_batch + p.d;
    E* out = h_out ? h_out + (int64_t)p.b * g.T * g.D + p.d : nullptr;
    const int nm = (g.T + LIF_GATED_MARK - 1) / LIF_GATED_MARK;
    float* mk = marks ? marks + (int64_t)p.b * nm * g.D + p.d : nullptr;

    Raw<E, CPL, 2> cur, nxt;
    auto load = [&](Raw<E, CPL, 2>& r, int t) {
        load_steps<E, CPL>(r.v[0], f0, g.f_time, t, p);
        load_steps<E, CPL>(r.v[1], x0, g.x_time, t, p);
    };
    if (t0 + w * kTS < t1) load(cur, t0 + w * kTS);

    float c[CPL];                       // the state carried into the tile, the same in every wave
#pragma unroll
    for (int k = 0; k < CPL; ++k) c[k] = h_first ? h_first[p.c + k] : 0.0f;
    fold_segments<CPL>(c, maps, chans, p.c, 0, seg, 1);

    int buf = 0;
    for (int tt = t0; tt < t1; tt += tile, buf ^= 1) {
        const int t = tt + w * kTS;
        float a[kTS][CPL], u[kTS][CPL], in[CPL];
        if (tt < p.n_max) {
            if (tt + tile < t1) load(nxt, t + tile);
            float A[CPL], H[CPL];
#pragma unroll
            for (int k = 0; k < CPL; ++k) A[k] = 1.0f, H[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < kTS; ++i) {
                const bool on = t + i < p.n;
#pragma unroll
                for (int k = 0; k < CPL; ++k) {
                    float s, ns;
                    gate(to_f32(cur.v[0][i][k]), s, ns);
                    const float v = to_f32(cur.v[1][i][k]);
                    a[i][k] = on ? s : 1.0f;
                    u[i][k] = on ? (COUPLED ? ns * v : v) : 0.0f;
                    H[k] = fmaf(a[i][k], H[k], u[i][k]);
                    A[k] *= a[i][k];
                }
            }
#pragma unroll
            for (int k = 0; k < CPL; ++k) sh[buf][w][k][lane] = make_float2(A[k], H[k]);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < CPL; ++k) in[k] = c[k];
            for (int q = 0; q < nw; ++q)
#pragma unroll
                for (int k = 0; k < CPL; ++k) {
                    const float2 m = sh[buf][q][k][lane];
                    if (q == w) in[k] = c[k];
                    c[k] = fmaf(m.x, c[k], m.y);
                }
        } else {                        // past every lane's length: the state stays
#pragma unroll
            for (int k = 0; k < CPL; ++k) {
                in[k] = c[k];
#pragma unroll
                for (int i = 0; i < kTS; ++i) a[i][k] = 1.0f, u[i][k] = 0.0f;
            }
        }
        if (p.live) {
            if (mk && t % LIF_GATED_MARK == 0 && t < g.T) store_elems<float, CPL>(mk + (int64_t)(t / LIF_GATED_MARK) * g.D, in);
            if (out) {
#pragma unroll
                for (int i = 0; i < kTS; ++i) {
                    E o[CPL];
#pragma unroll
                    for (int k = 0; k < CPL; ++k) {
                        in[k] = fmaf(a[i][k], in[k], u[i][k]);
                        o[k] = from_f32<E>(t + i < p.n ? in[k] : 0.0f);
                    }
                    if (t + i < t1) store_elems<E, CPL>(out + (int64_t)(t + i) * g.D, o);
                }
            }
        }
        cur = nxt;
    }
    if (h_last && seg == g.S - 1 && w == 0 && p.live) store_elems<float, CPL>(h_last + p.c, c);
}

// Backward: tiles of LIF_GATED_MARK steps from the last to the first.  The
// states of a tile are recomputed from its mark, so h is not read; both
// directions' maps meet in the same LDS exchange (their products A are the
// same).
template <typename E, int CPL, bool COUPLED>
__global__ __launch_bounds__(kMaxWaves* kWave) void k_back(const E* __restrict__ x, const E* __restrict__ f,
                                                           const int32_t* __restrict__ length,
                                                           const float* __restrict__ marks,
                                                           const E* __restrict__ grad_h,
                                                           const float* __restrict__ grad_last, Geometry g,
                                                           const float2* __restrict__ maps, E* __restrict__ grad_x,
                                                           E* __restrict__ grad_f, float* __restrict__ grad_first)
{
    __shared__ float sh[2][kMaxWaves][CPL][3][kWave];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int seg = blockIdx.y;
    constexpr int tile = kMaxWaves * kTS;
    const int64_t chans = (int64_t)g.B * g.D;
    const Place p = place_of<CPL>(g, length, lane);
    const int t0 = seg * g.seg_len, t1 = min(t0 + g.seg_len, g.T);
    const E* x0 = x + p.b * g.x_batch + p.d;
    const E* f0 = f + p.b * g.f_batch + p.d;
    const E* g0 = grad_h ? grad_h + p.b * g.g_batch + p.d : nullptr;
    const int64_t row0 = (int64_t)p.b * g.T * g.D + p.d;
    const int nm = (g.T + LIF_GATED_MARK - 1) / LIF_GATED_MARK;
    const float* mk = marks + (int64_t)p.b * nm * g.D + p.d;

    Raw<E, CPL, 3> cur, nxt;
    float h_cur[CPL], h_nxt[CPL];
    auto load = [&](Raw<E, CPL, 3>& r, float (&h)[CPL], int tt) {
        load_steps<E, CPL>(r.v[0], f0, g.f_time, tt + w * kTS, p);
        load_steps<E, CPL>(r.v[1], x0, g.x_time, tt + w * kTS, p);
        if (g0) load_steps<E, CPL>(r.v[2], g0, g.g_time, tt + w * kTS, p);
        load_elems<float, CPL>(mk + (int64_t)(tt / LIF_GATED_MARK) * g.D, h);
    };
    int tt = t1 > t0 ? t0 + (t1 - t0 - 1) / tile * tile : t0 - tile;
    if (tt >= t0) load(cur, h_cur, tt);

    float mu[CPL];                      // the adjoint carried into the tile from the later side
#pragma unroll
    for (int k = 0; k < CPL; ++k) mu[k] = grad_last ? grad_last[p.c + k] : 0.0f;
    fold_segments<CPL>(mu, maps, chans, p.c, g.S - 1, g.S - 1 - seg, -1);

    int buf = 0;
    for (; tt >= t0; tt -= tile, buf ^= 1) {
        const int t = tt + w * kTS;
        if (tt >= p.n_max) {            // past every lane's length
            if (tt - tile >= t0) load(nxt, h_nxt, tt - tile);
            if (p.live) {
                E o[CPL];
#pragma unroll
                for (int k = 0; k < CPL; ++k) o[k] = from_f32<E>(0.0f);
#pragma unroll
                for (int i = 0; i < kTS; ++i)
                    if (t + i < t1) {
                        store_elems<E, CPL>(grad_x + row0 + (int64_t)(t + i) * g.D, o);
                        store_elems<E, CPL>(grad_f + row0 + (int64_t)(t + i) * g.D, o);
                    }
            }
        } else {
            if (tt - tile >= t0) load(nxt, h_nxt, tt - tile);
            float a[kTS][CPL], na[kTS][CPL], A[CPL], H[CPL], M[CPL];
#pragma unroll
            for (int k = 0; k < CPL; ++k) A[k] = 1.0f, H[k] = 0.0f, M[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < kTS; ++i) {
                const bool on = t + i < p.n;
#pragma unroll
                for (int k = 0; k < CPL; ++k) {
                    float s, ns;
                    gate(to_f32(cur.v[0][i][k]), s, ns);
                    a[i][k] = on ? s : 1.0f;
                    na[i][k] = on ? ns : 0.0f;
                    const float v = to_f32(cur.v[1][i][k]);
                    H[k] = fmaf(a[i][k], H[k], on ? (COUPLED ? ns * v : v) : 0.0f);
                    A[k] *= a[i][k];
                }
            }
#pragma unroll
            for (int i = kTS - 1; i >= 0; --i)
#pragma unroll
                for (int k = 0; k < CPL; ++k)
                    M[k] = a[i][k] * (M[k] + (g0 && t + i < p.n ? to_f32(cur.v[2][i][k]) : 0.0f));
#pragma unroll
            for (int k = 0; k < CPL; ++k) {
                sh[buf][w][k][0][lane] = A[k];
                sh[buf][w][k][1][lane] = H[k];
                sh[buf][w][k][2][lane] = M[k];
            }
            __syncthreads();
            float h[CPL], lam[CPL];
#pragma unroll
            for (int k = 0; k < CPL; ++k) {
                h[k] = h_cur[k];
                for (int q = 0; q < w; ++q) h[k] = fmaf(sh[buf][q][k][0][lane], h[k], sh[buf][q][k][1][lane]);
                for (int q = kMaxWaves - 1; q >= 0; --q) {
                    if (q == w) lam[k] = mu[k];
                    mu[k] = fmaf(sh[buf][q][k][0][lane], mu[k], sh[buf][q][k][2][lane]);
                }
            }
            float before[kTS][CPL];
#pragma unroll
            for (int i = 0; i < kTS; ++i)
#pragma unroll
                for (int k = 0; k < CPL; ++k) {
                    before[i][k] = h[k];
                    const float v = to_f32(cur.v[1][i][k]);
                    h[k] = fmaf(a[i][k], h[k], t + i < p.n ? (COUPLED ? na[i][k] * v : v) : 0.0f);
                }
#pragma unroll
            for (int i = kTS - 1; i >= 0; --i) {
                E ox[CPL], of[CPL];
                const bool on = t + i < p.n;
#pragma unroll
                for (int k = 0; k < CPL; ++k) {
                    if (g0 && on) lam[k] += to_f32(cur.v[2][i][k]);
                    const float v = to_f32(cur.v[1][i][k]);
                    ox[k] = from_f32<E>(on ? (COUPLED ? lam[k] * na[i][k] : lam[k]) : 0.0f);
                    of[k] = from_f32<E>(on ? lam[k] * (COUPLED ? before[i][k] - v : before[i][k]) *
                                                 (a[i][k] * na[i][k]) : 0.0f);
                    lam[k] *= a[i][k];
                }
                if (p.live && t + i < t1) {
                    store_elems<E, CPL>(grad_x + row0 + (int64_t)(t + i) * g.D, ox);
                    store_elems<E, CPL>(grad_f + row0 + (int64_t)(t + i) * g.D, of);
                }
            }
        }
        cur = nxt;
#pragma unroll
        for (int k = 0; k < CPL; ++k) h_cur[k] = h_nxt[k];
    }
    if (grad_first && seg == 0 && w == 0 && p.live) store_elems<float, CPL>(grad_first + p.c, mu);
}

template <typename E, int CPL>
__global__ __launch_bounds__(256) void k_gated_step(const E* __restrict__ x, const E* __restrict__ f,
                                                    const int32_t* __restrict__ slot, float* __restrict__ state,
                                                    int n_slots, lif_gated_params p, E* __restrict__ h_out)
{
    const int per = p.D / CPL;
    const int64_t cg = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (cg >= (int64_t)p.B * per) return;
    const int b = (int)(cg / per), d = (int)(cg - (int64_t)b * per) * CPL;
    const int s = slot ? slot[b] : b;
    E o[CPL];
    if (s >= 0 && s < n_slots) {
        E xv[CPL], fv[CPL];
        float h[CPL];
        float* at = state + (int64_t)s * p.D + d;
        load_elems<E, CPL>(x + b * p.x_batch + d, xv);
        load_elems<E, CPL>(f + b * p.f_batch + d, fv);
        load_elems<float, CPL>(at, h);
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
            float a, na;
            gate(to_f32(fv[k]), a, na);
            const float v = to_f32(xv[k]);
            h[k] = fmaf(a, h[k], (p.flags & LIF_GATED_COUPLED) ? na * v : v);
            o[k] = from_f32<E>(h[k]);
        }
        store_elems<float, CPL>(at, h);
    } else {
#pragma unroll
        for (int k = 0; k < CPL; ++k) o[k] = from_f32<E>(0.0f);
    }
    store_elems<E, CPL>(h_out + (int64_t)b * p.D + d, o);
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

// Channels per lane and segments of the time axis.
struct Plan {
    int cpl;
    Geometry g;
};

Plan plan_of(const lif_gated_params& p)
{
    Plan q;
    const int64_t chans = (int64_t)p.B * p.D;
    // the widest group of up to 8 bytes that divides a row and leaves two workgroups for every CU
    q.cpl = p.dtype == LIF_F32 ? 2 : 4;
    while (q.cpl > 1 && (p.D % q.cpl != 0 || chans / q.cpl < 512 * kWave)) q.cpl >>= 1;
    Geometry& g = q.g;
    g.B = p.B;
    g.T = p.T;
    g.D = p.D;
    g.groups = (int)(chans / q.cpl);
    g.per_sample = p.D / q.cpl;
    const int columns = (g.groups + kWave - 1) / kWave;
    const int blocks = (p.T + LIF_GATED_MARK - 1) / LIF_GATED_MARK;
    int S = 1;
    if (columns < 128 && blocks > 4) {
        S = (1024 + columns - 1) / columns;
        if (S > (blocks + 3) / 4) S = (blocks + 3) / 4;
    }
    const int per = S > 0 ? (blocks + S - 1) / S : 1;
    g.seg_len = (per > 0 ? per : 1) * LIF_GATED_MARK;
    g.S = p.T > 0 ? (p.T + g.seg_len - 1) / g.seg_len : 1;
    g.x_batch = p.x_batch;
    g.x_time = p.x_time;
    g.f_batch = p.f_batch;
    g.f_time = p.f_time;
    g.g_batch = p.g_batch;
    g.g_time = p.g_time;
    return q;
}

size_t ws_size(const Plan& q) { return q.g.S > 1 ? (size_t)q.g.S * q.g.B * q.g.D * sizeof(float2) : 0; }

template <int N> struct Int { static constexpr int value = N; };

// Calls fn(element, channels per lane, coupled) with types that carry them.
template <typename Fn> void dispatch(const Plan& q, const lif_gated_params& p, Fn&& fn)
{
    with_dtype(p.dtype, [&](auto e) {
        auto with = [&](auto cpl) {
            if (p.flags & LIF_GATED_COUPLED) fn(e, cpl, Int<1>());
            else fn(e, cpl, Int<0>());
        };
        if constexpr (sizeof(e) == 2)
            if (q.cpl == 4) return with(Int<4>());
        if (q.cpl == 2) return with(Int<2>());
        with(Int<1>());
    });
}

}  // namespace
}  // namespace lif

extern "C" size_t lif_gated_scan_workspace_size(const lif_gated_params* p)
{
    if (lif::check_gated(p) != LIF_OK) return 0;
    return lif::ws_size(lif::plan_of(*p));
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
    const Plan q = plan_of(*p);
    const size_t need = ws_size(q);
    if (need > 0 && !ws) return LIF_ERR_ARG;
    if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    if (chans == 0) return LIF_OK;
    const Geometry& g = q.g;
    const unsigned columns = (unsigned)((g.groups + kWave - 1) / kWave);
    int nw = 1;                          // no more waves than the sequence has groups of TS steps
    while (nw < kMaxWaves && nw * kTS < p->T) nw *= 2;
    dispatch(q, *p, [&](auto e, auto cpl, auto coupled) {
        using E = decltype(e);
        constexpr int C = decltype(cpl)::value;
        constexpr bool K = decltype(coupled)::value;
        if (g.S > 1)
            TIMED_LAUNCH("gated_maps", (k_segment_maps<E, C, K, false>), dim3(columns, g.S - 1), dim3(kMaxWaves * kWave),
                         0, (hipStream_t)stream, (const E*)x, (const E*)f, length, g, (float2*)ws);
        TIMED_LAUNCH("gated_scan", (k_scan<E, C, K>), dim3(columns, g.S), dim3(nw * kWave), 0, (hipStream_t)stream,
                     (const E*)x, (const E*)f, length, h_first, g, (const float2*)ws, (E*)h, h_last, marks);
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
    const Plan q = plan_of(*p);
    const size_t need = ws_size(q);
    if (need > 0 && !ws) return LIF_ERR_ARG;
    if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    if (chans == 0) return LIF_OK;
    const Geometry& g = q.g;
    const unsigned columns = (unsigned)((g.groups + kWave - 1) / kWave);
    dispatch(q, *p, [&](auto e, auto cpl, auto coupled) {
        using E = decltype(e);
        constexpr int C = decltype(cpl)::value;
        constexpr bool K = decltype(coupled)::value;
        if (g.S > 1)
            TIMED_LAUNCH("gated_maps_back", (k_segment_maps<E, C, K, true>), dim3(columns, g.S - 1),
                         dim3(kMaxWaves * kWave), 0, (hipStream_t)stream, (const E*)grad_h, (const E*)f, length, g,
                         (float2*)ws);
        TIMED_LAUNCH("gated_back", (k_back<E, C, K>), dim3(columns, g.S), dim3(kMaxWaves * kWave), 0,
                     (hipStream_t)stream, (const E*)x, (const E*)f, length, marks, (const E*)grad_h, grad_last, g,
                     (const float2*)ws, (E*)grad_x, (E*)grad_f, grad_h_first);
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
    // four channels per lane where a row divides by them and enough lanes are left for every CU
    const bool wide = p->D % 4 == 0 && chans >= 4 * 256 * 256;
    with_dtype(p->dtype, [&](auto tag) {
        using E = decltype(tag);
        const int64_t lanes = wide ? chans / 4 : chans;
        const dim3 grid((unsigned)((lanes + 255) / 256));
        if (wide)
            TIMED_LAUNCH("gated_step", (k_gated_step<E, 4>), grid, dim3(256), 0, (hipStream_t)stream, (const E*)x,
                         (const E*)f, slot, state, n_slots, *p, (E*)h);
        else
            TIMED_LAUNCH("gated_step", (k_gated_step<E, 1>), grid, dim3(256), 0, (hipStream_t)stream, (const E*)x,
                         (const E*)f, slot, state, n_slots, *p, (E*)h);
    });
    return check_launch();
}
