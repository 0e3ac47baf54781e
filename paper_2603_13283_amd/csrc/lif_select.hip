// lif_select.hip -- the selective state space scan (lif_selective_scan), its
// gradient (lif_selective_scan_backward) and its single step on a pool of
// states (lif_selective_step).
//
// A lane holds one channel, a wave NS of its N states, a workgroup of W waves
// 64 channels with all their states, in registers for as long as it walks along
// time.  So B_t and C_t are the same for all lanes, and what a state needs of
// its step (delta, delta x) is made once per channel: a tile of LIF_SELECT_MARK
// steps goes through three phases, with a barrier between them:
//   A  the waves share out the tile's steps and put delta and delta x of their
//      steps into LDS, and B and C as float32
//   B  each wave runs all steps of the tile on its states and leaves its part
//      of sum_i C_t[i] h_t[i] in LDS
//   C  the waves share out the steps again, add up the parts, and write y
// Raw inputs of the next tile are loaded while a tile is worked on.
#include "lif_host.hpp"
#include "lif_types.hpp"
#include "lif_walk.hpp"

namespace lif {
namespace {

constexpr int kTile = LIF_SELECT_MARK;
constexpr float kLog2e = 1.44269504088896341f;
static_assert(kTile == 16, "the sums over lanes below put 16 steps x 4 states into the lanes of a wave");

// What a call works on.  Columns of 64 channels: column c is sample
// c / (G cols), group c / cols % G, channels 64 (c % cols) .. of that group.
struct Geometry {
    int B, T, D, N, G, Dg, cols;
    uint32_t flags;
    int64_t x_batch, x_time, dt_batch, dt_time, z_batch, z_time, b_batch, b_time, c_batch, c_time, g_batch, g_time;
};

struct Inputs {
    const void *x, *dt, *Bm, *C, *z, *gy;
    const float *A, *skip, *bias;
    const int32_t* length;
};

__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

// A workgroup's column, and a lane's channel in it.  Lanes past the group's
// last channel repeat it, with inputs of 0, and store nothing.
struct Place {
    int b, g, col, d, n;
    bool live;
};

__device__ __forceinline__ Place place_of(const Geometry& q, const int32_t* __restrict__ length, int lane)
{
    Place p;
    const int c = blockIdx.x;
    p.col = c % q.cols;
    p.g = c / q.cols % q.G;
    p.b = c / q.cols / q.G;
    const int at = p.col * kWave + lane;
    p.live = at < q.Dg;
    p.d = p.g * q.Dg + (p.live ? at : q.Dg - 1);
    p.n = length ? min(max(length[p.b], 0), q.T) : q.T;
    p.n = __builtin_amdgcn_readfirstlane(p.n);
    return p;
}

// e^{-|r|}, to a few units of 2^-24: the power of two of the rounded product,
// and to first order what the rounding left out.
__device__ __forceinline__ float exp_neg(float r)
{
    const float q = -fabsf(r), p = q * kLog2e;
    const float left = fmaf(q, kLog2e, -p) + q * 1.92596299e-8f;       // log2 e - kLog2e
    const float e = __builtin_amdgcn_exp2f(p);
    return fmaf(e, left * 0.693147181f, e);
}

// log(1 + e^r) = max(r, 0) + log1p(e^{-|r|}), and its derivative.  With
// s = e / (2 + e) <= 1/3, log1p(e) = 2 atanh(s) = 2 (s + s^3/3 + s^5/5 + ...):
// relative to the value to a few units of 2^-24 however small e is (the ninth
// term is 9^-8 / 17 of the first).
__device__ __forceinline__ float softplus(float r, float& slope)
{
    const float e = exp_neg(r);
    const float s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
    float v = 1.0f / 15.0f;
    v = fmaf(v, q, 1.0f / 13.0f);
    v = fmaf(v, q, 1.0f / 11.0f);
    v = fmaf(v, q, 1.0f / 9.0f);
    v = fmaf(v, q, 1.0f / 7.0f);
    v = fmaf(v, q, 1.0f / 5.0f);
    v = fmaf(v, q, 1.0f / 3.0f);
    v = fmaf(v, q, 1.0f);
    const float k = __builtin_amdgcn_rcpf(1.0f + e);
    slope = r >= 0.0f ? k : e * k;
    return (r != r) ? r : fmaf(2.0f * s, v, fmaxf(r, 0.0f));
}

__device__ __forceinline__ float step_length(const Geometry& q, float r, float& slope)
{
    if (q.flags & LIF_SELECT_SOFTPLUS) return softplus(r, slope);
    slope = 1.0f;
    return r;
}

// s(z) = z / (1 + e^-z) and its derivative.
__device__ __forceinline__ float silu(float z, float& slope)
{
    const float k = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * z));
    slope = k * fmaf(z, 1.0f - k, 1.0f);
    return z * k;
}

// A log2 e, the exponent per unit of delta.  An infinite A keeps a = 1 for
// delta = 0 (steps past the length inside a tile).
__device__ __forceinline__ float rate_of(float a)
{
    const float v = a * kLog2e;
    return fabsf(v) > 3.0e38f ? copysignf(3.0e38f, v) : v;
}

// The raw elements of a tile that one thread loads: the steps w, w + W, ... of
// its wave for its lane's channel, and a share of B and C.
template <typename E, int NS, int W, int IN>
struct Raw {
    static constexpr int kSteps = kTile / W;
    static constexpr int kShare = kTile * NS / kWave > 0 ? kTile * NS / kWave : 1;
    E v[IN][kSteps];
    E bc[2][kShare];
};

// Which share of a tile's B and C a thread brings: element j is step t[j],
// state n[j] (on[j] false: none, or past N).
template <int NS, int W> struct Share {
    static constexpr int kShare = kTile * NS / kWave > 0 ? kTile * NS / kWave : 1;
    int t[kShare], n[kShare];
    bool there[kShare], on[kShare];
    __device__ __forceinline__ Share(int N)
    {
#pragma unroll
        for (int j = 0; j < kShare; ++j) {
            const int i = threadIdx.x + j * W * kWave;
            n[j] = i % (W * NS);
            t[j] = i / (W * NS);
            there[j] = t[j] < kTile;
            on[j] = there[j] && n[j] < N;
        }
    }
};

template <typename E, int NS, int W, int IN>
__device__ __forceinline__ void load_bc(Raw<E, NS, W, IN>& r, const Share<NS, W>& s, const E* __restrict__ Bm,
                                        const E* __restrict__ C, const Geometry& q, const Place& p, int t0)
{
#pragma unroll
    for (int j = 0; j < Raw<E, NS, W, IN>::kShare; ++j) {
        r.bc[0][j] = r.bc[1][j] = from_f32<E>(0.0f);
        const int t = t0 + s.t[j];
        if (s.on[j] && t < p.n) {
            r.bc[0][j] = Bm[p.b * q.b_batch + t * q.b_time + p.g * q.N + s.n[j]];
            r.bc[1][j] = C[p.b * q.c_batch + t * q.c_time + p.g * q.N + s.n[j]];
        }
    }
}

// Puts B and C of a tile into LDS: per step and wave, NS of B and then NS of C.
template <typename E, int NS, int W, int IN>
__device__ __forceinline__ void store_bc(const Raw<E, NS, W, IN>& r, const Share<NS, W>& s, float* sh)
{
#pragma unroll
    for (int j = 0; j < Raw<E, NS, W, IN>::kShare; ++j)
        if (s.there[j]) {
            float* at = sh + (s.t[j] * W + s.n[j] / NS) * 2 * NS + s.n[j] % NS;
            at[0] = to_f32(r.bc[0][j]);
            at[NS] = to_f32(r.bc[1][j]);
        }
}

template <typename E, int NS, int W>
__global__ __launch_bounds__(W* kWave) void k_select_scan(Inputs in, Geometry q, const float* __restrict__ h_first,
                                                          E* __restrict__ y, float* __restrict__ h_last,
                                                          float* __restrict__ marks)
{
    constexpr int kSteps = kTile / W;
    __shared__ float2 shD[kTile][kWave];
    __shared__ float4 shBC[kTile * W * 2 * NS / 4];
    __shared__ float shY[W][kTile][kWave];
    const int lane = threadIdx.x & 63, w = wave_index();
    const Place p = place_of(q, in.length, lane);
    const Share<NS, W> share(q.N);
    const int n0 = w * NS, used = (q.N + NS - 1) / NS;
    const E *x = (const E*)in.x, *dt = (const E*)in.dt, *z = (const E*)in.z;
    float h[NS], rate[NS];
#pragma unroll
    for (int k = 0; k < NS; ++k) {
        const bool on = p.live && n0 + k < q.N;
        rate[k] = on ? rate_of(in.A[(int64_t)p.d * q.N + n0 + k]) : 0.0f;
        h[k] = on && h_first ? h_first[((int64_t)p.b * q.D + p.d) * q.N + n0 + k] : 0.0f;
    }
    const float bias = in.bias ? in.bias[p.d] : 0.0f, skip = in.skip ? in.skip[p.d] : 0.0f;

    Raw<E, NS, W, 3> cur, nxt;
    auto load = [&](Raw<E, NS, W, 3>& r, int t0) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int t = t0 + w + W * i;
            r.v[0][i] = r.v[1][i] = r.v[2][i] = from_f32<E>(0.0f);
            if (t < p.n) {
                r.v[0][i] = x[p.b * q.x_batch + t * q.x_time + p.d];
                r.v[1][i] = dt[p.b * q.dt_batch + t * q.dt_time + p.d];
                if (z && y) r.v[2][i] = z[p.b * q.z_batch + t * q.z_time + p.d];
            }
        }
        load_bc(r, share, (const E*)in.Bm, (const E*)in.C, q, p, t0);
    };
    if (p.n > 0) load(cur, 0);
    for (int t0 = 0; t0 < p.n; t0 += kTile) {
        const int cnt = min(kTile, p.n - t0);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            float slope;
            const float d = step_length(q, to_f32(cur.v[1][i]) + bias, slope);
            shD[w + W * i][lane] = p.live ? make_float2(d, d * to_f32(cur.v[0][i])) : make_float2(0.0f, 0.0f);
        }
        store_bc(cur, share, (float*)shBC);
        if (t0 + kTile < p.n) load(nxt, t0 + kTile);
        __syncthreads();
        if (n0 < q.N) {
            if (marks && p.live)
#pragma unroll
                for (int k = 0; k < NS; ++k)
                    if (n0 + k < q.N)
                        marks[(((int64_t)p.b * ((q.T + kTile - 1) / kTile) + t0 / kTile) * q.N + n0 + k) * q.D + p.d] =
                            h[k];
            auto step = [&](int i) {
                const float2 v = shD[i][lane];
                const float* bc = (const float*)shBC + (i * W + w) * 2 * NS;
                float sum = 0.0f;
#pragma unroll
                for (int k = 0; k < NS; ++k) {
                    const float a = __builtin_amdgcn_exp2f(v.x * rate[k]);
                    h[k] = fmaf(a, h[k], v.y * bc[k]);
                    sum = fmaf(bc[NS + k], h[k], sum);
                }
                shY[w][i][lane] = sum;
            };
            if (cnt == kTile) {
#pragma unroll
                for (int i = 0; i < kTile; ++i) step(i);
            } else {
                for (int i = 0; i < cnt; ++i) step(i);
            }
        }
        __syncthreads();
        if (y) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int t = t0 + w + W * i;
                if (t < p.n) {
                    float v = skip * to_f32(cur.v[0][i]);
                    for (int j = 0; j < used; ++j) v += shY[j][w + W * i][lane];
                    float slope;
                    if (z) v *= silu(to_f32(cur.v[2][i]), slope);
                    if (p.live) y[((int64_t)p.b * q.T + t) * q.D + p.d] = from_f32<E>(v);
                }
            }
        }
        cur = nxt;
    }
    if (!p.live) return;
    if (y)
        for (int t = p.n + w; t < q.T; t += W) y[((int64_t)p.b * q.T + t) * q.D + p.d] = from_f32<E>(0.0f);
    if (h_last)
#pragma unroll
        for (int k = 0; k < NS; ++k)
            if (n0 + k < q.N) h_last[((int64_t)p.b * q.D + p.d) * q.N + n0 + k] = h[k];
}

// ---------------------------------------------------------------------------
// Gradient.  The adjoint lambda_t = C_t g_t + mu, mu = a_{t+1} lambda_{t+1},
// runs backwards through the tiles; a tile's states are run forward again from
// its mark and kept in registers.
// ---------------------------------------------------------------------------

template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// Sums over the lanes of several values at once: each merge takes two values
// and leaves the sum of the first over pairs of lanes in one half of them and
// that of the second in the other half, so that 64 values end as one sum per
// lane, at about two instructions a value.
__device__ __forceinline__ float merge_halves(float a, float b)        // lanes 0-31: a, 32-63: b
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b),
                                                    false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ float merge_rows(float a, float b)          // even rows of 16 lanes: a, odd rows: b
{
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b),
                                                    false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
template <int CTRL> __device__ __forceinline__ float merge_in_row(float a, float b, bool second)
{
    return (second ? b : a) + dpp<CTRL>(second ? a : b);
}

// Four values of a step: rows 0 .. 3 of the wave get the sums of v[0], v[2],
// v[1], v[3] over the four rows.
__device__ __forceinline__ float merge_states(const float (&v)[4])
{
    return merge_rows(merge_halves(v[0], v[1]), merge_halves(v[2], v[3]));
}

// 16 steps: lane l gets its row's sum of step l % 16.
__device__ __forceinline__ float merge_steps(const float (&v)[16], int lane)
{
    float a[8], b[4], c[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = merge_in_row<0x128>(v[i], v[i + 8], lane & 8);      // lane ^ 8
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = merge_in_row<0x141>(a[i], a[i + 4], lane & 4);      // lane ^ 7
#pragma unroll
    for (int i = 0; i < 2; ++i) c[i] = merge_in_row<0x4e>(b[i], b[i + 2], lane & 2);       // lane ^ 2
    return merge_in_row<0xb1>(c[0], c[1], lane & 1);                                       // lane ^ 1
}

template <typename E> struct BackOut {
    E *gx, *gdt, *gz;
    float *partB, *partC;         // [B G cols][T][N] sums over a column's channels
    float *partA;                 // [B][D][N]
    float *partS;                 // [B][2][D]: of skip, of dt_bias
    float *g_first;
};

template <typename E, int W, int NB>
__global__ __launch_bounds__(W* kWave) void k_select_back(Inputs in, Geometry q, const float* __restrict__ marks,
                                                          const float* __restrict__ grad_last, BackOut<E> out)
{
    constexpr int kSteps = kTile / W, NS = 4;
    __shared__ float shD[3][kTile][kWave];                    // delta, delta x, g
    __shared__ float4 shBC[NB][kTile * W * 2 * NS / 4];
    __shared__ float shP[W][kTile][kWave], shQ[W][kTile][kWave], shY[W][kTile][kWave];
    const int lane = threadIdx.x & 63, w = wave_index();
    const Place p = place_of(q, in.length, lane);
    const Share<NS * NB, W> share(q.N);
    const int used = min(W, (q.N + NS - 1) / NS);
    const E *x = (const E*)in.x, *dt = (const E*)in.dt, *z = (const E*)in.z, *gy = (const E*)in.gy;
    float mu[NB][NS], A[NB][NS], rate[NB][NS], gA[NB][NS];
    auto state = [&](int nb, int k) { return (nb * W + w) * NS + k; };
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int k = 0; k < NS; ++k) {
            const int n = state(nb, k);
            const bool on = p.live && n < q.N;
            A[nb][k] = on ? in.A[(int64_t)p.d * q.N + n] : 0.0f;
            rate[nb][k] = rate_of(A[nb][k]);
            mu[nb][k] = on && grad_last ? grad_last[((int64_t)p.b * q.D + p.d) * q.N + n] : 0.0f;
            gA[nb][k] = 0.0f;
        }
    const float bias = in.bias ? in.bias[p.d] : 0.0f, skip = in.skip ? in.skip[p.d] : 0.0f;
    float g_skip = 0.0f, g_bias = 0.0f;

    Raw<E, NS * NB, W, 4> cur, nxt;
    auto load = [&](Raw<E, NS * NB, W, 4>& r, int t0) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int t = t0 + w + W * i;
            r.v[0][i] = r.v[1][i] = r.v[2][i] = r.v[3][i] = from_f32<E>(0.0f);
            if (t < p.n) {
                r.v[0][i] = x[p.b * q.x_batch + t * q.x_time + p.d];
                r.v[1][i] = dt[p.b * q.dt_batch + t * q.dt_time + p.d];
                if (z) r.v[2][i] = z[p.b * q.z_batch + t * q.z_time + p.d];
                if (gy) r.v[3][i] = gy[p.b * q.g_batch + t * q.g_time + p.d];
            }
        }
        load_bc(r, share, (const E*)in.Bm, (const E*)in.C, q, p, t0);
    };
    const int64_t column = blockIdx.x;
    const int last = (p.n - 1) / kTile * kTile;
    if (p.n > 0) load(cur, last);
    for (int t0 = last; t0 >= 0 && p.n > 0; t0 -= kTile) {
        const int cnt = min(kTile, p.n - t0);
        float delta[kSteps], g[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            float slope;
            delta[i] = step_length(q, to_f32(cur.v[1][i]) + bias, slope);
            g[i] = to_f32(cur.v[3][i]);
            if (z) g[i] *= silu(to_f32(cur.v[2][i]), slope);
            const bool on = p.live && w + W * i < cnt;
            shD[0][w + W * i][lane] = on ? delta[i] : 0.0f;
            shD[1][w + W * i][lane] = on ? delta[i] * to_f32(cur.v[0][i]) : 0.0f;
            shD[2][w + W * i][lane] = on ? g[i] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < Share<NS * NB, W>::kShare; ++j)
            if (share.there[j]) {
                const int n = share.n[j], slice = n / NS;            // slice nb * W + w
                float* at = (float*)shBC[slice / W] + (share.t[j] * W + slice % W) * 2 * NS + n % NS;
                at[0] = to_f32(cur.bc[0][j]);
                at[NS] = to_f32(cur.bc[1][j]);
            }
        if (t0 > 0) load(nxt, t0 - kTile);
        __syncthreads();
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            if (state(nb, 0) >= q.N) continue;
            float h0[NS];
#pragma unroll
            for (int k = 0; k < NS; ++k)
                h0[k] = p.live && state(nb, k) < q.N
                            ? marks[(((int64_t)p.b * ((q.T + kTile - 1) / kTile) + t0 / kTile) * q.N + state(nb, k)) *
                                        q.D + p.d]
                            : 0.0f;
            auto walk = [&](auto whole) {
                constexpr bool kWhole = decltype(whole)::value;
                float h[kTile][NS], a[kTile][NS], vb[kTile], vc[kTile];
#pragma unroll
                for (int i = 0; i < kTile; ++i) {
                    if (!kWhole && i >= cnt) continue;
                    const float* bc = (const float*)shBC[nb] + (i * W + w) * 2 * NS;
                    const float d = shD[0][i][lane], u = shD[1][i][lane];
                    float sum = 0.0f;
#pragma unroll
                    for (int k = 0; k < NS; ++k) {
                        a[i][k] = __builtin_amdgcn_exp2f(d * rate[nb][k]);
                        h[i][k] = fmaf(a[i][k], i ? h[i - 1][k] : h0[k], u * bc[k]);
                        sum = fmaf(bc[NS + k], h[i][k], sum);
                    }
                    shY[w][i][lane] = nb ? shY[w][i][lane] + sum : sum;
                }
#pragma unroll
                for (int i = kTile - 1; i >= 0; --i) {
                    vb[i] = vc[i] = 0.0f;
                    if (!kWhole && i >= cnt) continue;
                    const float* bc = (const float*)shBC[nb] + (i * W + w) * 2 * NS;
                    const float d = shD[0][i][lane], u = shD[1][i][lane], gg = shD[2][i][lane];
                    float P = 0.0f, Q = 0.0f, pb[NS], pc[NS];
#pragma unroll
                    for (int k = 0; k < NS; ++k) {
                        const float lam = fmaf(gg, bc[NS + k], mu[nb][k]);
                        pc[k] = gg * h[i][k];
                        pb[k] = lam * u;
                        Q = fmaf(lam, bc[k], Q);
                        mu[nb][k] = a[i][k] * lam;
                        const float f = mu[nb][k] * (i ? h[i - 1][k] : h0[k]);
                        P = fmaf(A[nb][k], f, P);
                        gA[nb][k] = fmaf(d, f, gA[nb][k]);
                    }
                    shP[w][i][lane] = nb ? shP[w][i][lane] + P : P;
                    shQ[w][i][lane] = nb ? shQ[w][i][lane] + Q : Q;
                    vb[i] = merge_states(pb);
                    vc[i] = merge_states(pc);
                }
                const float sb = merge_steps(vb, lane), sc = merge_steps(vc, lane);
                const int row = lane >> 4, n = state(nb, (row & 1) * 2 + (row >> 1)), i = lane & 15;
                if (i < cnt && n < q.N) {
                    const int64_t at = (column * q.T + t0 + i) * q.N + n;
                    out.partB[at] = sb;
                    out.partC[at] = sc;
                }
            };
            if (cnt == kTile) walk(std::true_type());
            else walk(std::false_type());
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int s = w + W * i, t = t0 + s;
            if (t < p.n) {
                float P = 0.0f, Q = 0.0f, Y = 0.0f;
                for (int j = 0; j < used; ++j) P += shP[j][s][lane], Q += shQ[j][s][lane], Y += shY[j][s][lane];
                const float xv = to_f32(cur.v[0][i]);
                float slope;
                step_length(q, to_f32(cur.v[1][i]) + bias, slope);
                const float g_r = fmaf(xv, Q, P) * slope;
                g_skip = fmaf(g[i], xv, g_skip);
                g_bias += g_r;
                if (p.live) {
                    const int64_t at = ((int64_t)p.b * q.T + t) * q.D + p.d;
                    out.gx[at] = from_f32<E>(fmaf(delta[i], Q, skip * g[i]));
                    out.gdt[at] = from_f32<E>(g_r);
                    if (z) {
                        silu(to_f32(cur.v[2][i]), slope);
                        out.gz[at] = from_f32<E>(to_f32(cur.v[3][i]) * fmaf(skip, xv, Y) * slope);
                    }
                }
            }
        }
        cur = nxt;
    }
    if (p.live) {
        for (int t = p.n + w; t < q.T; t += W) {
            const int64_t at = ((int64_t)p.b * q.T + t) * q.D + p.d;
            out.gx[at] = out.gdt[at] = from_f32<E>(0.0f);
            if (z) out.gz[at] = from_f32<E>(0.0f);
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int k = 0; k < NS; ++k)
                if (state(nb, k) < q.N) {
                    const int64_t at = ((int64_t)p.b * q.D + p.d) * q.N + state(nb, k);
                    out.partA[at] = gA[nb][k];
                    if (out.g_first) out.g_first[at] = mu[nb][k];
                }
    }
    __syncthreads();
    shP[w][0][lane] = g_skip;
    shP[w][1][lane] = g_bias;
    __syncthreads();
    if (w == 0 && p.live) {
        float s0 = 0.0f, s1 = 0.0f;
        for (int j = 0; j < W; ++j) s0 += shP[j][0][lane], s1 += shP[j][1][lane];
        out.partS[(int64_t)p.b * 2 * q.D + p.d] = s0;
        out.partS[((int64_t)p.b * 2 + 1) * q.D + p.d] = s1;
    }
}

// Adds up the columns' parts of grad_B and grad_C, and the samples' parts of
// the parameters' gradients, in the order of columns and samples.
template <typename E>
__global__ __launch_bounds__(256) void k_select_sums(Geometry q, const int32_t* __restrict__ length,
                                                     const float* __restrict__ partB, const float* __restrict__ partC,
                                                     const float* __restrict__ partA, const float* __restrict__ partS,
                                                     E* __restrict__ gB, E* __restrict__ gC, float* __restrict__ gA,
                                                     float* __restrict__ g_skip, float* __restrict__ g_bias,
                                                     int64_t bc_blocks)
{
    const int64_t states = (int64_t)q.D * q.N;
    if (blockIdx.x < bc_blocks) {
        const int64_t per = (int64_t)q.T * q.N, all = q.B * q.G * per;
        for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += bc_blocks * 256) {
            const int64_t bg = at / per, rest = at - bg * per;
            const int t = (int)(rest / q.N), n = (int)(rest - (int64_t)t * q.N);
            const int b = (int)(bg / q.G), g = (int)(bg % q.G);
            float sb = 0.0f, sc = 0.0f;
            if (t < (length ? min(max(length[b], 0), q.T) : q.T))
#pragma unroll 8
                for (int c = 0; c < q.cols; ++c) {
                    sb += partB[(bg * q.cols + c) * per + rest];
                    sc += partC[(bg * q.cols + c) * per + rest];
                }
            const int64_t to = (((int64_t)b * q.T + t) * q.G + g) * q.N + n;
            gB[to] = from_f32<E>(sb);
            gC[to] = from_f32<E>(sc);
        }
        return;
    }
    const int64_t at = (int64_t)(blockIdx.x - bc_blocks) * 256 + threadIdx.x;
    if (at < states) {
        float s = 0.0f;
#pragma unroll 8
        for (int b = 0; b < q.B; ++b) s += partA[b * states + at];
        gA[at] = s;
    } else if (at < states + 2 * q.D) {
        const int64_t i = at - states;                        // skip's, then dt_bias'
        float s = 0.0f;
#pragma unroll 8
        for (int b = 0; b < q.B; ++b) s += partS[(int64_t)b * 2 * q.D + i];
        float* to = i < q.D ? g_skip : g_bias;
        if (to) to[i < q.D ? i : i - q.D] = s;
    }
}

// ---------------------------------------------------------------------------
// One step.  L lanes share a channel (L a power of two with 4 L >= N), each
// holds four of its states.
// ---------------------------------------------------------------------------

template <typename E>
__global__ __launch_bounds__(256) void k_select_step(Inputs in, const int32_t* __restrict__ slot,
                                                     float* __restrict__ state, int n_slots, Geometry q, int L,
                                                     E* __restrict__ y)
{
    const int64_t at = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    const bool live = at < (int64_t)q.B * q.D;
    const int64_t c = live ? at : (int64_t)q.B * q.D - 1;
    const int b = (int)(c / q.D), d = (int)(c - (int64_t)b * q.D), g = d / q.Dg, n0 = threadIdx.x % L * 4;
    const int row = slot ? slot[b] : b;
    const bool there = row >= 0 && row < n_slots;
    const float xv = to_f32(((const E*)in.x)[b * q.x_batch + d]);
    float slope;
    const float r = to_f32(((const E*)in.dt)[b * q.dt_batch + d]) + (in.bias ? in.bias[d] : 0.0f);
    const float delta = step_length(q, r, slope), u = delta * xv;
    float sum = 0.0f;
    if (there && n0 < q.N) {
        const E* Bt = (const E*)in.Bm + b * q.b_batch + g * q.N + n0;
        const E* Ct = (const E*)in.C + b * q.c_batch + g * q.N + n0;
        float* h = state + ((int64_t)row * q.D + d) * q.N + n0;
        const float* A = in.A + (int64_t)d * q.N + n0;
        auto run = [&](float a, float hv, E bv, E cv) {
            const float v = fmaf(__builtin_amdgcn_exp2f(delta * rate_of(a)), hv, u * to_f32(bv));
            sum = fmaf(to_f32(cv), v, sum);
            return v;
        };
        if (n0 + 4 <= q.N) {
            float av[4], hv[4];
            E bv[4], cv[4];
            load_elems<float, 4>(A, av);
            load_elems<float, 4>(h, hv);
            load_elems<E, 4>(Bt, bv);
            load_elems<E, 4>(Ct, cv);
#pragma unroll
            for (int k = 0; k < 4; ++k) hv[k] = run(av[k], hv[k], bv[k], cv[k]);
            if (live) store_elems<float, 4>(h, hv);
        } else {
            for (int k = 0; n0 + k < q.N; ++k) {
                const float v = run(A[k], h[k], Bt[k], Ct[k]);
                if (live) h[k] = v;
            }
        }
    }
    for (int o = L >> 1; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (live && n0 == 0) {
        sum = fmaf(in.skip ? in.skip[d] : 0.0f, xv, sum);
        if (in.z) sum *= silu(to_f32(((const E*)in.z)[b * q.z_batch + d]), slope);
        y[c] = from_f32<E>(there ? sum : 0.0f);
    }
}

int check_select(const lif_select_params* p)
{
    if (!p || p->B < 0 || p->T < 0 || p->D < 1 || p->N < 1 || p->G < 1 || p->reserved != 0 ||
        (p->flags & ~LIF_SELECT_SOFTPLUS))
        return LIF_ERR_ARG;
    if (p->D % p->G != 0) return LIF_ERR_ARG;
    if (p->dtype != LIF_F32 && p->dtype != LIF_BF16 && p->dtype != LIF_F16) return LIF_ERR_ARG;
    const int64_t strides[] = {p->x_batch, p->x_time, p->dt_batch, p->dt_time, p->z_batch, p->z_time,
                               p->b_batch, p->b_time, p->c_batch, p->c_time, p->g_batch, p->g_time};
    for (int64_t s : strides)
        if (s < 0) return LIF_ERR_ARG;
    if (p->N > LIF_SELECT_MAX_STATES || (int64_t)p->B * p->D >= ((int64_t)1 << 26) || p->T > (1 << 30))
        return LIF_ERR_SIZE;
    // products of sizes stay within 64 bits, and a launch has fewer than 2^32
    // threads, at up to 512 for a column
    if ((int64_t)p->B * p->D * p->T >= ((int64_t)1 << 44) / p->N) return LIF_ERR_SIZE;
    const int64_t cols = (p->D / p->G + kWave - 1) / kWave;
    if (p->B * p->G * cols >= ((int64_t)1 << 32) / (8 * kWave)) return LIF_ERR_SIZE;
    return LIF_OK;
}

Geometry geometry_of(const lif_select_params& p)
{
    Geometry q;
    q.B = p.B, q.T = p.T, q.D = p.D, q.N = p.N, q.G = p.G;
    q.Dg = p.D / p.G;
    q.cols = (q.Dg + kWave - 1) / kWave;
    q.flags = p.flags;
    q.x_batch = p.x_batch, q.x_time = p.x_time, q.dt_batch = p.dt_batch, q.dt_time = p.dt_time;
    q.z_batch = p.z_batch, q.z_time = p.z_time, q.b_batch = p.b_batch, q.b_time = p.b_time;
    q.c_batch = p.c_batch, q.c_time = p.c_time, q.g_batch = p.g_batch, q.g_time = p.g_time;
    return q;
}

template <int V> struct Int { static constexpr int value = V; };

// Calls fn(states of a wave, waves) with types that carry them: the fewest
// waves that hold N states.
template <typename Fn> void with_waves(int N, Fn&& fn)
{
    if (N <= 4) fn(Int<4>(), Int<1>());
    else if (N <= 8) fn(Int<4>(), Int<2>());
    else if (N <= 16) fn(Int<4>(), Int<4>());
    else if (N <= 32) fn(Int<4>(), Int<8>());
    else fn(Int<8>(), Int<8>());
}

size_t align16(size_t n) { return (n + 15) & ~(size_t)15; }

struct BackLayout {
    size_t partB, partC, partA, partS, total;
};

BackLayout back_layout(const lif_select_params& p)
{
    const Geometry q = geometry_of(p);
    BackLayout l;
    const size_t bc = align16(sizeof(float) * q.B * q.G * q.cols * (size_t)q.T * q.N);
    l.partB = 0;
    l.partC = bc;
    l.partA = 2 * bc;
    l.partS = l.partA + align16(sizeof(float) * q.B * (size_t)q.D * q.N);
    l.total = l.partS + align16(sizeof(float) * 2 * q.B * (size_t)q.D);
    return l;
}

}  // namespace
}  // namespace lif

extern "C" size_t lif_selective_scan_workspace_size(const lif_select_params* p)
{
    using namespace lif;
    if (check_select(p) != LIF_OK) return 0;
    return 0;
}

extern "C" int lif_selective_scan(const void* x, const void* dt, const float* A, const void* Bm, const void* C,
                                  const float* skip, const void* z, const float* dt_bias, const int32_t* length,
                                  const float* h_first, const lif_select_params* p, void* y, float* h_last,
                                  float* marks, void* ws, size_t ws_bytes, lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_select(p);
    if (rc) return rc;
    if (p->B > 0 && p->T > 0 && (!x || !dt || !Bm || !C)) return LIF_ERR_ARG;
    if (p->B > 0 && (!A || (!y && !h_last && !marks))) return LIF_ERR_ARG;
    if (p->B == 0) return LIF_OK;
    const Geometry q = geometry_of(*p);
    const Inputs in = {x, dt, Bm, C, z, nullptr, A, skip, dt_bias, length};
    const dim3 grid((unsigned)(q.B * q.G * q.cols));
    with_dtype(p->dtype, [&](auto e) {
        using E = decltype(e);
        with_waves(q.N, [&](auto ns, auto waves) {
            constexpr int NS = decltype(ns)::value, W = decltype(waves)::value;
            TIMED_LAUNCH("select_scan", (k_select_scan<E, NS, W>), grid, dim3(W * kWave), 0, (hipStream_t)stream, in, q,
                         h_first, (E*)y, h_last, marks);
        });
    });
    return check_launch();
}

extern "C" size_t lif_selective_scan_backward_workspace_size(const lif_select_params* p)
{
    using namespace lif;
    if (check_select(p) != LIF_OK) return 0;
    return back_layout(*p).total;
}

extern "C" int lif_selective_scan_backward(const void* x, const void* dt, const float* A, const void* Bm,
                                           const void* C, const float* skip, const void* z, const float* dt_bias,
                                           const int32_t* length, const float* marks, const void* grad_y,
                                           const float* grad_last, const lif_select_params* p, void* grad_x,
                                           void* grad_dt, float* grad_A, void* grad_B, void* grad_C, float* grad_skip,
                                           void* grad_z, float* grad_dt_bias, float* grad_h_first, void* ws,
                                           size_t ws_bytes, lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_select(p);
    if (rc) return rc;
    if (p->B > 0 && p->T > 0 &&
        (!x || !dt || !Bm || !C || !marks || !grad_x || !grad_dt || !grad_B || !grad_C || (z && !grad_z)))
        return LIF_ERR_ARG;
    if (!A || !grad_A) return LIF_ERR_ARG;
    const BackLayout l = back_layout(*p);
    if (l.total > 0 && (!ws || (uintptr_t)ws % 16)) return LIF_ERR_ARG;
    if (ws_bytes < l.total) return LIF_ERR_WORKSPACE;
    const Geometry q = geometry_of(*p);
    const Inputs in = {x, dt, Bm, C, z, grad_y, A, skip, dt_bias, length};
    const int64_t bc = (int64_t)q.B * q.G * q.T * q.N;
    const int64_t bc_blocks = bc > ((int64_t)1 << 30) ? 1 << 22 : (bc + 255) / 256;
    const int64_t blocks = bc_blocks + ((int64_t)q.D * (q.N + 2) + 255) / 256;
    with_dtype(p->dtype, [&](auto e) {
        using E = decltype(e);
        char* base = (char*)ws;
        const BackOut<E> out = {(E*)grad_x, (E*)grad_dt, (E*)grad_z, (float*)(base + l.partB),
                                (float*)(base + l.partC), (float*)(base + l.partA), (float*)(base + l.partS),
                                grad_h_first};
        auto launch = [&](auto waves, auto nb) {
            constexpr int W = decltype(waves)::value, NB = decltype(nb)::value;
            TIMED_LAUNCH("select_back", (k_select_back<E, W, NB>), dim3((unsigned)(q.B * q.G * q.cols)),
                         dim3(W * kWave), 0, (hipStream_t)stream, in, q, marks, grad_last, out);
        };
        if (q.B > 0) {
            if (q.N <= 4) launch(Int<1>(), Int<1>());
            else if (q.N <= 8) launch(Int<2>(), Int<1>());
            else if (q.N <= 16) launch(Int<4>(), Int<1>());
            else if (q.N <= 32) launch(Int<8>(), Int<1>());
            else launch(Int<8>(), Int<2>());
        }
        TIMED_LAUNCH("select_sums", (k_select_sums<E>), dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, q,
                     length, out.partB, out.partC, out.partA, out.partS, (E*)grad_B, (E*)grad_C, grad_A, grad_skip,
                     grad_dt_bias, bc_blocks);
    });
    return check_launch();
}

extern "C" int lif_selective_step(const void* x, const void* dt, const float* A, const void* Bm, const void* C,
                                  const float* skip, const void* z, const float* dt_bias, const int32_t* slot,
                                  float* state, int n_slots, const lif_select_params* p, void* y, lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_select(p);
    if (rc) return rc;
    if (p->T != 1 || n_slots < 0 || (!slot && n_slots < p->B)) return LIF_ERR_ARG;
    if (p->B == 0) return LIF_OK;
    if (!x || !dt || !A || !Bm || !C || !y || (n_slots > 0 && !state)) return LIF_ERR_ARG;
    const Geometry q = geometry_of(*p);
    const Inputs in = {x, dt, Bm, C, z, nullptr, A, skip, dt_bias, nullptr};
    int L = 1;
    while (4 * L < q.N) L *= 2;
    const int64_t blocks = ((int64_t)q.B * q.D + 256 / L - 1) / (256 / L);
    with_dtype(p->dtype, [&](auto e) {
        using E = decltype(e);
        TIMED_LAUNCH("select_step", (k_select_step<E>), dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, in,
                     slot, state, n_slots, q, L, (E*)y);
    });
    return check_launch();
}
