// lif_select.hip -- the selective state space scan (lif_selective_scan), its
// gradient (lif_selective_scan_backward) and its single step on a pool of
// states (lif_selective_step).
//
// A lane holds one channel, a wave NS of its N states, a workgroup of W waves
// 64 channels with all their states, in registers for as long as it walks along
// time.  What a state needs of its step (delta, delta x) is made once per channel
// and shared through LDS: a tile of LIF_SELECT_MARK steps goes through three
// phases:
//   A  the waves share out the tile's steps and put delta and delta x of their
//      steps into LDS
//   B  each wave runs all steps of the tile on its states and leaves its part
//      of sum_i C_t[i] h_t[i] in LDS
//   C  the waves share out the steps again, add up the parts, and write y
// B_t and C_t are the same for all lanes: those of the tile's 16 steps lie in the
// 16 lanes of each row, where the vector unit's row broadcast reads them.
#include "lif_host.hpp"
#include "lif_types.hpp"
#include "lif_walk.hpp"

#include <type_traits>
#include <utility>

namespace lif {
namespace {

constexpr int kTile = LIF_SELECT_MARK;
constexpr float kLog2e = 1.44269504088896341f;
constexpr int kMaxOrder = 512;         // samples that are put in order
constexpr int kStepPairs = 8192;       // workgroups of a step from which they take two streams at a time
// The time axis is cut into segments where there are at most kSplitColumns
// columns, into as many as give kSplitWaves waves and at least kSplitTiles tiles
// each; kSplitLeast segments pay for reading the inputs twice.  In us, cut and
// not: 8 columns of 65521 steps 302 and 5700, 128 of 1000 (training, 8 states)
// 171 and 370, 32 of 1000 33 and 118; 192 of 2048 220 and 190.  2 x 4096 x 1024
// x 16, training: 287 us with 4096 waves, 329 with 8192.
constexpr int kMaxSegments = 256, kSplitColumns = 128, kSplitWaves = 4096, kSplitTiles = 4, kSplitLeast = 4;
static_assert(kTile == 16, "the sums over lanes below put 16 steps x 4 states into the lanes of a wave");

// What a call works on.  Columns of 64 channels: column c is sample
// c / (G cols), group c / cols % G, channels 64 (c % cols) .. of that group.
// S segments of seg_len steps (whole tiles) of the time axis.
struct Geometry {
    int B, T, D, N, G, Dg, cols, columns, S, seg_len;
    bool ordered;                 // samples in the order of their length
    uint32_t flags;
    int64_t x_batch, x_time, dt_batch, dt_time, z_batch, z_time, b_batch, b_time, c_batch, c_time, g_batch, g_time;
};

struct Inputs {
    const void *x, *dt, *Bm, *C, *z, *gy;
    const float *A, *skip, *bias;
    const int32_t* length;
};

__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

// A workgroup's column and segment, and a lane's channel in it.  Lanes past the
// group's last channel repeat it and store nothing.  The segment is steps t0 ..
// t1 - 1, of which the first n lie before the sample's length.
struct Place {
    int b, g, d, column, seg, t0, t1, n, length;
    bool live;
};

// The sample of this length's rank, longest first, the first of equals first:
// workgroups start in the order of their index, so the long samples do not come
// last (128 samples of 0 to 1000 steps x 512 channels: 263 -> 200 us).  The whole
// workgroup calls it, and scratch (B + 1 words of LDS) is free again after the
// next barrier.
__device__ __forceinline__ int sample_of(const int32_t* __restrict__ length, int B, int T, int rank, int* scratch)
{
    int *lengths = scratch + 1, &found = *scratch;
    for (int i = threadIdx.x; i < B; i += blockDim.x) lengths[i] = min(max(length[i], 0), T);
    __syncthreads();
    for (int i = threadIdx.x; i < B; i += blockDim.x) {
        const int n = lengths[i];
        int r = 0;
        for (int j = 0; j < B; ++j) r += lengths[j] > n || (lengths[j] == n && j < i);
        if (r == rank) found = i;
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(found);
}

__device__ __forceinline__ Place place_of(const Geometry& q, const int32_t* __restrict__ length, int lane,
                                          int* scratch)
{
    Place p;
    p.seg = blockIdx.x / q.columns;
    p.column = blockIdx.x - p.seg * q.columns;
    p.g = p.column / q.cols % q.G;
    p.b = p.column / q.cols / q.G;
    if (q.ordered && length) {
        p.b = sample_of(length, q.B, q.T, p.b, scratch);
        p.column = (p.b * q.G + p.g) * q.cols + p.column % q.cols;
    }
    const int at = p.column % q.cols * kWave + lane;
    p.live = at < q.Dg;
    p.d = p.g * q.Dg + (p.live ? at : q.Dg - 1);
    p.length = length ? min(max(length[p.b], 0), q.T) : q.T;
    p.length = __builtin_amdgcn_readfirstlane(p.length);
    p.t0 = p.seg * q.seg_len;
    p.t1 = min(p.t0 + q.seg_len, q.T);
    p.n = max(min(p.length, p.t1) - p.t0, 0);
    return p;
}

// log(1 + e^r) = max(r, 0) + log1p(e^{-|r|}), and its derivative, to a few
// units of 2^-24 relative to the value.  e^{-|r|} is the power of two of the
// rounded product, corrected to first order by what the rounding left out.
// With s = 2 e / (2 + e) <= 2/3, log1p(e) = 2 atanh(s / 2) = s v(s^2), v a power
// series with v(0) = 1; its polynomial of degree 4 that is best over [0, 4/9]
// relative to the value is off by 0.8 10^-8.
__device__ __forceinline__ float softplus(float r, float& slope)
{
    const float m = fminf(fabsf(r), 128.0f), p = -kLog2e * m;         // e is 0 from |r| = 104 on
    const float left = fmaf(m, -1.92596299e-8f, fmaf(m, -kLog2e, -p));       // log2 e - kLog2e = 1.9 10^-8
    float e = __builtin_amdgcn_exp2f(p);
    e = fmaf(e, left * 0.693147181f, e);
    const float s = e * __builtin_amdgcn_rcpf(fmaf(e, 0.5f, 1.0f)), q = s * s;
    float v = fmaf(q, 5.50358106e-4f, 2.18442209e-3f);
    v = fmaf(v, q, 1.25077845e-2f);
    v = fmaf(v, q, 8.33328934e-2f);
    v = fmaf(v, q, 1.0f);
    const float k = __builtin_amdgcn_rcpf(1.0f + e);
    slope = r >= 0.0f ? k : e * k;
    return fmaf(s, v, r <= 0.0f ? 0.0f : r);                          // 0 for -infinity, and a NaN stays one
}

__device__ __forceinline__ float step_length(const Geometry& q, float r, float& slope)
{
    const bool soft = q.flags & LIF_SELECT_SOFTPLUS;
    const float v = softplus(r, slope);
    slope = soft ? slope : 1.0f;
    return soft ? v : r;
}

// s(z) = z / (1 + e^-z) and its derivative.
__device__ __forceinline__ float silu(float z, float& slope)
{
    const float k = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * z));
    slope = k * fmaf(z, 1.0f - k, 1.0f);
    return z * k;
}

// A log2 e, the exponent per unit of delta.  An infinite A keeps a = 1 for
// delta = 0 (a masked step, steps past the length inside a tile).
__device__ __forceinline__ float rate_of(float a)
{
    const float v = a * kLog2e;
    return fabsf(v) > 3.0e38f ? copysignf(3.0e38f, v) : v;
}

// A as it enters the gradient of delta, A a lambda h: an infinite A has a = 0 and
// no slope for any delta > 0, and is given none at 0.
__device__ __forceinline__ float slope_of(float a) { return fabsf(a) == INFINITY ? 0.0f : a; }

template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// B_t[i] (or C_t[i]) of 16 steps lie in the lanes of each row of 16, step l % 16
// in lane l.  An instruction of the vector unit reads the value of step I for
// all lanes through its first operand.
template <int I> __device__ __forceinline__ float of_step(float v) { return dpp<0x150 | I>(v); }

// acc[j] += v of step I + j times x[j], for four steps.  The compiler has no
// such sum; the wait lets a write of v by the instruction before arrive.  Sums are
// written before the last inputs are read: no input may share a register with one,
// not even where both hold the same value.
template <int I> __device__ __forceinline__ void add_steps(float* acc, float v, float x0, float x1, float x2, float x3)
{
    asm("s_nop 1\n\t"
        "v_fmac_f32_dpp %0, %4, %5 row_newbcast:%9 row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %1, %4, %6 row_newbcast:%10 row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %2, %4, %7 row_newbcast:%11 row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %3, %4, %8 row_newbcast:%12 row_mask:0xf bank_mask:0xf"
        : "+&v"(acc[0]), "+&v"(acc[1]), "+&v"(acc[2]), "+&v"(acc[3])
        : "v"(v), "v"(x0), "v"(x1), "v"(x2), "v"(x3), "n"(I), "n"(I + 1), "n"(I + 2), "n"(I + 3));
}

// a += u of step I times x, b += v of step I times x.
template <int I> __device__ __forceinline__ void add_step(float& a, float& b, float u, float v, float x)
{
    asm("s_nop 1\n\t"
        "v_fmac_f32_dpp %0, %2, %4 row_newbcast:%5 row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %1, %3, %4 row_newbcast:%5 row_mask:0xf bank_mask:0xf"
        : "+&v"(a), "+&v"(b)
        : "v"(u), "v"(v), "v"(x), "n"(I));
}

template <int I> using Step = std::integral_constant<int, I>;
// fn(Step<0>()) .. fn(Step<15>()), or in reverse.
template <typename Fn, int... I>
__device__ __forceinline__ void each_of(Fn&& fn, std::integer_sequence<int, I...>)
{
    (fn(Step<I>()), ...);
}
template <typename Fn> __device__ __forceinline__ void each_step(Fn&& fn)
{
    each_of(fn, std::make_integer_sequence<int, kTile>());
}
template <typename Fn> __device__ __forceinline__ void each_step_back(Fn&& fn)
{
    each_of([&](auto i) { fn(Step<kTile - 1 - decltype(i)::value>()); }, std::make_integer_sequence<int, kTile>());
}

// An element on its way from memory, in a register of its own: the compiler
// packs pairs of 16-bit ones into one register, and waits for the loads to do
// so.
template <typename E> struct Bits {
    using type = std::conditional_t<sizeof(E) == 2, uint16_t, uint32_t>;
    uint32_t v;
    __device__ __forceinline__ void load(const E* at) { v = *reinterpret_cast<const type*>(at); }
    __device__ __forceinline__ float f32() const { return to_f32(__builtin_bit_cast(E, (type)v)); }
};

// The raw elements of a tile that one lane loads: IN inputs of its channel for
// the steps that its wave makes ready, w STEPS .. (w + 1) STEPS - 1, and B and
// C of step lane % 16 for the wave's states.
template <typename E, int NS, int STEPS, int IN> struct Raw {
    Bits<E> v[IN][STEPS];
    Bits<E> bc[2][NS];
};

// A lane's offset as a value of the place where it is used: otherwise its
// widening to 64 bits moves out of the loop, and every address is added up by
// the vector unit instead of in the access.
__device__ __forceinline__ uint32_t here(uint32_t offset)
{
    asm volatile("" : "+v"(offset));
    return offset;
}

// One input along time: the scalar address of a step's row, and bytes from one
// row to the next; a lane's channel is an offset to it.
struct Rows {
    const char* at;
    int64_t step;
};
template <typename E> __device__ __forceinline__ Rows rows_of(const void* in, int64_t batch, int64_t time, int b, int t)
{
    return {(const char*)((const E*)in + b * batch + t * time), time * (int64_t)sizeof(E)};
}
// STEPS steps, of which `there` are before the end; the last of those is
// repeated in place of the others.
template <typename E, int STEPS>
__device__ __forceinline__ void load_rows(Bits<E> (&v)[STEPS], const Rows& r, uint32_t offset, int there = STEPS)
{
    const char* at = r.at;
    offset = here(offset);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        v[i].load((const E*)(at + offset));
        if (i + 1 < there) at += r.step;
    }
}

// Where there are few columns, the time axis is cut into segments that
// workgroups share out.  A segment's map of the state that enters it is
//   h -> e^{A sum delta} h + H,
// one sum of delta per channel and one H per state: a first launch makes them,
// and every segment then starts from the maps before it.  The adjoint's maps
// (REVERSE: mu -> e^{A sum delta} mu + M) go the other way.
//   sums [S][B][D], ends [S][B][N][D]
template <typename E, int NS, int W, bool REVERSE>
__global__ __launch_bounds__(W* kWave) void k_select_maps(Inputs in, Geometry q, float* __restrict__ sums,
                                                          float* __restrict__ ends)
{
    constexpr int STEPS = kTile / W, IN = REVERSE ? 3 : 2;
    __shared__ float4 shD[2][kTile / 2][kWave];               // delta and delta x (delta and g) of two steps
    const int lane = threadIdx.x & 63, w = wave_index();
    Place p = place_of(q, in.length, lane, (int*)shD);
    if (REVERSE) {                                            // the first segment needs no map
        p.t0 += q.seg_len, p.t1 = min(p.t1 + q.seg_len, q.T), ++p.seg;
        p.n = max(min(p.length, p.t1) - p.t0, 0);
    }
    const int n0 = w * NS, s0 = w * STEPS;
    float h[NS], rate[NS], total = 0.0f;
    int at[NS];
#pragma unroll
    for (int k = 0; k < NS; ++k) {
        rate[k] = n0 + k < q.N ? rate_of(in.A[(int64_t)p.d * q.N + n0 + k]) : 0.0f;
        h[k] = 0.0f;
        at[k] = min(n0 + k, q.N - 1);
    }
    const float bias = in.bias ? in.bias[p.d] : 0.0f;
    const uint32_t offset = p.d * (uint32_t)sizeof(E);
    const bool gated = in.z != nullptr, driven = in.gy != nullptr;

    Raw<E, NS, STEPS, IN> r0, r1, r2;
    auto load = [&](Raw<E, NS, STEPS, IN>& r, int from) {
        const int left = p.n - from, t = p.t0 + from + min(s0, left - 1);
        const Rows dt = rows_of<E>(in.dt, q.dt_batch, q.dt_time, p.b, t);
        load_rows(r.v[0], dt, offset, left - s0);
        if constexpr (REVERSE) {
            load_rows(r.v[1], driven ? rows_of<E>(in.gy, q.g_batch, q.g_time, p.b, t) : dt, offset, left - s0);
            load_rows(r.v[2], gated ? rows_of<E>(in.z, q.z_batch, q.z_time, p.b, t) : dt, offset, left - s0);
        } else {
            load_rows(r.v[1], rows_of<E>(in.x, q.x_batch, q.x_time, p.b, t), offset, left - s0);
        }
        const int64_t tb = p.t0 + from + min(lane & 15, left - 1);
        const E* bc = REVERSE ? (const E*)in.C + p.b * q.c_batch + tb * q.c_time
                              : (const E*)in.Bm + p.b * q.b_batch + tb * q.b_time;
#pragma unroll
        for (int k = 0; k < NS; ++k) r.bc[0][k].load(bc + (int64_t)p.g * q.N + at[k]);
    };
    // steps past the end have delta = 0: the identity
    auto ready = [&](const Raw<E, NS, STEPS, IN>& r, float4 (*to)[kWave], int left) {
#pragma unroll
        for (int i = 0; i < STEPS; i += 2) {
            float slope, dl[2], u[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const bool on = s0 + i + j < left;
                dl[j] = step_length(q, r.v[0][i + j].f32() + bias, slope);
                u[j] = r.v[1][i + j].f32();
                if constexpr (REVERSE) {
                    const float s = silu(r.v[2][i + j].f32(), slope);
                    u[j] = !driven ? 0.0f : gated ? u[j] * s : u[j];
                } else {
                    u[j] *= dl[j];
                }
                dl[j] = on ? dl[j] : 0.0f, u[j] = on ? u[j] : 0.0f;
            }
            to[(s0 + i) / 2][lane] = make_float4(dl[0], u[0], dl[1], u[1]);
        }
    };
    auto walk = [&](const Raw<E, NS, STEPS, IN>& r, const float4 (*from)[kWave]) {
        float B[NS];
        float4 v[kTile / 2];
#pragma unroll
        for (int i = 0; i < kTile / 2; ++i) v[i] = from[i][lane];
#pragma unroll
        for (int k = 0; k < NS; ++k) B[k] = n0 + k < q.N ? r.bc[0][k].f32() : 0.0f;
        float part = 0.0f;                                    // of the tile: long sums go in two levels
        auto step = [&](auto at_step) {
            constexpr int i = decltype(at_step)::value;
            const float dl = i % 2 ? v[i / 2].z : v[i / 2].x, u = i % 2 ? v[i / 2].w : v[i / 2].y;
            part += dl;
#pragma unroll
            for (int k = 0; k < NS; ++k) {
                const float a = __builtin_amdgcn_exp2f(dl * rate[k]), b = u * of_step<i>(B[k]);
                h[k] = REVERSE ? a * (h[k] + b) : fmaf(a, h[k], b);
            }
        };
        if constexpr (REVERSE) each_step_back(step);
        else each_step(step);
        total += part;
    };
    const int tiles = (p.n + kTile - 1) / kTile;
    if (tiles > 0) {
        int j = 0;
        auto from = [&](int i) { return (REVERSE ? tiles - 1 - i : i) * kTile; };
        auto turn = [&](const auto& cur, const auto& next, auto& far) {
            if (j + 2 < tiles) load(far, from(j + 2));
            if (j + 1 < tiles) ready(next, shD[(j + 1) & 1], p.n - from(j + 1));
            if (n0 < q.N) walk(cur, shD[j & 1]);
            __syncthreads();
            return ++j < tiles;
        };
        load(r0, from(0));
        if (tiles > 1) load(r1, from(1));
        ready(r0, shD[0], p.n - from(0));
        __syncthreads();
        while (turn(r0, r1, r2) && turn(r1, r2, r0) && turn(r2, r0, r1)) {
        }
    }
    if (!p.live) return;
    const int64_t row = (int64_t)p.seg * q.B + p.b;
    if (w == 0) sums[row * q.D + p.d] = total;
#pragma unroll
    for (int k = 0; k < NS; ++k)
        if (n0 + k < q.N) ends[(row * q.N + n0 + k) * q.D + p.d] = h[k];
}

// c carried through the maps of segments from, from + by, ... (count of them).
// With A > 0 (or negative step lengths) the factor of a segment can lie past the
// largest float while the state is 0 or small: 2^126 of it goes into c first.
template <int NS>
__device__ __forceinline__ void carry(float (&c)[NS], const float (&rate)[NS], const float* __restrict__ sums,
                                      const float* __restrict__ ends, const Geometry& q, const Place& p, int n0,
                                      int from, int count, int by)
{
#pragma unroll 4
    for (int i = 0; i < count; ++i) {
        const int64_t row = (int64_t)(from + i * by) * q.B + p.b;
        const float sum = fminf(sums[row * q.D + p.d], 3.0e38f);      // finite, for rates of 0
#pragma unroll
        for (int k = 0; k < NS; ++k) {
            const float v = fminf(sum * rate[k], 252.0f);
            const bool large = v > 126.0f;
            c[k] = fmaf(__builtin_amdgcn_exp2f(large ? v - 126.0f : v), large ? c[k] * 0x1p126f : c[k],
                        ends[(row * q.N + min(n0 + k, q.N - 1)) * q.D + p.d]);
        }
    }
}

// A scan is bound by the vector unit, 60 to 78 % busy (5.5 instructions a state
// and step: a product and 2^x for the decay, three and a half for state and
// readout; 60 a channel and step in phases A and C; an FMA takes 2.9 cycles of a
// SIMD, one with a broadcast 4.7, 2^x 8.5): 128 x 1000 x 512 x 16 bf16, ragged,
// 200 us; 8 x 2048 x 2048 x 16 bf16 with marks 230 us, 308 MB at 1.3 TB/s.
// The phases of three tiles run in one stretch between two barriers (B of a
// tile, C of the one before, A of the one after), so that the waits of one are
// filled by the others.  Only whole tiles go through that loop: it has no
// branches but for the stores.
template <typename E, int NS, int W>
__global__ __launch_bounds__(W* kWave) void k_select_scan(Inputs in, Geometry q, const float* __restrict__ h_first,
                                                          const float* __restrict__ sums,
                                                          const float* __restrict__ ends,
                                                          E* __restrict__ y, float* __restrict__ h_last,
                                                          float* __restrict__ marks)
{
    constexpr int STEPS = kTile / W;
    __shared__ float4 shD[2][kTile / 2][kWave];               // delta, delta x of two steps
    __shared__ float4 shY[2][W][kTile / 4][kWave];            // the waves' parts of y of four
    const int lane = threadIdx.x & 63, w = wave_index();
    const Place p = place_of(q, in.length, lane, (int*)shY);
    const int n0 = w * NS, s0 = w * STEPS;
    const bool gated = in.z != nullptr, busy = n0 < q.N;
    float h[NS], rate[NS];
    int at[NS];                                               // places past N repeat the last state, with B = C = 0
#pragma unroll
    for (int k = 0; k < NS; ++k) {
        const bool on = p.live && n0 + k < q.N;
        rate[k] = on ? rate_of(in.A[(int64_t)p.d * q.N + n0 + k]) : 0.0f;
        h[k] = on && h_first ? h_first[((int64_t)p.b * q.D + p.d) * q.N + n0 + k] : 0.0f;
        at[k] = min(n0 + k, q.N - 1);
    }
    if (p.n > 0) carry(h, rate, sums, ends, q, p, n0, 0, p.seg, 1);
    const float bias = in.bias ? in.bias[p.d] : 0.0f, skip = in.skip ? in.skip[p.d] : 0.0f;
    const uint32_t offset = p.d * (uint32_t)sizeof(E), offset4 = p.d * 4u;

    // From step t0 on: the rows of the wave's steps, and B and C of the lane's.
    const int64_t bt = q.b_time, ct = q.c_time;
    auto states_at = [&](const E* (&to)[2][NS], int t) {
        const E* Bt = (const E*)in.Bm + p.b * q.b_batch + t * bt + (int64_t)p.g * q.N;
        const E* Ct = (const E*)in.C + p.b * q.c_batch + t * ct + (int64_t)p.g * q.N;
#pragma unroll
        for (int k = 0; k < NS; ++k) to[0][k] = Bt + at[k], to[1][k] = Ct + at[k];
    };
    auto rows_at = [&](Rows (&to)[3], int t) {
        to[0] = rows_of<E>(in.x, q.x_batch, q.x_time, p.b, t);
        to[1] = rows_of<E>(in.dt, q.dt_batch, q.dt_time, p.b, t);
        to[2] = gated ? rows_of<E>(in.z, q.z_batch, q.z_time, p.b, t) : to[0];
    };
    auto load_states = [&](Raw<E, NS, STEPS, 3>& r, const E* const (&from)[2][NS]) {
#pragma unroll
        for (int k = 0; k < NS; ++k) r.bc[0][k].load(from[0][k]), r.bc[1][k].load(from[1][k]);
    };
    auto ready = [&](const Raw<E, NS, STEPS, 3>& r, float4 (*to)[kWave]) {
#pragma unroll
        for (int i = 0; i < STEPS; i += 2) {
            float slope, dl[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) dl[j] = step_length(q, r.v[1][i + j].f32() + bias, slope);
            to[(s0 + i) / 2][lane] = make_float4(dl[0], dl[0] * r.v[0][i].f32(), dl[1], dl[1] * r.v[0][i + 1].f32());
        }
    };
    // A tile's delta and delta x, read ahead of what comes between.
    auto fetch = [&](float4 (&to)[kTile / 2], const float4 (*from)[kWave]) {
#pragma unroll
        for (int i = 0; i < kTile / 2; ++i) to[i] = from[i][lane];
    };
    auto walk = [&](const Raw<E, NS, STEPS, 3>& r, const float4 (&at_step)[kTile / 2], float4 (*to)[kWave], auto whole,
                    int cnt) {
        float B[NS], Cv[NS], sum[kTile], hs[kTile][NS], a[kTile][NS];
#pragma unroll
        for (int k = 0; k < NS; ++k) {
            B[k] = n0 + k < q.N ? r.bc[0][k].f32() : 0.0f;
            Cv[k] = n0 + k < q.N ? r.bc[1][k].f32() : 0.0f;
        }
        auto decays = [&](int i) {
            const float dl = i % 2 ? at_step[i / 2].z : at_step[i / 2].x;
#pragma unroll
            for (int k = 0; k < NS; ++k) a[i][k] = __builtin_amdgcn_exp2f(dl * rate[k]);
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) decays(i);
        each_step([&](auto step) {
            constexpr int i = decltype(step)::value;
            if constexpr (i + 4 < kTile) decays(i + 4);
            if (decltype(whole)::value || i < cnt) {
                const float u = i % 2 ? at_step[i / 2].w : at_step[i / 2].y;
#pragma unroll
                for (int k = 0; k < NS; ++k) h[k] = fmaf(a[i][k], h[k], u * of_step<i>(B[k]));
            }
#pragma unroll
            for (int k = 0; k < NS; ++k) hs[i][k] = h[k];
            sum[i] = of_step<i>(Cv[0]) * h[0];
            if constexpr (i % 4 == 3) {
#pragma unroll
                for (int k = 1; k < NS; ++k)
                    add_steps<i - 3>(sum + i - 3, Cv[k], hs[i - 3][k], hs[i - 2][k], hs[i - 1][k], hs[i][k]);
                to[i / 4][lane] = make_float4(sum[i - 3], sum[i - 2], sum[i - 1], sum[i]);
                __builtin_amdgcn_sched_barrier(0);
            }
        });
    };
    auto put_marks = [&](int t0) {
        if (marks && p.live) {
            const int64_t tile = (int64_t)p.b * ((q.T + kTile - 1) / kTile) + (p.t0 + t0) / kTile;
            char* to = (char*)(marks + (tile * q.N + n0) * q.D);
            const uint32_t o = here(offset4);
#pragma unroll
            for (int k = 0; k < NS; ++k, to += q.D * (int64_t)4)
                if (n0 + k < q.N) *(float*)(to + o) = h[k];
        }
    };
    auto read_out = [&](const Raw<E, NS, STEPS, 3>& r, const float4 (*from)[kTile / 4][kWave], int t0, int cnt) {
        if (!y) return;
        float v[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) v[i] = skip * r.v[0][i].f32();
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int i = 0; i < STEPS; ++i) v[i] += ((const float*)&from[j][(s0 + i) / 4][lane])[(s0 + i) % 4];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            float slope;
            const float s = silu(r.v[2][i].f32(), slope);
            v[i] = gated ? v[i] * s : v[i];
        }
        char* to = (char*)(y + ((int64_t)p.b * q.T + p.t0 + t0 + s0) * q.D);
        if (p.live) {
            const uint32_t o = here(offset);
#pragma unroll
            for (int i = 0; i < STEPS; ++i, to += q.D * (int64_t)sizeof(E))
                if (s0 + i < cnt) *(E*)(to + o) = from_f32<E>(v[i]);
        }
    };

    __syncthreads();
    if (!busy)                                                // the parts of a wave without states stay 0
#pragma unroll
        for (int i = 0; i < kTile / 4; ++i)
            shY[0][w][i][lane] = shY[1][w][i][lane] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);

    // Four tiles' raw elements in turn: copies from one to the next would wait
    // for loads that are still on their way.
    const int whole = p.n / kTile;
    Raw<E, NS, STEPS, 3> r0, r1, r2, r3;
    if (whole > 0) {
        Rows rows[3];
        const E* states[2][NS];
        int j = -2;                                           // the tile that is loaded is j + 2
        auto load = [&](Raw<E, NS, STEPS, 3>& r) {
#pragma unroll
            for (int i = 0; i < 3; ++i) load_rows(r.v[i], rows[i], offset);
            load_states(r, states);
            if (j + 3 < whole) {                              // the last tile is loaded again where there are no more
#pragma unroll
                for (int i = 0; i < 3; ++i) rows[i].at += kTile * rows[i].step;
#pragma unroll
                for (int k = 0; k < NS; ++k) states[0][k] += kTile * bt, states[1][k] += kTile * ct;
            }
        };
        auto turn = [&](const auto& before, const auto& cur, const auto& next, auto& far) {
            load(far);
            put_marks(j * kTile);
            float4 steps[kTile / 2];
            fetch(steps, shD[j & 1]);
            __builtin_amdgcn_sched_barrier(0);
            ready(next, shD[(j + 1) & 1]);
            if (busy) walk(cur, steps, shY[j & 1][w], std::true_type(), kTile);
            if (j > 0) read_out(before, shY[(j - 1) & 1], (j - 1) * kTile, kTile);
            __syncthreads();
            if (++j < whole) return true;
            read_out(cur, shY[(j - 1) & 1], (j - 1) * kTile, kTile);
            return false;
        };
        rows_at(rows, p.t0 + s0);
        states_at(states, p.t0 + (lane & 15));
        load(r0), ++j;
        load(r1), ++j;
        ready(r0, shD[0]);
        __syncthreads();
        while (turn(r3, r0, r1, r2) && turn(r0, r1, r2, r3) && turn(r1, r2, r3, r0) && turn(r2, r3, r0, r1)) {
        }
        __syncthreads();
    }
    const int left = p.n - whole * kTile;
    if (left > 0) {
        const int t0 = whole * kTile;
        Rows rows[3];
        const E* states[2][NS];
        rows_at(rows, p.t0 + min(t0 + s0, p.n - 1));
        states_at(states, p.t0 + min(t0 + (lane & 15), p.n - 1));
#pragma unroll
        for (int i = 0; i < 3; ++i) load_rows(r0.v[i], rows[i], offset, left - s0);
        load_states(r0, states);
        put_marks(t0);
        ready(r0, shD[0]);
        __syncthreads();
        float4 steps[kTile / 2];
        fetch(steps, shD[0]);
        if (busy) walk(r0, steps, shY[0][w], std::false_type(), left);
        __syncthreads();
        read_out(r0, shY[0], t0, left);
    }
    if (!p.live) return;
    if (y)
        for (int t = p.t0 + p.n + w; t < p.t1; t += W) y[((int64_t)p.b * q.T + t) * q.D + p.d] = from_f32<E>(0.0f);
    // the segment that the sample ends in has the last state
    if (h_last && (p.n > 0 ? p.t0 + p.n == p.length : p.seg == 0 && p.length == 0))
#pragma unroll
        for (int k = 0; k < NS; ++k)
            if (n0 + k < q.N) h_last[((int64_t)p.b * q.D + p.d) * q.N + n0 + k] = h[k];
}

// ---------------------------------------------------------------------------
// Gradient.  The adjoint lambda_t = C_t g_t + mu, mu = a_{t+1} lambda_{t+1},
// runs backwards through the tiles; a tile's states are run forward again from
// its mark and kept in registers.
// ---------------------------------------------------------------------------

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

// Two values each of two states (or of one) of a step: rows 0 .. 3 of the wave
// get the sums over the four rows of the first state's b and c, and of the
// second's.
__device__ __forceinline__ float merge_states(float b0, float b1, float c0, float c1)
{
    return merge_rows(merge_halves(b0, b1), merge_halves(c0, c1));
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
    float *partA;                 // [S B][D][N]
    float *partS;                 // [S B][2][D]: of skip, of dt_bias
    float *g_first;
};

// Bound by the vector unit, 76 % busy: 14 instructions a state and step, 4 more
// for the sums over channels that grad_B and grad_C are, 100 a channel and step in
// phases A and C; 8 x 2048 x 2048 x 16 bf16 530 us, 477 MB at 0.9 TB/s.  A wave
// holds two states at a time, NB times over, so that a tile's states and decays
// fit its registers; what lasts from tile to tile is in LDS but for the first two
// (all in registers spill 113 a lane at 64 states: training, 8 x 2048 x 1024 x 64
// bf16 2550 us, this 1710; of 32 states 948 and 897).  Between two barriers a tile
// is walked; then its results are written while the tile before it is made ready
// and the one before that is on its way.
template <typename E, int W, int NB>
__global__ __launch_bounds__(W* kWave) void k_select_back(Inputs in, Geometry q, const float* __restrict__ marks,
                                                          const float* __restrict__ grad_last,
                                                          const float* __restrict__ sums,
                                                          const float* __restrict__ ends, BackOut<E> out)
{
    constexpr int STEPS = kTile / W, NS = 2;
    __shared__ float4 shD[kTile / 2][kWave];                  // delta, delta x of two steps
    __shared__ float2 shG[kTile / 2][kWave];                  // g of two
    __shared__ float2 shP[3][W][kTile / 2][kWave];            // the waves' parts of P, Q and y of two
    __shared__ float2 shS[NB > 1 ? NB - 1 : 1][3][W][kWave];  // mu, the gradient of A, and A of a wave's later states
    const int lane = threadIdx.x & 63, w = wave_index();
    const Place p = place_of(q, in.length, lane, (int*)shP);
    const int s0 = w * STEPS;
    const bool gated = in.z != nullptr, driven = in.gy != nullptr;
    auto first = [&](int nb) { return (nb * W + w) * NS; };
    // Of a wave's states, the first two are held in registers, the others in LDS.
    struct States {
        float mu[NS], A[NS], gA[NS];
    } held;
    const int segments = (p.length + q.seg_len - 1) / q.seg_len;       // that have steps
    // places past N repeat the last state, with B = C = 0
    const int at0[NS] = {min(first(0), q.N - 1), min(first(0) + 1, q.N - 1)};
    auto at = [&](int nb, int k) { return nb ? min(first(nb) + k, q.N - 1) : at0[k]; };
    auto begin = [&](int nb) {
        States s;
        float rate[NS];
#pragma unroll
        for (int k = 0; k < NS; ++k) {
            const int n = first(nb) + k;
            const bool on = p.live && n < q.N;
            s.A[k] = on ? in.A[(int64_t)p.d * q.N + n] : 0.0f;
            rate[k] = rate_of(s.A[k]);
            s.mu[k] = on && grad_last ? grad_last[((int64_t)p.b * q.D + p.d) * q.N + n] : 0.0f;
            s.gA[k] = 0.0f;
        }
        if (p.seg + 1 < segments)
            carry(s.mu, rate, sums, ends, q, p, first(nb), segments - 1, segments - 1 - p.seg, -1);
        return s;
    };
    auto keep = [&](int nb, const States& s) {
        shS[nb - 1][0][w][lane] = make_float2(s.mu[0], s.mu[1]);
        shS[nb - 1][1][w][lane] = make_float2(s.gA[0], s.gA[1]);
    };
    auto kept = [&](int nb) {
        const float2 mu = shS[nb - 1][0][w][lane], gA = shS[nb - 1][1][w][lane], A = shS[nb - 1][2][w][lane];
        return States{{mu.x, mu.y}, {A.x, A.y}, {gA.x, gA.y}};
    };
    held = begin(0);
#pragma unroll 1
    for (int nb = 1; nb < NB; ++nb) {
        const States s = begin(nb);
        keep(nb, s);
        shS[nb - 1][2][w][lane] = make_float2(s.A[0], s.A[1]);
    }
    const float bias = in.bias ? in.bias[p.d] : 0.0f, skip = in.skip ? in.skip[p.d] : 0.0f;
    float g_skip = 0.0f, g_bias = 0.0f;

    // A tile's raw elements and marks on their way, and what phase A makes of
    // the steps of this wave.  Of the states, the first two only: the others of a
    // tile are loaded while those before them are walked.
    Raw<E, NS, STEPS, 4> raw;
    float mark[NS];
    struct Made {
        float x[STEPS], delta[STEPS], slope[STEPS], g[STEPS], z_slope[STEPS];
        float B[NS], C[NS], h0[NS];
    } made;
    // Where the lane's steps of the tile that is loaded next lie, and where their
    // gradients go: addresses of the lanes, for as scalars they spill the scalar
    // registers (training, 8 x 2048 x 2048 x 16 bf16: 738 us, this 710).
    const char *in_at[4], *mark_at;
    const E *Bt, *Ct;
    char* out_at[3];
    const int64_t steps[4] = {q.x_time * (int64_t)sizeof(E), q.dt_time * (int64_t)sizeof(E),
                              (gated ? q.z_time : q.x_time) * (int64_t)sizeof(E),
                              (driven ? q.g_time : q.x_time) * (int64_t)sizeof(E)};
    const int64_t out_step = q.D * (int64_t)sizeof(E), mark_step = q.D * (int64_t)4;
    auto find = [&](int t0, int left) {
        const int t = p.t0 + t0 + min(s0, left - 1), tb = p.t0 + t0 + min(lane & 15, left - 1);
        auto lane_at = [&](const void* v, int64_t batch, int64_t time) {
            return (const char*)((const E*)v + p.b * batch + t * time + p.d);
        };
        in_at[0] = lane_at(in.x, q.x_batch, q.x_time);
        in_at[1] = lane_at(in.dt, q.dt_batch, q.dt_time);
        in_at[2] = gated ? lane_at(in.z, q.z_batch, q.z_time) : in_at[0];
        in_at[3] = driven ? lane_at(in.gy, q.g_batch, q.g_time) : in_at[0];
        Bt = (const E*)in.Bm + p.b * q.b_batch + tb * q.b_time + (int64_t)p.g * q.N;
        Ct = (const E*)in.C + p.b * q.c_batch + tb * q.c_time + (int64_t)p.g * q.N;
        mark_at = (const char*)(marks + ((int64_t)p.b * ((q.T + kTile - 1) / kTile) + (p.t0 + t0) / kTile) * q.N * q.D +
                                p.d);
        const int64_t row = ((int64_t)p.b * q.T + p.t0 + t0 + s0) * q.D + p.d;
        out_at[0] = (char*)(out.gx + row), out_at[1] = (char*)(out.gdt + row), out_at[2] = (char*)(out.gz + row);
    };
    auto load_states = [&](int nb, int tiles, auto& bc, float (&m)[NS]) {      // of the tile `tiles` after Bt
#pragma unroll
        for (int k = 0; k < NS; ++k) {
            bc[0][k].load(Bt + tiles * kTile * q.b_time + at(nb, k));
            bc[1][k].load(Ct + tiles * kTile * q.c_time + at(nb, k));
            m[k] = *(const float*)(mark_at + (tiles * q.N + at(nb, k)) * mark_step);
        }
    };
    auto take_states = [&](int nb, auto& bc, const float (&m)[NS]) {
#pragma unroll
        for (int k = 0; k < NS; ++k) {
            const bool on = first(nb) + k < q.N;
            made.B[k] = on ? bc[0][k].f32() : 0.0f;
            made.C[k] = on ? bc[1][k].f32() : 0.0f;
            made.h0[k] = on ? m[k] : 0.0f;
        }
    };
    auto load = [&](auto whole, int left) {
        load_states(0, 0, raw.bc, mark);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const char* from = in_at[j];
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                raw.v[j][i].load((const E*)from);
                if (decltype(whole)::value || s0 + i + 1 < left) from += steps[j];   // the last one again past the end
            }
        }
    };
    auto back = [&] {
#pragma unroll
        for (int j = 0; j < 4; ++j) in_at[j] -= kTile * steps[j];
        Bt -= kTile * q.b_time, Ct -= kTile * q.c_time;
        mark_at -= q.N * mark_step;
    };
    auto ready = [&](int left) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            made.x[i] = raw.v[0][i].f32();
            made.delta[i] = step_length(q, raw.v[1][i].f32() + bias, made.slope[i]);
            made.g[i] = driven ? raw.v[3][i].f32() : 0.0f;
            const float gate = silu(raw.v[2][i].f32(), made.z_slope[i]);
            made.z_slope[i] *= made.g[i];
            made.g[i] = gated ? made.g[i] * gate : made.g[i];
        }
        // a channel past the group's last has no part in the sums over channels,
        // steps past the end are the identity
#pragma unroll
        for (int i = 0; i < STEPS; i += 2) {
            float v[2][3];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const bool on = p.live && s0 + i + j < left;
                v[j][0] = on ? made.delta[i + j] : 0.0f;
                v[j][1] = on ? made.delta[i + j] * made.x[i + j] : 0.0f;
                v[j][2] = on ? made.g[i + j] : 0.0f;
            }
            shD[(s0 + i) / 2][lane] = make_float4(v[0][0], v[0][1], v[1][0], v[1][1]);
            shG[(s0 + i) / 2][lane] = make_float2(v[0][2], v[1][2]);
        }
        take_states(0, raw.bc, mark);
    };
    auto put = [&](auto first_pass, int what, int i, float a, float b) {
        float2* to = &shP[what][w][i / 2][lane];
        *to = decltype(first_pass)::value ? make_float2(a, b) : make_float2(to->x + a, to->y + b);
    };
    auto walk = [&](auto whole, int t0, int cnt, int tiles) {
        constexpr bool kWhole = decltype(whole)::value;
        float4 D[kTile / 2];
        float2 G[kTile / 2];
#pragma unroll
        for (int i = 0; i < kTile / 2; ++i) D[i] = shD[i][lane], G[i] = shG[i][lane];
        auto delta = [&](int i) { return i % 2 ? D[i / 2].z : D[i / 2].x; };
        auto input = [&](int i) { return i % 2 ? D[i / 2].w : D[i / 2].y; };
        auto grad = [&](int i) { return i % 2 ? G[i / 2].y : G[i / 2].x; };
        auto pass = [&](auto first_pass, int nb, States& s) {
            float h[kTile][NS], a[kTile][NS], sum[kTile], P[kTile], Q[kTile], lam[kTile][NS], part[kTile];
            float gA_tile[NS] = {}, rate[NS], A[NS];          // long sums go in two levels
            const float(&B)[NS] = made.B, (&C)[NS] = made.C, (&h0)[NS] = made.h0;
            Bits<E> bc[2][NS];
            float m[NS];
            if (nb + 1 < NB) load_states(nb + 1, tiles, bc, m);
#pragma unroll
            for (int k = 0; k < NS; ++k) rate[k] = rate_of(s.A[k]), A[k] = slope_of(s.A[k]);
            each_step([&](auto step) {
                constexpr int i = decltype(step)::value;
#pragma unroll
                for (int k = 0; k < NS; ++k) {
                    a[i][k] = __builtin_amdgcn_exp2f(delta(i) * rate[k]);
                    h[i][k] = fmaf(a[i][k], i ? h[i ? i - 1 : 0][k] : h0[k], input(i) * of_step<i>(B[k]));
                }
                sum[i] = of_step<i>(C[0]) * h[i][0];
                if constexpr (i % 4 == 3) {
                    add_steps<i - 3>(sum + i - 3, C[1], h[i - 3][1], h[i - 2][1], h[i - 1][1], h[i][1]);
                    put(first_pass, 2, i - 3, sum[i - 3], sum[i - 2]);
                    put(first_pass, 2, i - 1, sum[i - 1], sum[i]);
                }
            });
            each_step_back([&](auto step) {
                constexpr int i = decltype(step)::value;
                float pb[NS], pc[NS];
                lam[i][0] = s.mu[0], lam[i][1] = s.mu[1];
                add_step<i>(lam[i][0], lam[i][1], C[0], C[1], grad(i));
#pragma unroll
                for (int k = 0; k < NS; ++k) {
                    pc[k] = grad(i) * h[i][k];
                    pb[k] = lam[i][k] * input(i);
                    s.mu[k] = a[i][k] * lam[i][k];
                    float f = s.mu[k] * (i ? h[i ? i - 1 : 0][k] : h0[k]);
                    if (!kWhole) f = i < cnt ? f : 0.0f;
                    P[i] = k ? fmaf(A[k], f, P[i]) : A[k] * f;
                    gA_tile[k] = fmaf(delta(i), f, gA_tile[k]);
                }
                Q[i] = of_step<i>(B[0]) * lam[i][0];
                part[i] = merge_states(pb[0], pb[1], pc[0], pc[1]);
                if constexpr (i % 4 == 0) {
                    add_steps<i>(Q + i, B[1], lam[i][1], lam[i + 1][1], lam[i + 2][1], lam[i + 3][1]);
#pragma unroll
                    for (int j = 0; j < 4; j += 2) {
                        put(first_pass, 0, i + j, P[i + j], P[i + j + 1]);
                        put(first_pass, 1, i + j, Q[i + j], Q[i + j + 1]);
                    }
                }
            });
#pragma unroll
            for (int k = 0; k < NS; ++k) s.gA[k] += gA_tile[k];
            // rows 0 .. 3 hold b and c of the first state, b and c of the second
            const float all = merge_steps(part, lane);
            const int row = lane >> 4, i = lane & 15, n = first(nb) + (row >> 1);
            if (i < cnt && n < q.N)
                (row & 1 ? out.partC : out.partB)[((int64_t)p.column * q.T + p.t0 + t0 + i) * q.N + n] = all;
            if (nb + 1 < NB) take_states(nb + 1, bc, m);
        };
        if (first(0) < q.N) pass(std::true_type(), 0, held);
#pragma unroll 1
        for (int nb = 1; nb < NB && first(nb) < q.N; ++nb) {
            States s = kept(nb);
            pass(std::false_type(), nb, s);
            keep(nb, s);
        }
    };
    auto write = [&](int cnt) {
        float P[STEPS], Q[STEPS], Y[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) P[i] = Q[i] = 0.0f, Y[i] = skip * made.x[i];
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int i = 0; i < STEPS; i += 2) {
                const float2 a = shP[0][j][(s0 + i) / 2][lane], b = shP[1][j][(s0 + i) / 2][lane];
                const float2 c = shP[2][j][(s0 + i) / 2][lane];
                P[i] += a.x, P[i + 1] += a.y, Q[i] += b.x, Q[i + 1] += b.y, Y[i] += c.x, Y[i + 1] += c.y;
            }
        float g_r[STEPS], skips = 0.0f, biases = 0.0f;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            g_r[i] = fmaf(made.x[i], Q[i], P[i]) * made.slope[i];
            const bool on = s0 + i < cnt;
            skips = on ? fmaf(made.g[i], made.x[i], skips) : skips;
            biases = on ? biases + g_r[i] : biases;
        }
        g_skip += skips, g_bias += biases;
        if (p.live)
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
                if (s0 + i < cnt) {
                    *(E*)(out_at[0] + i * out_step) = from_f32<E>(fmaf(made.delta[i], Q[i], skip * made.g[i]));
                    *(E*)(out_at[1] + i * out_step) = from_f32<E>(g_r[i]);
                    if (gated) *(E*)(out_at[2] + i * out_step) = from_f32<E>(Y[i] * made.z_slope[i]);
                }
#pragma unroll
        for (int j = 0; j < 3; ++j) out_at[j] -= kTile * out_step;
    };

    __syncthreads();
    if (first(0) >= q.N)                                      // the parts of a wave without states stay 0
#pragma unroll
        for (int j = 0; j < 3; ++j)
#pragma unroll
            for (int i = 0; i < kTile / 2; ++i) shP[j][w][i][lane] = make_float2(0.0f, 0.0f);

    int t0 = p.n / kTile * kTile;                             // after the last whole tile
    if (t0 < p.n) {
        find(t0, p.n - t0);
        load(std::false_type(), p.n - t0);
        ready(p.n - t0);
        __syncthreads();
        walk(std::false_type(), t0, p.n - t0, 0);
        __syncthreads();
        write(p.n - t0);
    }
    if (t0 > 0) {
        t0 -= kTile;
        find(t0, kTile);
        load(std::true_type(), kTile);
        ready(kTile);
        if (t0 > 0) back();
        load(std::true_type(), kTile);                        // (the first tile again where there is none before it)
        for (;;) {
            __syncthreads();
            walk(std::true_type(), t0, kTile, t0 > 0);
            __syncthreads();
            write(kTile);
            if (t0 == 0) break;
            t0 -= kTile;
            ready(kTile);
            if (t0 > 0) back();
            load(std::true_type(), kTile);
        }
    }
    if (p.live) {
        for (int t = p.t0 + p.n + w; t < p.t1; t += W) {
            const int64_t to = ((int64_t)p.b * q.T + t) * q.D + p.d;
            out.gx[to] = out.gdt[to] = from_f32<E>(0.0f);
            if (gated) out.gz[to] = from_f32<E>(0.0f);
        }
        const int64_t states = (int64_t)q.D * q.N;
#pragma unroll 1
        for (int nb = 0; nb < NB; ++nb) {
            const States s = nb ? kept(nb) : held;
#pragma unroll
            for (int k = 0; k < NS; ++k)
                if (first(nb) + k < q.N) {
                    const int64_t to = (int64_t)p.d * q.N + first(nb) + k;
                    out.partA[((int64_t)p.seg * q.B + p.b) * states + to] = s.gA[k];
                    if (out.g_first && p.seg == 0) out.g_first[p.b * states + to] = s.mu[k];
                }
        }
    }
    __syncthreads();
    shP[0][w][0][lane] = make_float2(g_skip, g_bias);
    __syncthreads();
    if (w == 0 && p.live) {
        float skips = 0.0f, biases = 0.0f;
        for (int j = 0; j < W; ++j) skips += shP[0][j][0][lane].x, biases += shP[0][j][0][lane].y;
        float* to = out.partS + ((int64_t)p.seg * q.B + p.b) * 2 * q.D + p.d;
        to[0] = skips;
        to[q.D] = biases;
    }
}

// Adds up the columns' parts of grad_B and grad_C, and the samples' parts of
// the parameters' gradients, in the order of columns, segments and samples: 8 x
// 2048 x 2048 x 16 16 us, 69 MB at 4.3 TB/s.
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
    // 64 of the sums to a workgroup at a time, a contiguous quarter of the rows to a
    // wave
    __shared__ float sh[4][kWave];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t rows = (int64_t)q.S * q.B, sums = states + 2 * (int64_t)q.D;
    for (int64_t at0 = (int64_t)(blockIdx.x - bc_blocks) * kWave; at0 < sums; at0 += (gridDim.x - bc_blocks) * kWave) {
        const int64_t at = at0 + lane;
        const float* from = at < states ? partA + at : partS + (at - states);
        const int64_t per = at < states ? states : 2 * (int64_t)q.D;
        float s = 0.0f;
        if (at < sums)
#pragma unroll 8
            for (int64_t i = rows * w / 4; i < rows * (w + 1) / 4; ++i) s += from[i * per];
        sh[w][lane] = s;
        __syncthreads();
        if (w == 0 && at < sums) {
            s = (sh[0][lane] + sh[1][lane]) + (sh[2][lane] + sh[3][lane]);
            const int64_t i = at - states;                    // skip's, then dt_bias'
            float* to = at < states ? gA : i < q.D ? g_skip : g_bias;
            if (to) to[at < states ? at : i < q.D ? i : i - q.D] = s;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// One step.  2^shift lanes share a channel, each holds four of its states.
// ---------------------------------------------------------------------------

// The second axis of the grid goes over streams, U at a time, whose loads are in
// flight together.  Bound by memory: 256 x 4096 x 16 states 28 us, 142 MB at 5.1
// TB/s; 400 x 3999 x 33 f32 199 us a call with two streams, 238 with one, 235
// with four.
template <typename E, int U>
__global__ __launch_bounds__(256) void k_select_step(Inputs in, const int32_t* __restrict__ slot,
                                                     float* __restrict__ state, int n_slots, Geometry q, int shift,
                                                     E* __restrict__ y)
{
    const int at = blockIdx.x * blockDim.x + threadIdx.x, d = at >> shift, n0 = (at & ((1 << shift) - 1)) * 4;
    const bool live = d < q.D, wide = n0 + 4 <= q.N;
    const int c = live ? d : q.D - 1, g = q.G > 1 ? c / q.Dg : 0, left = q.N - n0;
    const float bias = in.bias ? in.bias[c] : 0.0f, skip = in.skip ? in.skip[c] : 0.0f;
    // four of a channel's or group's values, those past N as 0
    auto load = [&](auto& v, const auto* from) {
        if (wide) {
            load_elems<std::remove_cv_t<std::remove_reference_t<decltype(*from)>>, 4>(from, v);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k] = 0;
                if (k < left) v[k] = from[k];
            }
        }
    };
    float rate[4];
    load(rate, in.A + (int64_t)c * q.N + n0);
#pragma unroll
    for (int k = 0; k < 4; ++k) rate[k] = rate_of(rate[k]);
    for (int b0 = blockIdx.y * U; b0 < q.B; b0 += gridDim.y * U) {
        float h[U][4], z[U];
        E xv[U], dt[U], Bt[U][4], Ct[U][4];
        int row[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int b = min(b0 + j, q.B - 1);
            row[j] = slot ? slot[b] : b;
            if (row[j] < 0 || row[j] >= n_slots || b0 + j >= q.B) row[j] = -1;
            xv[j] = ((const E*)in.x + b * q.x_batch)[c];
            dt[j] = ((const E*)in.dt + b * q.dt_batch)[c];
            z[j] = in.z ? to_f32(((const E*)in.z + b * q.z_batch)[c]) : 0.0f;
            load(Bt[j], (const E*)in.Bm + b * q.b_batch + g * q.N + n0);
            load(Ct[j], (const E*)in.C + b * q.c_batch + g * q.N + n0);
#pragma unroll
            for (int k = 0; k < 4; ++k) h[j][k] = 0.0f;
            if (row[j] >= 0) load(h[j], state + ((int64_t)row[j] * q.D + c) * q.N + n0);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            float slope, sum = 0.0f;
            const float x = to_f32(xv[j]), delta = step_length(q, to_f32(dt[j]) + bias, slope), u = delta * x;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                h[j][k] = fmaf(__builtin_amdgcn_exp2f(delta * rate[k]), h[j][k], u * to_f32(Bt[j][k]));
                sum = k < left ? fmaf(to_f32(Ct[j][k]), h[j][k], sum) : sum;
            }
            if (live && row[j] >= 0) {
                float* to = state + ((int64_t)row[j] * q.D + c) * q.N + n0;
                if (wide) {
                    store_elems<float, 4>(to, h[j]);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < left) to[k] = h[j][k];
                }
            }
            for (int o = 1 << shift >> 1; o; o >>= 1) sum += __shfl_xor(sum, o);
            if (live && n0 == 0 && b0 + j < q.B) {
                sum = fmaf(skip, x, sum);
                if (in.z) sum *= silu(z[j], slope);
                (y + (int64_t)(b0 + j) * q.D)[c] = from_f32<E>(row[j] >= 0 ? sum : 0.0f);
            }
        }
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

template <int V> struct Int { static constexpr int value = V; };

// Calls fn(states of a wave, waves) with types that carry them.  Four waves at
// least share out the steps of a tile, also where fewer hold states: 10 x 2091 x
// 3069 f16 with one state, training, 650 us (one wave: 1204).  Eight waves of one
// state instead of four of two: 30 x 2283 x 319 x 5 f16 174 -> 146 us; backward the
// other way, 9 x 1658 x 3230 x 5 631 with four waves, 748 with eight (waves_back).
template <typename Fn> void with_waves(int N, Fn&& fn)
{
    if (N <= 4) fn(Int<1>(), Int<4>());
    else if (N <= 8) fn(Int<1>(), Int<8>());
    else if (N <= 16) fn(Int<2>(), Int<8>());
    else if (N <= 32) fn(Int<4>(), Int<8>());
    else fn(Int<8>(), Int<8>());
}

int waves_of(int N)
{
    int waves = 0;
    with_waves(N, [&](auto, auto w) { waves = decltype(w)::value; });
    return waves;
}

// Segments of the time axis, by the rule above.
int segments_of(const lif_select_params& p, int columns, int waves)
{
    const int tiles = (p.T + kTile - 1) / kTile;
    if (columns > kSplitColumns) return 1;
    int S = columns > 0 ? kSplitWaves / (columns * waves) : 1;
    S = min(min(S, kMaxSegments), tiles / kSplitTiles);
    return S < kSplitLeast ? 1 : S;
}

int waves_back(int N) { return N <= 8 ? 4 : 8; }

Geometry geometry_of(const lif_select_params& p, int waves)
{
    Geometry q;
    q.B = p.B, q.T = p.T, q.D = p.D, q.N = p.N, q.G = p.G;
    q.Dg = p.D / p.G;
    q.cols = (q.Dg + kWave - 1) / kWave;
    q.columns = q.B * q.G * q.cols;
    const int tiles = (q.T + kTile - 1) / kTile, S = segments_of(p, q.columns, waves);
    const int per = tiles > 0 ? (tiles + S - 1) / S : 1;
    q.seg_len = per * kTile;
    q.S = tiles > 0 ? (tiles + per - 1) / per : 1;
    q.ordered = q.S == 1 && q.B > 1 && q.B <= kMaxOrder;
    q.flags = p.flags;
    q.x_batch = p.x_batch, q.x_time = p.x_time, q.dt_batch = p.dt_batch, q.dt_time = p.dt_time;
    q.z_batch = p.z_batch, q.z_time = p.z_time, q.b_batch = p.b_batch, q.b_time = p.b_time;
    q.c_batch = p.c_batch, q.c_time = p.c_time, q.g_batch = p.g_batch, q.g_time = p.g_time;
    return q;
}

size_t align16(size_t n) { return (n + 15) & ~(size_t)15; }

// Segments' sums and ends (none where there is one segment).
size_t sums_size(const Geometry& q) { return q.S > 1 ? align16(sizeof(float) * q.S * (size_t)q.B * q.D) : 0; }
size_t ends_size(const Geometry& q) { return q.S > 1 ? align16(sizeof(float) * q.S * (size_t)q.B * q.D * q.N) : 0; }

struct BackLayout {
    size_t partB, partC, partA, partS, sums, ends, total;
};

BackLayout back_layout(const lif_select_params& p)
{
    const Geometry q = geometry_of(p, waves_back(p.N));
    BackLayout l;
    const size_t bc = align16(sizeof(float) * q.B * q.G * q.cols * (size_t)q.T * q.N);
    l.partB = 0;
    l.partC = bc;
    l.partA = 2 * bc;
    l.partS = l.partA + align16(sizeof(float) * q.S * (size_t)q.B * q.D * q.N);
    l.sums = l.partS + align16(sizeof(float) * 2 * q.S * (size_t)q.B * q.D);
    l.ends = l.sums + sums_size(q);
    l.total = l.ends + ends_size(q);
    return l;
}

}  // namespace
}  // namespace lif

extern "C" size_t lif_selective_scan_workspace_size(const lif_select_params* p)
{
    using namespace lif;
    if (check_select(p) != LIF_OK) return 0;
    const Geometry q = geometry_of(*p, waves_of(p->N));
    return sums_size(q) + ends_size(q);
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
    const size_t need = lif_selective_scan_workspace_size(p);
    if (need > 0 && (!ws || (uintptr_t)ws % 16)) return LIF_ERR_ARG;
    if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    if (p->B == 0) return LIF_OK;
    const Geometry q = geometry_of(*p, waves_of(p->N));
    const Inputs in = {x, dt, Bm, C, z, nullptr, A, skip, dt_bias, length};
    float *sums = (float*)ws, *ends = (float*)((char*)ws + sums_size(q));
    with_dtype(p->dtype, [&](auto e) {
        using E = decltype(e);
        with_waves(q.N, [&](auto ns, auto waves) {
            constexpr int NS = decltype(ns)::value, W = decltype(waves)::value;
            if (q.S > 1)
                TIMED_LAUNCH("select_maps", (k_select_maps<E, NS, W, false>), dim3((unsigned)(q.columns * (q.S - 1))),
                             dim3(W * kWave), 0, (hipStream_t)stream, in, q, sums, ends);
            TIMED_LAUNCH("select_scan", (k_select_scan<E, NS, W>), dim3((unsigned)(q.columns * q.S)), dim3(W * kWave),
                         0, (hipStream_t)stream, in, q, h_first, sums, ends, (E*)y, h_last, marks);
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
    const Geometry q = geometry_of(*p, waves_back(p->N));
    const Inputs in = {x, dt, Bm, C, z, grad_y, A, skip, dt_bias, length};
    const int64_t bc = (int64_t)q.B * q.G * q.T * q.N;
    // the last launch's workgroups, for each of its two halves at most 2^22
    const int64_t bc_blocks = min((bc + 255) / 256, (int64_t)1 << 22);
    const int64_t blocks = bc_blocks + min(((int64_t)q.D * (q.N + 2) + kWave - 1) / kWave, (int64_t)1 << 22);
    with_dtype(p->dtype, [&](auto e) {
        using E = decltype(e);
        char* base = (char*)ws;
        const BackOut<E> out = {(E*)grad_x, (E*)grad_dt, (E*)grad_z, (float*)(base + l.partB),
                                (float*)(base + l.partC), (float*)(base + l.partA), (float*)(base + l.partS),
                                grad_h_first};
        float *sums = (float*)(base + l.sums), *ends = (float*)(base + l.ends);
        auto launch = [&](auto waves, auto nb) {
            constexpr int W = decltype(waves)::value, NB = decltype(nb)::value;
            TIMED_LAUNCH("select_back", (k_select_back<E, W, NB>), dim3((unsigned)(q.columns * q.S)),
                         dim3(W * kWave), 0, (hipStream_t)stream, in, q, marks, grad_last, sums, ends, out);
        };
        if (q.S > 1)
            with_waves(q.N, [&](auto ns, auto waves) {
                constexpr int NS = decltype(ns)::value, W = decltype(waves)::value;
                TIMED_LAUNCH("select_maps_back", (k_select_maps<E, NS, W, true>),
                             dim3((unsigned)(q.columns * (q.S - 1))), dim3(W * kWave), 0, (hipStream_t)stream, in, q,
                             sums, ends);
            });
        if (q.B > 0) {
            if (q.N <= 8) launch(Int<4>(), Int<1>());
            else if (q.N <= 16) launch(Int<8>(), Int<1>());
            else if (q.N <= 32) launch(Int<8>(), Int<2>());
            else launch(Int<8>(), Int<4>());
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
    const Geometry q = geometry_of(*p, 1);
    const Inputs in = {x, dt, Bm, C, z, nullptr, A, skip, dt_bias, nullptr};
    int shift = 0;                                            // 2^shift lanes to a channel
    while (4 << shift < q.N) ++shift;
    const int64_t lanes = (int64_t)q.D << shift;
    const unsigned threads = lanes >= 256 ? 256 : (unsigned)((lanes + kWave - 1) / kWave * kWave);
    // two streams at a time where that still fills the chip
    const unsigned blocks = (unsigned)((lanes + threads - 1) / threads);
    const bool pairs = (int64_t)blocks * q.B >= kStepPairs;
    const int rows = pairs ? (q.B + 1) / 2 : q.B;
    const dim3 grid(blocks, rows < 65535 ? rows : 65535);
    with_dtype(p->dtype, [&](auto e) {
        using E = decltype(e);
        if (pairs)
            TIMED_LAUNCH("select_step", (k_select_step<E, 2>), grid, dim3(threads), 0, (hipStream_t)stream, in, slot,
                         state, n_slots, q, shift, (E*)y);
        else
            TIMED_LAUNCH("select_step", (k_select_step<E, 1>), grid, dim3(threads), 0, (hipStream_t)stream, in, slot,
                         state, n_slots, q, shift, (E*)y);
    });
    return check_launch();
}
