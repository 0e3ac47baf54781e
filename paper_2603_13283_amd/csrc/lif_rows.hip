// lif_rows.hip -- probabilities read off rows of logits: log probabilities of
// given tokens with entropy and the likeliest alternatives
// (lif_token_logprobs), and distillation from a teacher's likeliest classes
// (lif_distill_top), each with its gradient.
//
// With m the row's largest logit, c = log2(e) / temperature and o = m c
// rounded, every term is e_j = 2^{z_j} with z_j = x_j c - o, one FMA;
// S = sum e_j and U = sum e_j z_j give p_j = e_j / S, the entropy
// log S - log(2) U / S, and, with the rounding error of o put back, lse.
//
// Rows of up to kNarrow logits: a workgroup stages many rows in LDS with
// contiguous loads, and a few lanes work on each (k_narrow_*).  Longer rows:
// a workgroup holds a row in registers, so that the logits are read once for
// the maximum, the sums, the alternatives and the gradient (k_wide_*).  Where
// there are few rows, or a row does not fit, the row is cut into segments: a
// first launch leaves each segment's statistics and alternatives, a second
// one joins them and writes the results (and the gradient, from a second read).
#include "lif_host.hpp"
#include "lif_types.hpp"

#include <type_traits>

namespace lif {
namespace {

constexpr float kLn2 = 0.693147180559945309f;
constexpr float kNegInf = -INFINITY;
// Longest row of the narrow kernels.  50000 x 256 bf16, narrow and wide, us: 8
// alternatives 40 45, gradient 31 33, distillation 42 57 (x 160: 34 48, 23 33, 35
// 58); 30000 x 320: 36 30, 30 22, 39 38 (x 257, an odd row: 29 37, 22 29, 30 43).
constexpr int kNarrow = 256;
constexpr int kNarrowThreads = 128;
constexpr int kMaxV = 1 << 24;
constexpr int kCand = 512;              // candidates of a top-k selection held in LDS

struct RowArgs {
    int R, V, k;
    int64_t stride, grad_stride;
    float c, c_pow2, inv_t;             // log2(e) / temperature, a power of two from there on, 1 / temperature
    double inv_td;
    bool tail;
    int nseg, seg;                      // segments of a row and their length
};

// m c rounded, wherever it is used: contracted into the difference of two
// offsets it would not be the offset that the terms were taken by.
__device__ __forceinline__ float rounded_product(float m, float c)
{
#pragma clang fp contract(off)
    return m * c;
}

// The exponents of a row: z = x c - o, for the largest logit m.  The rounding
// of o multiplies all terms by the same factor, below 2^64 while |m| c < 2^30.
// From there on (rows masked by the type's lowest value, say) logits that
// differ lie at least 64 / c apart, so that the largest ones alone count: any
// power of two from c on makes the products exact, e = 1 for those and below
// 2^-64 for others, and 2^-60 one that does not overflow from |m| = 2^100 on.
struct Exponent {
    float m, c, o;                      // m is 0 where nothing is above -infinity
    bool plain, none;                   // c is the row's; nothing is above -infinity
    __device__ __forceinline__ Exponent(float largest, const RowArgs& a)
    {
        none = largest == kNegInf;
        m = none ? 0.0f : largest;
        plain = fabsf(m * a.c) < 0x1p30f;
        c = plain ? a.c : fabsf(m) < 0x1p100f ? a.c_pow2 : 0x1p-60f;
        o = rounded_product(m, c);
    }
    __device__ __forceinline__ float z(float x) const { return fmaf(x, c, -o); }
    // The exponent of the factor that makes sums of a part's terms, by the
    // part's own exponents, sums by these.  A part without anything above
    // -infinity has sums of 0 (or a NaN).
    __device__ __forceinline__ float from(const Exponent& part) const
    {
        if (part.none || part.m == m) return 0.0f;
        return part.plain && plain ? part.o - o : -200.0f;
    }
};
__device__ __forceinline__ float pow2(float z) { return __builtin_amdgcn_exp2f(z); }
// z where it is multiplied by e: -infinity (e = 0) must not give a NaN.
__device__ __forceinline__ float z_finite(float z) { return fmaxf(z, -200.0f); }

// A row's result from its exponents and sums.
struct RowStat {
    float m, s;
    float lz, ls;                       // log S as summed, and with the rounding of o put back
    float H;                            // entropy
    bool empty;                         // nothing above -infinity
};
__device__ __forceinline__ RowStat row_stat(const Exponent& x, float s, float u)
{
    RowStat r;
    r.m = x.m;
    r.s = s;
    r.empty = s == 0.0f;
    r.lz = r.empty ? kNegInf : logf(s);
    r.ls = r.lz - kLn2 * fmaf(x.m, x.c, -x.o);
    r.H = r.empty ? 0.0f : r.lz - kLn2 * (u / s);
    return r;
}
__device__ __forceinline__ float row_logp(const RowStat& r, const RowArgs& a, float x)
{
    return r.empty ? kNegInf : (x - r.m) * a.inv_t - r.ls;
}
__device__ __forceinline__ float row_lse(const RowStat& r, const RowArgs& a)
{
    return r.empty ? kNegInf : (float)((double)r.m * a.inv_td + (double)r.ls);
}

// Orders float32 values as unsigned integers: -0 and +0 are equal, a NaN
// ranks below -infinity, 0 is left for "none".
__device__ __forceinline__ uint32_t order_key(float v)
{
    if (v != v) return 1;
    const uint32_t u = __float_as_uint(v + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k)
{
    if (k == 1) return NAN;
    return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}
// The same order as signed integers, with a value below all for an element
// that is out.
constexpr int kTaken = INT32_MIN;
__device__ __forceinline__ int signed_key(float v) { return (int)(order_key(v) ^ 0x80000000u); }
__device__ __forceinline__ float signed_value(int k) { return key_value((uint32_t)k ^ 0x80000000u); }
// Larger logits first, then smaller indices.
using Cand = unsigned long long;
__device__ __forceinline__ Cand make_cand(float v, int j) { return ((Cand)order_key(v) << 32) | (0xffffffffu - (uint32_t)j); }
__device__ __forceinline__ int cand_index(Cand c) { return (int)(0xffffffffu - (uint32_t)c); }
__device__ __forceinline__ float cand_value(Cand c) { return key_value((uint32_t)(c >> 32)); }

// ---------------------------------------------------------------------------
// Sums and maxima over lanes: within 16 lanes by DPP (pairs, quads, mirrored
// halves), over the wave's four rows of 16 by lane reads.  The result is the
// same in all lanes, and the order of a sum is fixed.
// ---------------------------------------------------------------------------
template <int Ctrl> __device__ __forceinline__ float dpp(float v)
{
    const int i = __float_as_int(v);
    return __int_as_float(__builtin_amdgcn_update_dpp(i, i, Ctrl, 0xf, 0xf, false));
}
template <int Ctrl> __device__ __forceinline__ int dpp(int v)
{
    return __builtin_amdgcn_update_dpp(v, v, Ctrl, 0xf, 0xf, false);
}
template <int Ctrl> __device__ __forceinline__ double dpp(double v)
{
    return __hiloint2double(dpp<Ctrl>(__double2hiint(v)), dpp<Ctrl>(__double2loint(v)));
}
// Combines with the lanes of a group of L <= 16 (aligned) lanes.
template <int L, typename V, typename Op> __device__ __forceinline__ V over_lanes(V v, Op op)
{
    if constexpr (L >= 2) v = op(v, dpp<0xb1>(v));          // quad_perm 1,0,3,2
    if constexpr (L >= 4) v = op(v, dpp<0x4e>(v));          // quad_perm 2,3,0,1
    if constexpr (L >= 8) v = op(v, dpp<0x141>(v));         // mirrored in 8
    if constexpr (L >= 16) v = op(v, dpp<0x140>(v));        // mirrored in 16
    return v;
}
struct Add { template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; } };
struct Max { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct Min { __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); } };

template <typename Op> __device__ __forceinline__ float over_wave(float v, Op op)
{
    v = over_lanes<16>(v, op);
    const int i = __float_as_int(v);
    const float a = __int_as_float(__builtin_amdgcn_readlane(i, 0)), b = __int_as_float(__builtin_amdgcn_readlane(i, 16));
    const float c = __int_as_float(__builtin_amdgcn_readlane(i, 32)), d = __int_as_float(__builtin_amdgcn_readlane(i, 48));
    return op(op(a, b), op(c, d));
}
__device__ __forceinline__ double sum_over_wave(double v)
{
    v = over_lanes<16>(v, Add());
    auto row = [&](int lane) {
        return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane),
                                __builtin_amdgcn_readlane(__double2loint(v), lane));
    };
    return (row(0) + row(16)) + (row(32) + row(48));
}

// ---------------------------------------------------------------------------
// Narrow rows.  A workgroup takes kNarrowThreads / L rows, L lanes a row; lane
// l of a row holds its elements j = l + L i.  The rows pass through LDS, with
// a row length of an odd multiple of L words, so that the lanes of a wave read
// different banks.  Bound by instructions (vector units busy for two thirds of
// the time; 95 a logit with 5 alternatives, 140 in distillation, most of them
// for the alternatives, the list and the staging): 128000 x 20 f32 with 5
// alternatives 12 us, 17 MB, distillation 18 us, 27 MB; with a wave a row it
// would be 128000 waves of one element a lane.
// ---------------------------------------------------------------------------
constexpr int kNarrowPer = 32;          // at most this many elements a lane: one bit each in a mask

__host__ __device__ __forceinline__ int narrow_pitch(int V, int L) { return ((V + L - 1) / L | 1) * L; }

// Calls fn(row, element) for the elements of `rows` rows: thread by thread
// along the rows, so that several short rows lie side by side in a wave.
template <typename Fn> __device__ __forceinline__ void each_staged(int rows, int V, Fn&& fn)
{
    const int dr = kNarrowThreads / V, dj = kNarrowThreads - dr * V;
    int r = (int)threadIdx.x / V, j = (int)threadIdx.x - r * V;
    while (r < rows) {
        fn(r, j);
        r += dr;
        j += dj;
        if (j >= V) j -= V, ++r;
    }
}
template <typename E>
__device__ __forceinline__ void stage_rows(const E* __restrict__ in, int64_t stride, int rows, int V, int pitch,
                                           float* sh)
{
    each_staged(rows, V, [&](int r, int j) { sh[r * pitch + j] = to_f32(in[r * stride + j]); });
}
template <typename E>
__device__ __forceinline__ void unstage_rows(E* __restrict__ out, int64_t stride, int rows, int V, int pitch,
                                             const float* sh)
{
    each_staged(rows, V, [&](int r, int j) { out[r * stride + j] = from_f32<E>(sh[r * pitch + j]); });
}

template <typename E, int L>
__global__ __launch_bounds__(kNarrowThreads) void k_narrow_logprobs(
    const E* __restrict__ logits, const int32_t* __restrict__ token, RowArgs a, float* __restrict__ logp,
    float* __restrict__ entropy, float* __restrict__ lse, float* __restrict__ top_logp, int32_t* __restrict__ top_idx,
    const float* __restrict__ g_logp, const float* __restrict__ g_ent, E* __restrict__ grad)
{
    extern __shared__ float sh[];
    constexpr int per_group = kNarrowThreads / L;
    const int64_t row0 = (int64_t)blockIdx.x * per_group;
    const int rows = (int)min((int64_t)per_group, a.R - row0);
    const int pitch = narrow_pitch(a.V, L);
    stage_rows(logits + row0 * a.stride, a.stride, rows, a.V, pitch, sh);
    __syncthreads();
    const int rl = threadIdx.x / L, l = threadIdx.x % L;
    const int64_t r = row0 + rl;
    float* x = sh + rl * pitch + l;
    const int n = rl < rows ? (a.V - l + L - 1) / L : 0;       // this lane's elements x[L i]
    float m = kNegInf, s = 0.0f, u = 0.0f;
#pragma unroll 4
    for (int i = 0; i < n; ++i) m = fmaxf(m, x[L * i]);
    const Exponent ex(over_lanes<L>(m, Max()), a);
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const float z = ex.z(x[L * i]), e = pow2(z);
        s += e;
        u = fmaf(e, z_finite(z), u);
    }
    s = over_lanes<L>(s, Add());
    u = over_lanes<L>(u, Add());
    const RowStat st = row_stat(ex, s, u);
    int tok = -1;
    bool there = false;
    if (rl < rows) {
        tok = token ? token[r] : -1;
        there = tok >= 0 && tok < a.V;
        if (l == 0) {
            if (logp) logp[r] = there ? row_logp(st, a, sh[rl * pitch + tok]) : 0.0f;
            if (entropy) entropy[r] = st.H;
            if (lse) lse[r] = row_lse(st, a);
        }
    }
    if (a.k > 0) {                              // the elements become their keys' bits
        for (int i = 0; i < n; ++i) x[L * i] = __int_as_float(signed_key(x[L * i]));
        for (int q = 0; q < a.k; ++q) {
            int best = kTaken, at = 0;          // equal ones by index
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
                const int w = __float_as_int(x[L * i]);
                if (w > best) best = w, at = i;
            }
            int j = l + L * at;
            auto better = [&](int w, int o) {
                if (w > best || (w == best && o < j)) best = w, j = o;
            };
            if constexpr (L >= 2) better(dpp<0xb1>(best), dpp<0xb1>(j));
            if constexpr (L >= 4) better(dpp<0x4e>(best), dpp<0x4e>(j));
            if constexpr (L >= 8) better(dpp<0x141>(best), dpp<0x141>(j));
            if constexpr (L >= 16) better(dpp<0x140>(best), dpp<0x140>(j));
            if (rl < rows) {
                if (j % L == l) x[j - l] = __int_as_float(kTaken);
                if (l == 0) {
                    top_idx[r * a.k + q] = j;
                    top_logp[r * a.k + q] = row_logp(st, a, signed_value(best));
                }
            }
        }
        if (grad) {                             // the elements again
            __syncthreads();
            stage_rows(logits + row0 * a.stride, a.stride, rows, a.V, pitch, sh);
            __syncthreads();
        }
    }
    if (!grad) return;
    const float g = there && g_logp ? g_logp[r] : 0.0f, ge = rl < rows && g_ent ? g_ent[r] : 0.0f;
    const float inv_s = st.empty ? 0.0f : 1.0f / st.s;
    for (int i = 0; i < n; ++i) {
        const float z = ex.z(x[L * i]), p = pow2(z) * inv_s;
        const float lp = st.empty ? 0.0f : fmaf(kLn2, z_finite(z), -st.lz);
        float v = -p * fmaf(ge, lp + st.H, g);
        if (there && l + L * i == tok && !st.empty) v += g;
        x[L * i] = v * a.inv_t;
    }
    __syncthreads();
    unstage_rows(grad + row0 * a.grad_stride, a.grad_stride, rows, a.V, pitch, sh);
}

// The teacher's side of a row: sums over its used entries.  A list that is
// made to sum to 1 is taken relative to its largest entry, so that unlikely
// classes (a logp below -104 is 0 in float32) have a mass to divide by.  With
// a tail q = e^logp; its sum is of float64 terms, since 1 - sum q is small for
// a sure teacher.
struct Teacher {
    double sq;                          // sum of q as kept
    bool none;                          // no mass
    double q_rest, scale;               // the tail's share; what q is multiplied by
};
// What is taken off the list's logps, of which the largest is m.
__device__ __forceinline__ float list_shift(float m, bool tail) { return tail || m == kNegInf ? 0.0f : m; }
__device__ __forceinline__ Teacher teacher_of(double sq, float m, bool tail, bool all_listed)
{
    Teacher t;
    t.sq = sq;
    t.none = m == kNegInf && sq == 0.0;             // a NaN is kept
    t.q_rest = tail && 1.0 - sq >= LIF_DISTILL_TAIL_MIN && !all_listed ? 1.0 - sq : 0.0;
    t.scale = tail || t.none ? 1.0 : 1.0 / sq;
    return t;
}
// What is added to a logp for log q.
__device__ __forceinline__ double log_scale(const Teacher& t, float m, bool tail)
{
    return tail ? 0.0 : -(double)list_shift(m, tail) - (double)logf((float)t.sq);
}
constexpr float kLogTiny = -745.13f;    // e to this is float64's smallest number
// One entry's share q (log q - log p) of the loss; lp the student's log p.
__device__ __forceinline__ double entry_loss(double q, double log_q, double lp)
{
    return q > 0.0 ? q * (log_q - lp) : q != q ? q : 0.0;
}
// The classes that are not listed.  Their terms are taken by their own largest
// logit, not by the row's: next to a list that the student is sure of they
// would all be 0 in float32 (from a distance of 87 temperatures on), where
// their log probability and their shares of it are ordinary numbers.
struct Rest {
    Exponent own;
    float s, f;                         // sum of the terms; s f is a part of the row's S
    __device__ __forceinline__ Rest(const Exponent& own_, const Exponent& row, float sum)
        : own(own_), s(sum), f(pow2(row.from(own_)))
    {
    }
};
__device__ __forceinline__ double tail_loss(const Teacher& t, const Rest& rest, const RowStat& st, const RowArgs& a)
{
    if (!(t.q_rest > 0.0)) return 0.0;
    const RowStat r = row_stat(rest.own, rest.s, 0.0f);
    const double lp = r.empty ? (double)kNegInf
                              : ((double)r.m - (double)st.m) * a.inv_td + ((double)r.ls - (double)st.ls);
    return t.q_rest * ((double)logf((float)t.q_rest) - lp);
}
// dloss/dz_j = e_j c_top - q_j for a listed class, e_j c_rest for another, by
// the exponents of its kind.
__device__ __forceinline__ void grad_factors(const Teacher& t, const RowStat& st, const Rest& rest, float& c_top,
                                             float& c_rest)
{
    const double mass = t.scale == 1.0 && !t.none ? t.sq + t.q_rest : 1.0;
    c_top = t.none || st.empty ? 0.0f : (float)mass / st.s;
    c_rest = c_top * rest.f;
    // mass f / S - q_rest / s: the difference, which may be small, in float64
    if (!t.none && !st.empty && t.q_rest > 0.0 && rest.s > 0.0f)
        c_rest = (float)(mass * (double)rest.f * (double)rest.s - t.q_rest * (double)st.s) / st.s / rest.s;
}

template <typename E, int L>
__global__ __launch_bounds__(kNarrowThreads) void k_narrow_distill(const E* __restrict__ logits,
                                                                   const float* __restrict__ t_logp,
                                                                   const int32_t* __restrict__ t_idx, RowArgs a,
                                                                   const float* __restrict__ weight,
                                                                   float* __restrict__ loss, E* __restrict__ grad)
{
    extern __shared__ float sh[];
    constexpr int per_group = kNarrowThreads / L;
    const int64_t row0 = (int64_t)blockIdx.x * per_group;
    const int rows = (int)min((int64_t)per_group, a.R - row0);
    const int pitch = narrow_pitch(a.V, L);
    stage_rows(logits + row0 * a.stride, a.stride, rows, a.V, pitch, sh);
    __syncthreads();
    const int rl = threadIdx.x / L, l = threadIdx.x % L;
    const int64_t r = row0 + rl;
    float* row = sh + rl * pitch;
    float* x = row + l;
    const int n = rl < rows ? (a.V - l + L - 1) / L : 0;
    const int k = rl < rows ? a.k : 0;
    const int32_t* idx = t_idx + r * a.k;
    const float* lt = t_logp + r * a.k;
    uint32_t listed = 0;                        // this lane's elements that the teacher lists
#pragma unroll 4
    for (int i = 0; i < k; ++i) {
        const int j = idx[i];
        if (j >= 0 && j < a.V && j % L == l) listed |= 1u << (j / L);
    }
    float* q = sh + per_group * pitch + rl * a.k;               // of every entry
    float m_list = kNegInf;
    if (!a.tail) {
        for (int i = l; i < k; i += L)
            if (idx[i] >= 0 && idx[i] < a.V) m_list = fmaxf(m_list, lt[i]);
        m_list = over_lanes<L>(m_list, Max());
    }
    const float shift = list_shift(m_list, a.tail);
    double sq = 0.0;
    for (int i = l; i < k; i += L) {
        const bool used = idx[i] >= 0 && idx[i] < a.V;
        const double e = used ? exp((double)lt[i] - (double)shift) : 0.0;
        if (used) m_list = fmaxf(m_list, lt[i]);
        q[i] = (float)e;
        sq += e;
    }
    m_list = over_lanes<L>(m_list, Max());
    sq = over_lanes<L>(sq, Add());
    float m = kNegInf, m_rest = kNegInf, s_top = 0.0f, s_rest = 0.0f;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const float v = x[L * i];
        m = fmaxf(m, v);
        m_rest = fmaxf(m_rest, listed >> i & 1 ? kNegInf : v);
    }
    const Exponent ex(over_lanes<L>(m, Max()), a), er(over_lanes<L>(m_rest, Max()), a);
    auto term = [&](float v, bool top) { return pow2(fmaf(v, top ? ex.c : er.c, top ? -ex.o : -er.o)); };
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const bool top = listed >> i & 1;
        const float e = term(x[L * i], top);
        if (top) s_top += e;
        else s_rest += e;
    }
    s_top = over_lanes<L>(s_top, Add());
    const int n_top = over_lanes<L>((int)__popc(listed), [](int p, int o) { return p + o; });
    const Rest rest(er, ex, over_lanes<L>(s_rest, Add()));
    const RowStat st = row_stat(ex, fmaf(rest.s, rest.f, s_top), 0.0f);
    const Teacher t = teacher_of(sq, m_list, a.tail, n_top == a.V);
    if (loss) {
        const double add = log_scale(t, m_list, a.tail);
        double v = 0.0;
        for (int i = l; i < k; i += L) {
            const int j = idx[i];
            if (j < 0 || j >= a.V) continue;
            const double lp = st.empty ? (double)kNegInf
                                       : ((double)row[j] - (double)st.m) * a.inv_td - (double)st.ls;
            v += entry_loss((double)q[i] * t.scale, (double)lt[i] + add, lp);
            // where log p is -infinity or a NaN it matters whether q is 0 or only its float32
            if (q[i] == 0.0f && !(lp > (double)kNegInf) && lt[i] - shift > kLogTiny) v -= lp;
        }
        v = over_lanes<L>(v, Add());
        if (l == 0 && rl < rows) loss[r] = t.none ? 0.0f : (float)(v + tail_loss(t, rest, st, a));
    }
    if (!grad) return;
    float c_top, c_rest;
    grad_factors(t, st, rest, c_top, c_rest);
    const float w = rl < rows ? (weight ? weight[r] : 1.0f) * a.inv_t : 0.0f;
    const bool dead = t.none || st.empty;
    c_top *= w;
    c_rest *= w;
    for (int i = 0; i < n; ++i) {
        const bool top = listed >> i & 1;
        x[L * i] = dead ? 0.0f : term(x[L * i], top) * (top ? c_top : c_rest);
    }
    __syncthreads();
    // the lanes of a row hold its elements apart, so every element is changed by one lane
    const float scale = (float)t.scale;
    for (int i = 0; i < k && !dead; ++i) {
        const int j = idx[i];
        if (j >= 0 && j < a.V && j % L == l) row[j] -= q[i] * scale * w;
    }
    __syncthreads();
    unstage_rows(grad + row0 * a.grad_stride, a.grad_stride, rows, a.V, pitch, sh);
}

// ---------------------------------------------------------------------------
// Wide rows, read once.  At 2 bytes a logit the vector units take nearly as
// long as the memory (15 instructions a logit with 64 alternatives, 19 with the
// gradient, 22 in distillation, against about 15 that fit the time of its load
// and as many that of its store), so two workgroups share a CU and one computes
// while the other loads: rows of 65536 16-bit logits take 64 of 128 registers.
// 4096 x 50048 bf16 with 5 alternatives 102 us, 410 MB at 4.0 TB/s; gradient of
// 4096 x 32768 f32 200 us, 1.07 GB at 5.4 TB/s; distillation 4096 x 50048 bf16
// with 64 entries 170 us, 820 MB at 4.8 TB/s.
//
// A workgroup of NT threads holds a segment in registers: NV
// vectors of 16 bytes a thread, vector i of thread t at element
// (i NT + t) VEC, at whatever address that is: the order of a row's sums does
// not depend on where the row lies.  What a vector holds past the segment
// counts as -infinity.
// ---------------------------------------------------------------------------
template <typename E> constexpr int kVec = 16 / (int)sizeof(E);

// Four words at an address that is aligned to one element.
template <typename E> struct __attribute__((packed, aligned(sizeof(E)))) Words {
    uint32_t w[4];
};

// Element e of four words.
template <typename E> __device__ __forceinline__ float unpack(const uint32_t (&w)[4], int e)
{
    if constexpr (sizeof(E) == 4) return __uint_as_float(w[e]);
    const uint32_t u = w[e >> 1];
    if constexpr (std::is_same<E, bf16>::value) return __uint_as_float(e & 1 ? u & 0xffff0000u : u << 16);
    else return (float)__builtin_bit_cast(f16, (uint16_t)(e & 1 ? u >> 16 : u));
}
template <typename E> __device__ __forceinline__ uint32_t pack_pair(float a, float b)
{
    const uint32_t lo = __builtin_bit_cast(uint16_t, from_f32<E>(a)), hi = __builtin_bit_cast(uint16_t, from_f32<E>(b));
    return lo | hi << 16;
}

template <typename E, int NT, int NV> struct Held {
    static constexpr int VEC = kVec<E>;
    uint32_t v[NV][4];
    int len;                            // elements of the segment

    __device__ __forceinline__ int first(int i) const { return (i * NT + (int)threadIdx.x) * VEC; }
    // whether any thread of the workgroup holds elements in vector i
    __device__ __forceinline__ bool any(int i) const { return i * NT * VEC < len; }
    __device__ __forceinline__ float get(int i, int e) const { return unpack<E>(v[i], e); }

    // The vector at element j, element by element.
    __device__ __forceinline__ void load_each(uint32_t (&w)[4], const E* __restrict__ x, int j) const
    {
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = j + e < len ? to_f32(x[j + e]) : kNegInf;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if constexpr (sizeof(E) == 4) w[k] = __float_as_uint(f[k]);
            else w[k] = pack_pair<E>(f[2 * k], f[2 * k + 1]);
    }
    // Whole vectors are loaded wide.  The one that the segment's end cuts is read
    // by its thread apart and put in its place afterwards: a branch for it at
    // every vector makes the code outgrow the instruction cache (4096 x 50048
    // bf16 distillation 168 -> 212 us).
    //
    // Rows of 16-bit elements off the 4-byte grid: wide loads there take a
    // quarter longer (4096 x 50001 bf16 111 us, 91 for 50002).  So a thread
    // loads from one element before its vector, on the grid, gets the last
    // element from the next lane's first word, and shifts; every thread ends
    // up with the elements that it has in any other row.  The first vector is
    // then read like the last.
    __device__ __forceinline__ void load(const E* __restrict__ x, int n)
    {
        len = __builtin_amdgcn_readfirstlane(n);               // the same in all threads
        const bool odd = sizeof(E) == 2 && ((uintptr_t)x & 2);
        const int cut = len / VEC;                             // the vector that the end cuts, if any
        const bool mine = len % VEC && (int)threadIdx.x == cut % NT;
        uint32_t edge[4], head[4];
        if (!odd) {
#pragma unroll
            for (int i = 0; i < NV; ++i) load_wide(i, x, 0);
            if (mine) load_each(edge, x, cut * VEC);
        } else {
            const bool last = (threadIdx.x & 63) == 63;
            uint32_t end[NV];                                  // the last element, where the next lane has it not
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                load_wide(i, x, 1);
                end[i] = 0;
                const int j = first(i);
                if (j + VEC <= len && (last || j + 2 * VEC > len))
                    end[i] = *reinterpret_cast<const uint16_t*>(x + j + VEC - 1);
            }
            if (mine) load_each(edge, x, cut * VEC);
            if (threadIdx.x == 0) load_each(head, x, 0);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int j = first(i);
                const uint32_t next = (uint32_t)dpp<0x130>((int)v[i][0]);      // of the next lane
                const uint32_t tail = last || j + 2 * VEC > len ? end[i] : next;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t u = __builtin_amdgcn_alignbyte(k < 3 ? v[i][k + 1] : tail, v[i][k], 2);
                    v[i][k] = j + VEC <= len ? u : none();
                }
            }
            if (threadIdx.x == 0)
#pragma unroll
                for (int k = 0; k < 4; ++k) v[0][k] = head[k];
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i == cut / NT && mine)
#pragma unroll
                for (int k = 0; k < 4; ++k) v[i][k] = edge[k];
    }
    // Vector i from `back` elements before its place, if the segment has all of
    // its elements (and, with back, it is not the first).
    __device__ __forceinline__ void load_wide(int i, const E* __restrict__ x, int back)
    {
        const int j = first(i);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[i][k] = none();
        if (j + VEC <= len && j >= back) {
            const Words<E> q = *reinterpret_cast<const Words<E>*>(x + j - back);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i][k] = q.w[k];
        }
    }
    static __device__ __forceinline__ uint32_t none()
    {
        if constexpr (sizeof(E) == 4) return __float_as_uint(kNegInf);
        else return pack_pair<E>(kNegInf, kNegInf);
    }
    // From here on the elements and the length count as new values to the
    // compiler, which otherwise keeps all elements unpacked, and a mask for
    // every vector, in registers from one pass to the next.
    __device__ __forceinline__ void fresh()
    {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(v[i][k]));
        asm volatile("" : "+s"(len));
    }
    // vm: the largest element of each vector; returns the thread's largest.
    __device__ __forceinline__ float maxima(float (&vm)[NV])
    {
        float m = kNegInf;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            vm[i] = kNegInf;
            if (!any(i)) continue;
#pragma unroll
            for (int e = 0; e < VEC; ++e) vm[i] = fmaxf(vm[i], get(i, e));
            m = fmaxf(m, vm[i]);
        }
        fresh();
        return m;
    }
    // Calls fn(element) for each element.
    template <typename Fn> __device__ __forceinline__ void each(Fn&& fn)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!any(i)) continue;
#pragma unroll
            for (int e = 0; e < VEC; ++e) fn(get(i, e));
        }
        fresh();
    }
    // Takes out the elements of vector i that `bits` names.
    __device__ __forceinline__ void drop(int i, uint32_t bits)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if constexpr (sizeof(E) == 4) {
                if (bits >> k & 1) v[i][k] = __float_as_uint(kNegInf);
            } else {
                if (bits >> (2 * k) & 1) v[i][k] = (v[i][k] & 0xffff0000u) | (none() & 0xffffu);
                if (bits >> (2 * k + 1) & 1) v[i][k] = (v[i][k] & 0xffffu) | (none() & 0xffff0000u);
            }
    }
    // Stores fn(element) for each element of the segment, which is x's.
    template <typename Fn>
    __device__ __forceinline__ void store(E* __restrict__ out, const E* __restrict__ x, Fn&& fn)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = first(i);
            if (!any(i) || j + VEC > len) continue;
            float f[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = fn(get(i, e));
            Words<E> q;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if constexpr (sizeof(E) == 4) q.w[k] = __float_as_uint(f[k]);
                else q.w[k] = pack_pair<E>(f[2 * k], f[2 * k + 1]);
            *reinterpret_cast<Words<E>*>(out + j) = q;
        }
        const int j = len / VEC * VEC + (int)threadIdx.x;      // the vector that the end cuts
        if (j < len) out[j] = from_f32<E>(fn(to_f32(x[j])));
    }
};

constexpr int kGroups = 256;            // groups whose maxima bound the k-th largest logit

template <int NT> struct WideLds {
    float part[3][NT / 64];
    float group[kGroups];
    float bound;                        // at least k logits reach it, or -infinity
    int count;
    Cand cand[kCand];
};

// Maximum over the workgroup.
template <int NT, typename Op> __device__ __forceinline__ float join_parts(const float* part, Op op)
{
    float v = part[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) v = op(v, part[i]);
    return v;
}

// A value that at least k logits of the segment reach, from the maxima of
// disjoint groups of threads: the k-th largest of them, nearly (ten halvings
// of the interval between the smallest and the largest).  -infinity where
// fewer than k groups have anything above it.  Run by one wave.
template <int NG> __device__ __forceinline__ float bound_of_kth(const float* group, int k, int lane)
{
    constexpr int N = NG / 64;
    float v[N], lo = INFINITY, hi = kNegInf;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = group[i * 64 + lane];
        hi = fmaxf(hi, v[i]);
        lo = fminf(lo, v[i] > kNegInf ? v[i] : INFINITY);
    }
    hi = over_wave(hi, Max());
    lo = over_wave(lo, Min());
    auto reach = [&](float b) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__ballot(v[i] >= b));
        return n;
    };
    if (!(lo < INFINITY) || reach(lo) < k) return kNegInf;
    for (int i = 0; i < 10; ++i) {
        const float mid = 0.5f * lo + 0.5f * hi;
        if (reach(mid) >= k) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The elements j .. j + VEC - 1 of a segment for which fn(element) holds, one
// bit each.  A selection reads the few vectors that it needs again (from the
// L2): indexing the held ones by a loop's variable would cost more.
template <typename E, typename Fn>
__device__ __forceinline__ uint32_t which(const E* __restrict__ x, int j, int len, Fn&& fn)
{
    constexpr int VEC = kVec<E>;
    uint32_t hit = 0;
    if (j + VEC <= len) {
        const Words<E> q = *reinterpret_cast<const Words<E>*>(x + j);
        uint32_t v[4] = {q.w[0], q.w[1], q.w[2], q.w[3]};
#pragma unroll
        for (int e = 0; e < VEC; ++e) hit |= fn(unpack<E>(v, e)) ? 1u << e : 0u;
    } else {
        for (int e = 0; j + e < len; ++e) hit |= fn(to_f32(x[j + e])) ? 1u << e : 0u;
    }
    return hit;
}

// Collects the logits that reach `from` (not NaN) in LDS; returns their
// number, of which the first kCand are there.
template <typename E, int NT, int NV>
__device__ __forceinline__ int collect(const float (&vm)[NV], const E* __restrict__ x, int len, float from,
                                       WideLds<NT>& sh)
{
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    uint32_t vectors = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) vectors |= vm[i] >= from ? 1u << i : 0u;
    for (; vectors; vectors &= vectors - 1) {
        const int j = (__builtin_ctz(vectors) * NT + (int)threadIdx.x) * kVec<E>;
        for (uint32_t hit = which(x, j, len, [&](float v) { return v >= from; }); hit; hit &= hit - 1) {
            const int e = j + __builtin_ctz(hit), at = atomicAdd(&sh.count, 1);
            if (at < kCand) sh.cand[at] = make_cand(to_f32(x[e]), e);
        }
    }
    __syncthreads();
    return sh.count;
}

// Ranks the n collected candidates and gives out the first k.
template <int NT, typename Out>
__device__ __forceinline__ void rank_collected(const WideLds<NT>& sh, int n, int k, Out&& out)
{
    for (int i = threadIdx.x; i < n; i += NT) {
        const Cand c = sh.cand[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += sh.cand[j] > c;
        if (rank < k) out(rank, c);
    }
}

// Gives out the logits that equal t (NaN: the NaN ones) in the order of their
// indices, from rank n on, until k are out; returns the number that are out.
template <typename E, int NT, typename Out>
__device__ __forceinline__ int fill_equal(const E* __restrict__ x, int len, float t, int n, int k, WideLds<NT>& sh,
                                          Out&& out)
{
    const int lane = threadIdx.x & 63, w = (int)threadIdx.x >> 6;
    for (int base = 0; base < len && n < k; base += NT * kVec<E>) {
        const int j0 = base + (int)threadIdx.x * kVec<E>;
        uint32_t hit = which(x, j0, len, [&](float v) { return v == t || (t != t && v != v); });
        const int mine = __popc(hit);
        int upto = mine;                // of this wave's lanes so far
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        __syncthreads();
        if (lane == 63) sh.part[0][w] = __int_as_float(upto);
        __syncthreads();
        int rank = n + upto - mine;
        for (int q = 0; q < NT / 64; ++q) {
            const int c = __float_as_int(sh.part[0][q]);
            if (q < w) rank += c;
            n += c;
        }
        for (; hit && rank < k; hit &= hit - 1, ++rank) out(rank, make_cand(t, j0 + __builtin_ctz(hit)));
    }
    return min(n, k);
}

// Number of logits that reach v, over the workgroup.
template <typename E, int NT>
__device__ __forceinline__ int count_reaching(const E* __restrict__ x, int len, float v, WideLds<NT>& sh)
{
    int n = 0;
    for (int j = (int)threadIdx.x * kVec<E>; j < len; j += NT * kVec<E>)
        n += __popc(which(x, j, len, [&](float u) { return u >= v; }));
    for (int o = 32; o; o >>= 1) n += __shfl_xor(n, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.part[0][threadIdx.x >> 6] = __int_as_float(n);
    __syncthreads();
    n = 0;
    for (int q = 0; q < NT / 64; ++q) n += __float_as_int(sh.part[0][q]);
    return n;
}

// Gives out(rank, candidate) for the k largest logits of the segment (k <= its
// length); candidate indices count from the segment's start.
//
// The logits that reach the bound are collected in LDS, a little more than k
// of them as a rule, and each finds its rank by counting those before it.
// Two things need more.  Fewer than k groups hold anything above -infinity
// (rows masked to few classes): all such logits are collected, and the places
// that they leave go to the others in the order of their indices.  More than
// kCand reach the bound (many equal logits, as in an untrained layer's rows):
// the bound is raised by halving the interval of keys up to the maximum until
// few enough reach it, or until it is the k-th largest value itself; then the
// larger ones are ranked and equal ones fill up by index.
template <typename E, int NT, int NV, typename Out>
__device__ __forceinline__ void select_top(const float (&vm)[NV], float m, const E* __restrict__ x, int len, int k,
                                           WideLds<NT>& sh, Out&& out)
{
    float bound = sh.bound;
    if (bound == kNegInf) bound = key_value(order_key(kNegInf) + 1);
    int n = collect<E, NT, NV>(vm, x, len, bound, sh);
    if (n > kCand) {
        uint32_t lo = order_key(bound), hi = order_key(m) + 1;     // n reach lo; none reach hi
        while (hi - lo > 1 && n > kCand) {
            const uint32_t mid = lo + (hi - lo) / 2;
            const int c = count_reaching<E, NT>(x, len, key_value(mid), sh);
            if (c >= k) lo = mid, n = c;
            else hi = mid;
        }
        const float t = key_value(lo);
        if (n > kCand) {                // hi = lo + 1: the k-th largest is t
            n = 0;
            if (t < m) {
                n = collect<E, NT, NV>(vm, x, len, key_value(hi), sh);
                rank_collected<NT>(sh, n, k, out);
            }
            fill_equal<E, NT>(x, len, t, n, k, sh, out);
            return;
        }
        n = collect<E, NT, NV>(vm, x, len, t, sh);
    }
    rank_collected<NT>(sh, n, k, out);
    if (n < k) n = fill_equal<E, NT>(x, len, kNegInf, n, k, sh, out);
    if (n < k) fill_equal<E, NT>(x, len, NAN, n, k, sh, out);
}

struct LogprobOutputs {
    float *logp, *entropy, *lse, *top_logp;
    int32_t* top_idx;
    const float *g_logp, *g_ent;
};

// A segment's statistics for the join.
struct Part {
    float m, s, u, pad;
};

template <typename E, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void k_wide_logprobs(const E* __restrict__ logits, const int32_t* __restrict__ token,
                                                      RowArgs a, LogprobOutputs o, E* __restrict__ grad,
                                                      Part* __restrict__ parts, Cand* __restrict__ lists)
{
    __shared__ WideLds<NT> sh;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int r = blockIdx.x / a.nseg, sg = blockIdx.x - r * a.nseg;
    const int j0 = sg * a.seg;
    const E* x = logits + r * a.stride + j0;
    Held<E, NT, NV> h;
    h.load(x, min(a.seg, a.V - j0));
    float vm[NV];
    float m = h.maxima(vm);
    const int k = min(a.k, h.len);
    if (k > 0) {                        // the maxima of kGroups groups: adjacent threads, or one wave's vectors
        if constexpr (NT >= kGroups) {
            constexpr int T = NT / kGroups;
            const float g = over_lanes<T>(m, Max());
            if (tid % T == 0) sh.group[tid / T] = g;
        } else {
            static_assert(NT * NV == kGroups, "one group a vector");
#pragma unroll
            for (int i = 0; i < NV; ++i) sh.group[i * NT + tid] = vm[i];
        }
    }
    m = over_wave(m, Max());
    if (lane == 0) sh.part[0][w] = m;
    __syncthreads();
    m = join_parts<NT>(sh.part[0], Max());
    const Exponent ex(m, a);
    float s = 0.0f, u = 0.0f;
    h.each([&](float v) {
        const float z = ex.z(v), e = pow2(z);
        s += e;
        u = fmaf(e, z_finite(z), u);
    });
    s = over_wave(s, Add());
    u = over_wave(u, Add());
    if (lane == 0) sh.part[1][w] = s, sh.part[2][w] = u;
    if (k > 0 && w == 0) {
        const float b = bound_of_kth<kGroups>(sh.group, k, lane);
        if (lane == 0) sh.bound = b;
    }
    __syncthreads();
    s = join_parts<NT>(sh.part[1], Add());
    u = join_parts<NT>(sh.part[2], Add());
    if (a.nseg > 1) {
        const int64_t at = (int64_t)r * a.nseg + sg;
        if (tid == 0) parts[at] = Part{m, s, u, 0.0f};
        if (a.k > 0) {
            Cand* list = lists + at * a.k;
            for (int i = k + tid; i < a.k; i += NT) list[i] = 0;
            select_top<E, NT, NV>(vm, m, x, h.len, k, sh, [&](int rank, Cand c) {
                list[rank] = c - (Cand)j0;          // the index counts from the row's start
            });
        }
        return;
    }
    const RowStat st = row_stat(ex, s, u);
    const int tok = token ? token[r] : -1;
    const bool there = tok >= 0 && tok < a.V;
    if (tid == 0) {
        if (o.logp) o.logp[r] = there ? row_logp(st, a, to_f32(x[tok])) : 0.0f;
        if (o.entropy) o.entropy[r] = st.H;
        if (o.lse) o.lse[r] = row_lse(st, a);
    }
    if (k > 0)
        select_top<E, NT, NV>(vm, m, x, h.len, k, sh, [&](int rank, Cand c) {
            o.top_idx[(int64_t)r * a.k + rank] = cand_index(c);
            o.top_logp[(int64_t)r * a.k + rank] = row_logp(st, a, cand_value(c));
        });
    if (!grad) return;
    E* out = grad + r * a.grad_stride;
    const float g = there && o.g_logp ? o.g_logp[r] : 0.0f, ge = o.g_ent ? o.g_ent[r] : 0.0f;
    const float inv_s = st.empty ? 0.0f : a.inv_t / st.s, k0 = st.empty ? 0.0f : fmaf(ge, st.H - st.lz, g);
    auto value = [&](float v) {
        const float z = ex.z(v);
        return -(pow2(z) * inv_s) * fmaf(ge * kLn2, z_finite(z), k0);
    };
    h.store(out, x, value);
    __syncthreads();
    if (tid == 0 && there && !st.empty) out[tok] = from_f32<E>(value(to_f32(x[tok])) + g * a.inv_t);
}

// Joins the statistics of a row's segments: the row's exponents, s and u, the
// same in every thread.
template <int NT>
__device__ __forceinline__ Exponent join_row(const Part* __restrict__ parts, const RowArgs& a, float& s, float& u,
                                             float (*part)[NT / 64])
{
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    float m = kNegInf;
    for (int i = tid; i < a.nseg; i += NT) m = fmaxf(m, parts[i].m);
    m = over_wave(m, Max());
    if (lane == 0) part[0][w] = m;
    __syncthreads();
    const Exponent ex(join_parts<NT>(part[0], Max()), a);
    s = u = 0.0f;
    for (int i = tid; i < a.nseg; i += NT) {
        const Part p = parts[i];
        const Exponent own(p.m, a);
        const float d = ex.from(own), f = pow2(d);
        s += p.s * f;
        u += f * fmaf(p.s, z_finite(d), p.u);
    }
    s = over_wave(s, Add());
    u = over_wave(u, Add());
    if (lane == 0) part[1][w] = s, part[2][w] = u;
    __syncthreads();
    s = join_parts<NT>(part[1], Add());
    u = join_parts<NT>(part[2], Add());
    __syncthreads();
    return ex;
}

constexpr int kJoinThreads = 256;
constexpr int kJoinHeads = 2048;        // list heads whose k-th largest bounds the row's
constexpr int kJoinLanes = 4;
constexpr int kJoinRank = 512;          // candidates that are ranked by counting, at least LIF_TOP_MAX

struct JoinLds {
    float part[3][kJoinThreads / 64];
    Cand bound, top;
    int count;
    Cand cand[kJoinHeads];
};

// Number of candidates in the sorted lists that reach c.
__device__ __forceinline__ int count_listed(const Cand* __restrict__ lists, int nseg, int k, Cand c, JoinLds& sh)
{
    int n = 0;
    for (int s = threadIdx.x; s < nseg; s += kJoinThreads) {
        int lo = 0, hi = k;             // the first entry of list s below c
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (lists[(int64_t)s * k + mid] >= c) lo = mid + 1;
            else hi = mid;
        }
        n += lo;
    }
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    if (n) atomicAdd(&sh.count, n);
    __syncthreads();
    return sh.count;
}

// Calls fn for the candidates that reach c: kJoinLanes lanes a list, each
// until its first entry below c. Join of a row of 300000 with 128 alternatives:
// 18 us, 41 with every entry read; 8 lanes 20, 16 lanes 24, 2 lanes 18 but 58
// for 48 where all logits are equal.
template <typename Fn>
__device__ __forceinline__ void for_listed(const Cand* __restrict__ lists, int nseg, int k, Cand c, Fn&& fn)
{
    for (int s = threadIdx.x / kJoinLanes; s < nseg; s += kJoinThreads / kJoinLanes)
        for (int i = threadIdx.x % kJoinLanes; i < k; i += kJoinLanes) {
            const Cand v = lists[(int64_t)s * k + i];
            if (v < c) break;
            fn(v);
        }
}

// The k largest of the sorted lists of a row's segments: the k-th largest of
// the lists' first entries bounds the row's k-th largest from below; what
// reaches it is collected and ranked by counting. The lists are sorted from
// the largest down, unused entries 0.
template <typename Out>
__device__ __forceinline__ void join_lists(const Cand* __restrict__ lists, int nseg, int k, JoinLds& sh, Out&& out)
{
    const int tid = threadIdx.x;
    const int heads = min(k, min(2 * k / nseg + 2, kJoinHeads / nseg));      // of each list; nseg <= kJoinHeads / 2
    const int nh = heads * nseg;
    for (int i = tid; i < nh; i += kJoinThreads) sh.cand[i] = lists[(int64_t)(i / heads) * k + i % heads];
    if (tid == 0) sh.bound = 1, sh.top = ~0ull, sh.count = 0;
    __syncthreads();
    if (nh >= k)
        for (int i = tid; i < nh; i += kJoinThreads) {
            const Cand c = sh.cand[i];
            int rank = 0;
            for (int j = 0; j < nh; ++j) rank += sh.cand[j] > c;
            if (rank == k - 1 && c) sh.bound = c;
            if (rank == 0 && c) sh.top = c;
        }
    __syncthreads();
    const Cand bound = sh.bound;
    for_listed(lists, nseg, k, bound, [&](Cand c) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < kJoinHeads) sh.cand[at] = c;
    });
    __syncthreads();
    int n = sh.count;
    if (n > kJoinRank) {
        // The largest come from few of the lists (equal or ordered logits): the
        // bound rises by halving. At least k and n > kJoinRank candidates reach
        // lo, at most k reach hi; all differ, so n falls below kJoinRank before
        // the two meet. 300000 equal logits, 128 alternatives: 48 us; 1728 with
        // every listed candidate ranked.
        Cand lo = bound, hi = sh.top;
        while (n > kJoinRank) {
            const Cand mid = lo + (hi - lo) / 2;
            const int c = count_listed(lists, nseg, k, mid, sh);
            if (c >= k) lo = mid, n = c;
            else hi = mid;
        }
        __syncthreads();
        if (tid == 0) sh.count = 0;
        __syncthreads();
        for_listed(lists, nseg, k, lo, [&](Cand c) { sh.cand[atomicAdd(&sh.count, 1)] = c; });
        __syncthreads();
    }
    for (int i = tid; i < n; i += kJoinThreads) {
        const Cand c = sh.cand[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += sh.cand[j] > c;
        if (rank < k) out(rank, c);
    }
}

// Second launch over a row's segments: grid (segments that write the
// gradient, or one) x rows.
template <typename E>
__global__ __launch_bounds__(kJoinThreads) void k_join_logprobs(const E* __restrict__ logits,
                                                                const int32_t* __restrict__ token, RowArgs a,
                                                                LogprobOutputs o, E* __restrict__ grad, int pieces,
                                                                int piece, const Part* __restrict__ parts,
                                                                const Cand* __restrict__ lists)
{
    __shared__ JoinLds sh;
    const int tid = threadIdx.x;
    const int r = blockIdx.x / pieces, pc = blockIdx.x - r * pieces;
    const E* x = logits + r * a.stride;
    float s, u;
    const Exponent ex = join_row<kJoinThreads>(parts + (int64_t)r * a.nseg, a, s, u, sh.part);
    const RowStat st = row_stat(ex, s, u);
    const int tok = token ? token[r] : -1;
    const bool there = tok >= 0 && tok < a.V;
    if (pc == 0) {
        if (tid == 0) {
            if (o.logp) o.logp[r] = there ? row_logp(st, a, to_f32(x[tok])) : 0.0f;
            if (o.entropy) o.entropy[r] = st.H;
            if (o.lse) o.lse[r] = row_lse(st, a);
        }
        if (a.k > 0)
            join_lists(lists + (int64_t)r * a.nseg * a.k, a.nseg, a.k, sh, [&](int rank, Cand c) {
                o.top_idx[(int64_t)r * a.k + rank] = cand_index(c);
                o.top_logp[(int64_t)r * a.k + rank] = row_logp(st, a, cand_value(c));
            });
    }
    if (!grad) return;
    E* out = grad + r * a.grad_stride;
    const float g = there && o.g_logp ? o.g_logp[r] : 0.0f, ge = o.g_ent ? o.g_ent[r] : 0.0f;
    const float inv_s = st.empty ? 0.0f : a.inv_t / st.s, k0 = st.empty ? 0.0f : fmaf(ge, st.H - st.lz, g);
    auto value = [&](float v) {
        const float z = ex.z(v);
        return -(pow2(z) * inv_s) * fmaf(ge * kLn2, z_finite(z), k0);
    };
    const int j0 = pc * piece, j1 = min(j0 + piece, a.V);
    for (int j = j0; j < j1; j += kJoinThreads * kVec<E>) {
        Held<E, kJoinThreads, 1> h;
        h.load(x + j, j1 - j);
        h.store(out + j, x + j, value);
    }
    __syncthreads();
    if (tid == 0 && there && !st.empty && tok >= j0 && tok < j1)
        out[tok] = from_f32<E>(value(to_f32(x[tok])) + g * a.inv_t);
}

// ---------------------------------------------------------------------------
// Distillation of wide rows.  The listed classes are found with a bitmap in
// LDS and taken out of the held elements (set to -infinity) before the maximum
// and the sums, which are then the others'; the listed logits are read one by
// one.  Their gradients are written last.
// ---------------------------------------------------------------------------
template <int NT> struct ListLds {
    int idx[LIF_TOP_MAX];               // -1: unused
    int first[LIF_TOP_MAX];             // the one entry of its class that counts there
    float lt[LIF_TOP_MAX], x[LIF_TOP_MAX];
    double q[LIF_TOP_MAX], sq;
    float m;                            // the largest logp
    int used, distinct;
    float part[3][NT / 64];
};

// Entries lane and lane + 64 of the teacher's list (class -1: unused) and the
// student's logits there, kept by one wave, with the sum of q.
static_assert(LIF_TOP_MAX <= 128, "at most two entries a lane");
template <int NT>
__device__ __forceinline__ void keep_list(ListLds<NT>& sh, const RowArgs& a, const int (&j)[2], const float (&lt)[2],
                                          const float (&x)[2], int lane)
{
    float m = kNegInf;
#pragma unroll
    for (int q = 0; q < 2; ++q)
        if (j[q] >= 0) m = fmaxf(m, lt[q]);
    m = over_wave(m, Max());
    const float shift = list_shift(m, a.tail);
    double sq = 0.0;
    int used = 0;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int i = lane + 64 * q;
        const bool is = j[q] >= 0;
        const double e = is ? exp((double)lt[q] - (double)shift) : 0.0;
        sq += e;
        used += __popcll(__ballot(is));
        if (i >= a.k) continue;
        sh.idx[i] = j[q];
        sh.lt[i] = is ? lt[q] : kNegInf;
        sh.q[i] = e;
        sh.x[i] = is ? x[q] : kNegInf;
    }
    sq = sum_over_wave(sq);
    if (lane == 0) sh.sq = sq, sh.m = m, sh.used = used;
}

// Marks the first entry of each class.
template <int NT> __device__ __forceinline__ void find_first(ListLds<NT>& sh, int k, int from, int step)
{
    for (int i = from; i < k; i += step) {
        bool first = sh.idx[i] >= 0;
        for (int p = 0; p < i; ++p) first &= sh.idx[p] != sh.idx[i];
        sh.first[i] = first;
    }
}

// The student's largest logit in the list, the same in every lane.
template <int NT> __device__ __forceinline__ float list_max(const ListLds<NT>& sh, int k, int lane)
{
    return over_wave(fmaxf(lane < k ? sh.x[lane] : kNegInf, lane + 64 < k ? sh.x[lane + 64] : kNegInf), Max());
}

// The sum of the terms e of distinct classes, by one wave.
template <int NT>
__device__ __forceinline__ float sum_list(ListLds<NT>& sh, int k, const Exponent& ex, int lane)
{
    float e = 0.0f;
    int distinct = 0;
    for (int i = lane; i < 128; i += 64) {
        const bool first = i < k && sh.first[i];
        if (first) e += pow2(ex.z(sh.x[i]));
        distinct += __popcll(__ballot(first));
    }
    if (lane == 0) sh.distinct = distinct;
    return over_wave(e, Add());
}

// The loss of a row, by one wave.
template <int NT>
__device__ __forceinline__ double list_loss(const ListLds<NT>& sh, int k, const RowArgs& a, const RowStat& st,
                                            const Teacher& t, const Rest& rest, int lane)
{
    const double add = log_scale(t, sh.m, a.tail);
    double v = 0.0;
    for (int i = lane; i < k; i += 64) {
        if (sh.idx[i] < 0) continue;
        const double lp = st.empty ? (double)kNegInf : ((double)sh.x[i] - (double)st.m) * a.inv_td - (double)st.ls;
        v += entry_loss(sh.q[i] * t.scale, (double)sh.lt[i] + add, lp);
    }
    v = sum_over_wave(v);
    return t.none ? 0.0 : v + tail_loss(t, rest, st, a);
}

// The gradients at the listed classes in [j0, j1), after those of the others.
template <typename E, int NT>
__device__ __forceinline__ void store_listed(const ListLds<NT>& sh, int k, const Exponent& ex, const RowStat& st,
                                             const Teacher& t, float c_top, float w, int j0, int j1,
                                             E* __restrict__ out)
{
    const bool dead = t.none || st.empty;
    for (int i = threadIdx.x; i < k; i += NT) {
        const int j = sh.idx[i];
        if (j < j0 || j >= j1) continue;
        double q = sh.q[i];
        if (sh.distinct < sh.used) {    // repeated entries write the same value
            q = 0.0;
            for (int p = 0; p < k; ++p)
                if (sh.idx[p] == j) q += sh.q[p];
        }
        const double v = (double)pow2(ex.z(sh.x[i])) * (double)c_top - q * t.scale;     // one rounding at the end
        out[j] = from_f32<E>(dead ? 0.0f : (float)(v * (double)w));
    }
}

template <typename E, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void k_wide_distill(const E* __restrict__ logits, const float* __restrict__ t_logp,
                                                     const int32_t* __restrict__ t_idx, RowArgs a,
                                                     const float* __restrict__ weight, float* __restrict__ loss,
                                                     E* __restrict__ grad, Part* __restrict__ parts)
{
    constexpr int VEC = kVec<E>;
    __shared__ ListLds<NT> sh;
    __shared__ uint32_t bits[NT * NV * VEC / 32];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int r = blockIdx.x / a.nseg, sg = blockIdx.x - r * a.nseg;
    const int j0 = sg * a.seg;
    const E* row = logits + r * a.stride;
    // the list's loads first: they are short, and the logits that it names are
    // on their way right behind the row; the first wave works on it meanwhile
    int ej[2] = {-1, -1};
    float el[2] = {}, xl[2] = {};
    if (w == 0)
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (lane + 64 * q < a.k) {
                ej[q] = t_idx[(int64_t)r * a.k + lane + 64 * q];
                el[q] = t_logp[(int64_t)r * a.k + lane + 64 * q];
            }
    Held<E, NT, NV> h;
    h.load(row + j0, min(a.seg, a.V - j0));
    if (w == 0) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (ej[q] < 0 || ej[q] >= a.V) ej[q] = -1;
            else if (a.nseg == 1) xl[q] = to_f32(row[ej[q]]);
        }
        if (a.nseg == 1) keep_list(sh, a, ej, el, xl, lane);
    }
    for (int i = tid; i < (h.len + 31) / 32; i += NT) bits[i] = 0;
    __syncthreads();
    if (w == 0) {
        bool again = false;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int i = lane + 64 * q, j = ej[q] - j0;
            if (i >= a.k) continue;
            bool first = false;
            if (ej[q] >= 0 && j >= 0 && j < h.len) {
                first = !(atomicOr(&bits[j >> 5], 1u << (j & 31)) >> (j & 31) & 1);
                again |= !first;
            }
            sh.first[i] = first;
        }
        // a class listed twice counts at the entry of the lowest index, whichever came first to its bit
        if (a.nseg == 1 && __any(again)) find_first(sh, a.k, lane, 64);
    }
    const float m_list = a.nseg == 1 ? list_max(sh, a.k, lane) : kNegInf;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (!h.any(i) || h.first(i) >= h.len) continue;
        const uint32_t b = bits[h.first(i) >> 5] >> (h.first(i) & 31) & ((1u << VEC) - 1u);
        if (b) h.drop(i, b);
    }
    float vm[NV];
    float m = over_wave(h.maxima(vm), Max());
    if (lane == 0) sh.part[0][w] = m;
    __syncthreads();
    m = join_parts<NT>(sh.part[0], Max());
    const Exponent er(m, a), ex(fmaxf(m, m_list), a);
    float s = 0.0f;
    h.each([&](float v) { s += pow2(er.z(v)); });
    s = over_wave(s, Add());
    if (lane == 0) sh.part[1][w] = s;
    if (a.nseg > 1) {
        __syncthreads();
        if (tid == 0) parts[(int64_t)r * a.nseg + sg] = Part{m, join_parts<NT>(sh.part[1], Add()), 0.0f, 0.0f};
        return;
    }
    if (w == 0) {
        const float e = sum_list<NT>(sh, a.k, ex, lane);
        if (lane == 0) sh.part[2][0] = e;
    }
    __syncthreads();
    const Rest rest(er, ex, join_parts<NT>(sh.part[1], Add()));
    const RowStat st = row_stat(ex, fmaf(rest.s, rest.f, sh.part[2][0]), 0.0f);
    const Teacher t = teacher_of(sh.sq, sh.m, a.tail, sh.distinct == a.V);
    if (grad) {
        float c_top, c_rest;
        grad_factors(t, st, rest, c_top, c_rest);
        const float wt = (weight ? weight[r] : 1.0f) * a.inv_t, f = t.none || st.empty ? 0.0f : c_rest * wt;
        E* out = grad + r * a.grad_stride;
        // a row without a gradient may hold a NaN, which 0 f would keep
        if (t.none || st.empty) h.store(out, row, [&](float) { return 0.0f; });
        else h.store(out, row, [&](float v) { return pow2(er.z(v)) * f; });
        __syncthreads();
        store_listed<E, NT>(sh, a.k, ex, st, t, c_top, wt, 0, a.V, out);
    }
    if (loss && w == 0) {
        const double v = list_loss<NT>(sh, a.k, a, st, t, rest, lane);
        if (lane == 0) loss[r] = (float)v;
    }
}

template <typename E>
__global__ __launch_bounds__(kJoinThreads) void k_join_distill(const E* __restrict__ logits,
                                                               const float* __restrict__ t_logp,
                                                               const int32_t* __restrict__ t_idx, RowArgs a,
                                                               const float* __restrict__ weight,
                                                               float* __restrict__ loss, E* __restrict__ grad,
                                                               int pieces, int piece, const Part* __restrict__ parts)
{
    constexpr int NT = kJoinThreads;
    __shared__ ListLds<NT> sh;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int r = blockIdx.x / pieces, pc = blockIdx.x - r * pieces;
    const E* row = logits + r * a.stride;
    if (w == 0) {
        int ej[2] = {-1, -1};
        float el[2] = {}, xl[2] = {};
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int64_t at = (int64_t)r * a.k + lane + 64 * q;
            if (lane + 64 * q >= a.k || t_idx[at] < 0 || t_idx[at] >= a.V) continue;
            ej[q] = t_idx[at];
            el[q] = t_logp[at];
            xl[q] = to_f32(row[ej[q]]);
        }
        keep_list(sh, a, ej, el, xl, lane);
    }
    __syncthreads();
    find_first(sh, a.k, tid, NT);
    float s_rest, u;
    const Exponent er = join_row<NT>(parts + (int64_t)r * a.nseg, a, s_rest, u, sh.part);
    const float m_list = list_max(sh, a.k, lane);
    const Exponent ex(er.none ? m_list : fmaxf(er.m, m_list), a);
    if (w == 0) {
        const float e = sum_list<NT>(sh, a.k, ex, lane);
        if (lane == 0) sh.part[2][0] = e;
    }
    __syncthreads();
    const Rest rest(er, ex, s_rest);
    const RowStat st = row_stat(ex, fmaf(rest.s, rest.f, sh.part[2][0]), 0.0f);
    const Teacher t = teacher_of(sh.sq, sh.m, a.tail, sh.distinct == a.V);
    if (loss && pc == 0 && w == 0) {
        const double v = list_loss<NT>(sh, a.k, a, st, t, rest, lane);
        if (lane == 0) loss[r] = (float)v;
    }
    if (!grad) return;
    float c_top, c_rest;
    grad_factors(t, st, rest, c_top, c_rest);
    const float wt = (weight ? weight[r] : 1.0f) * a.inv_t, f = t.none || st.empty ? 0.0f : c_rest * wt;
    E* out = grad + r * a.grad_stride;
    const int j0 = pc * piece, j1 = min(j0 + piece, a.V);
    for (int j = j0; j < j1; j += NT * kVec<E>) {
        Held<E, NT, 1> h;
        h.load(row + j, j1 - j);
        if (t.none || st.empty) h.store(out + j, row + j, [&](float) { return 0.0f; });
        else h.store(out + j, row + j, [&](float v) { return pow2(er.z(v)) * f; });
    }
    __syncthreads();
    store_listed<E, NT>(sh, a.k, ex, st, t, c_top, wt, j0, j1, out);
}

int check_rows(const lif_rows_params* p)
{
    if (!p || p->R < 0 || p->V < 1 || p->k < 0 || p->k > p->V || p->reserved != 0) return LIF_ERR_ARG;
    if (p->dtype != LIF_F32 && p->dtype != LIF_BF16 && p->dtype != LIF_F16) return LIF_ERR_ARG;
    if (p->flags & ~LIF_DISTILL_TAIL) return LIF_ERR_ARG;
    if (p->stride < p->V || p->grad_stride < p->V) return LIF_ERR_ARG;
    if (!(p->temperature >= 1.0 / 1048576.0 && p->temperature <= 1048576.0)) return LIF_ERR_ARG;
    if (p->k > LIF_TOP_MAX || p->V > kMaxV) return LIF_ERR_SIZE;
    return LIF_OK;
}

// Workgroup shapes of the wide kernels: threads and vectors a thread.  us, 20
// alternatives, (gradient,) distillation, with the shape and with another:
//   20000 x   700 bf16  30 35         {128, 2}   37 42
//    8000 x  4096       33 42         {512, 2}   56 57
//    4000 x 12000       50 54 51      {256, 16}  36 43 53
//    4000 x 30000       70 115 98     {256, 16}  55 101 101
//    2000 x 40000       49 80 80      {1024, 8}  72 100 75
// (The third suits distillation; the other two would gain by 256 threads.)
struct Shape {
    int nt, nv;
};
constexpr Shape kShapes[] = {{64, 4}, {256, 4}, {512, 8}, {512, 16}, {1024, 16}};
constexpr int kFewRows = 64, kLongVectors = 4096;       // at most and more than
constexpr int kNumShapes = sizeof(kShapes) / sizeof(kShapes[0]);

struct RowPlan {
    RowArgs a;
    int shape;                          // -1: narrow
};

RowPlan plan_rows(const lif_rows_params& p)
{
    RowPlan q;
    RowArgs& a = q.a;
    a.R = p.R;
    a.V = p.V;
    a.k = p.k;
    a.stride = p.stride;
    a.grad_stride = p.grad_stride;
    a.c = (float)(1.4426950408889634074 / p.temperature);
    a.c_pow2 = (float)exp2(ceil(log2((double)a.c)));
    a.inv_t = (float)(1.0 / p.temperature);
    a.inv_td = 1.0 / p.temperature;
    a.tail = p.flags & LIF_DISTILL_TAIL;
    a.nseg = 1;
    a.seg = p.V;
    q.shape = -1;
    if (p.V <= kNarrow) return q;
    const int vec = p.dtype == LIF_F32 ? 4 : 8;
    auto holds = [&](int s) { return kShapes[s].nt * kShapes[s].nv * vec; };
    int seg = p.V;
    if (seg > holds(kNumShapes - 1)) seg = holds(2);            // does not fit: segments of a middling size
    // Few long rows: enough segments for two workgroups on every CU.  That costs
    // a second launch and, for a gradient, a second read, which rows of more
    // than 4096 vectors and up to 64 of them make up for (bf16, in segments and
    // whole, us; 20 alternatives, gradient, distillation with gradient):
    //    8 x  16384  12.2  7.7    7.6  7.1   10.6  8.9
    //    8 x  50048  12.3 10.3    7.8 12.4   10.9 14.0
    //    8 x 131072  12.8 16.5    8.1 23.4   11.0 22.5
    //   64 x  50048  13.6 10.8   11.9 13.6   15.4 15.2
    //   64 x 131072  16.6 18.3   17.3 26.6   20.3 25.5
    //  128 x 131072  19.6 22.0   25.5 29.4   28.9 28.1
    //  192 x 131072  26.5 24.9   36.6 32.1   40.5 31.0
    //  255 x   4104  12.4  7.4    8.9  5.9   12.1  7.9
    if (p.R > 0 && p.R <= kFewRows && seg > kLongVectors * vec) {
        const int want = (512 + p.R - 1) / p.R;
        int few = (p.V + want - 1) / want;
        few = few < 512 * vec ? 512 * vec : few;
        if (few < seg) seg = few;
    }
    a.nseg = (p.V + seg - 1) / seg;
    a.seg = ((p.V + a.nseg - 1) / a.nseg + vec - 1) / vec * vec;
    a.nseg = (p.V + a.seg - 1) / a.seg;
    for (q.shape = 0; holds(q.shape) < a.seg;) ++q.shape;
    return q;
}

size_t rows_ws(const RowPlan& q)
{
    return q.a.nseg > 1 ? (size_t)q.a.R * q.a.nseg * (sizeof(Part) + (size_t)q.a.k * sizeof(Cand)) : 0;
}

// A launch has fewer than 2^32 threads.
bool too_many(const RowPlan& q)
{
    // a narrow row takes up to 16 threads; the join's 256 a row are fewer than the segments' in all
    const int64_t per_row = q.shape < 0 ? 16 : (int64_t)q.a.nseg * kShapes[q.shape].nt;
    return (int64_t)q.a.R * per_row > ((int64_t)1 << 32) - 1024;
}

// Calls fn(element, threads, vectors) with types that carry them.
template <int N> struct Int { static constexpr int value = N; };
template <typename Fn> void with_shape(int dtype, int shape, Fn&& fn)
{
    with_dtype(dtype, [&](auto e) {
        switch (shape) {
            case 0: fn(e, Int<kShapes[0].nt>(), Int<kShapes[0].nv>()); break;
            case 1: fn(e, Int<kShapes[1].nt>(), Int<kShapes[1].nv>()); break;
            case 2: fn(e, Int<kShapes[2].nt>(), Int<kShapes[2].nv>()); break;
            case 3: fn(e, Int<kShapes[3].nt>(), Int<kShapes[3].nv>()); break;
            default: fn(e, Int<kShapes[4].nt>(), Int<kShapes[4].nv>()); break;
        }
    });
}
// Lanes for a narrow row: up to 16 elements a lane (128000 x 20 f32 with 5
// alternatives: 12 us; with up to 24 elements 14.5, with up to 6 13;
// 200000 x 40 f32 distillation 40, 35, 55).
template <typename Fn> void with_lanes(int dtype, int V, Fn&& fn)
{
    with_dtype(dtype, [&](auto e) {
        if (V <= 16) fn(e, Int<1>());
        else if (V <= 32) fn(e, Int<2>());
        else if (V <= 64) fn(e, Int<4>());
        else if (V <= 128) fn(e, Int<8>());
        else fn(e, Int<16>());
    });
}
static_assert((kNarrow + 15) / 16 <= kNarrowPer && 16 <= kNarrowPer, "a lane's elements have a bit each");

// The staged rows, and behind them k more values a row.
size_t narrow_lds(int V, int L, int k)
{
    return (size_t)(kNarrowThreads / L) * (narrow_pitch(V, L) + k) * sizeof(float);
}

// The pieces of a row that the second launch writes gradients of.
void gradient_pieces(const RowArgs& a, bool grad, int elem, int& pieces, int& piece)
{
    const int unit = kJoinThreads * (16 / elem);                // one vector a thread
    pieces = 1;
    piece = a.V;
    if (!grad) return;
    const int units = (a.V + unit - 1) / unit;
    int want = a.R >= 1024 ? 1 : (1024 + a.R - 1) / a.R;
    if (want > units) want = units;
    piece = (units + want - 1) / want * unit;
    pieces = (a.V + piece - 1) / piece;
}

}  // namespace
}  // namespace lif

extern "C" size_t lif_rows_workspace_size(const lif_rows_params* p)
{
    if (lif::check_rows(p) != LIF_OK) return 0;
    return lif::rows_ws(lif::plan_rows(*p));
}

extern "C" int lif_token_logprobs(const void* logits, const int32_t* token, const lif_rows_params* p, float* logp,
                                  float* entropy, float* lse, float* top_logp, int32_t* top_idx,
                                  const float* grad_logp, const float* grad_entropy, void* grad, void* ws,
                                  size_t ws_bytes, lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_rows(p);
    if (rc) return rc;
    if ((p->R > 0 && !logits) || (p->flags & LIF_DISTILL_TAIL)) return LIF_ERR_ARG;
    if (p->k > 0 && p->R > 0 && (!top_logp != !top_idx)) return LIF_ERR_ARG;
    RowPlan q = plan_rows(*p);
    const size_t need = rows_ws(q);
    if (need > 0 && (!ws || (uintptr_t)ws % sizeof(Part))) return LIF_ERR_ARG;
    if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    if (p->R == 0) return LIF_OK;
    RowArgs& a = q.a;
    if (!top_idx) a.k = 0;
    const hipStream_t s = (hipStream_t)stream;
    if (too_many(q)) return LIF_ERR_SIZE;
    if (q.shape < 0) {
        with_lanes(p->dtype, p->V, [&](auto e, auto l) {
            using E = decltype(e);
            constexpr int L = decltype(l)::value, per = kNarrowThreads / L;
            TIMED_LAUNCH("token_logprobs", (k_narrow_logprobs<E, L>), dim3((unsigned)(((int64_t)a.R + per - 1) / per)),
                         dim3(kNarrowThreads), narrow_lds(a.V, L, 0), s, (const E*)logits, token, a, logp, entropy, lse,
                         top_logp, top_idx, grad_logp, grad_entropy, (E*)grad);
        });
        return check_launch();
    }
    const LogprobOutputs o{logp, entropy, lse, top_logp, top_idx, grad_logp, grad_entropy};
    Part* parts = (Part*)ws;
    Cand* lists = (Cand*)(parts + (size_t)a.R * a.nseg);
    with_shape(p->dtype, q.shape, [&](auto e, auto nt, auto nv) {
        using E = decltype(e);
        constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
        TIMED_LAUNCH("token_logprobs", (k_wide_logprobs<E, NT, NV>), dim3(a.R * a.nseg), dim3(NT), 0, s,
                     (const E*)logits, token, a, o, (E*)grad, parts, lists);
        if (a.nseg > 1) {
            int pieces, piece;
            gradient_pieces(a, grad != nullptr, sizeof(E), pieces, piece);
            TIMED_LAUNCH("token_logprobs_join", (k_join_logprobs<E>), dim3(a.R * pieces), dim3(kJoinThreads), 0, s,
                         (const E*)logits, token, a, o, (E*)grad, pieces, piece, parts, lists);
        }
    });
    return check_launch();
}

extern "C" int lif_distill_top(const void* logits, const float* teacher_logp, const int32_t* teacher_idx,
                               const lif_rows_params* p, const float* weight, float* loss, void* grad, void* ws,
                               size_t ws_bytes, lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_rows(p);
    if (rc) return rc;
    if (p->R > 0 && (!logits || (!loss && !grad) || (p->k > 0 && (!teacher_logp || !teacher_idx)))) return LIF_ERR_ARG;
    const RowPlan q = plan_rows(*p);
    const size_t need = rows_ws(q);
    if (need > 0 && (!ws || (uintptr_t)ws % sizeof(Part))) return LIF_ERR_ARG;
    if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    if (p->R == 0) return LIF_OK;
    const RowArgs& a = q.a;
    const hipStream_t s = (hipStream_t)stream;
    if (too_many(q)) return LIF_ERR_SIZE;
    if (q.shape < 0) {
        with_lanes(p->dtype, p->V, [&](auto e, auto l) {
            using E = decltype(e);
            constexpr int L = decltype(l)::value, per = kNarrowThreads / L;
            TIMED_LAUNCH("distill_top", (k_narrow_distill<E, L>), dim3((unsigned)(((int64_t)a.R + per - 1) / per)),
                         dim3(kNarrowThreads), narrow_lds(a.V, L, a.k), s, (const E*)logits, teacher_logp, teacher_idx,
                         a, weight, loss, (E*)grad);
        });
        return check_launch();
    }
    Part* parts = (Part*)ws;
    with_shape(p->dtype, q.shape, [&](auto e, auto nt, auto nv) {
        using E = decltype(e);
        constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
        TIMED_LAUNCH("distill_top", (k_wide_distill<E, NT, NV>), dim3(a.R * a.nseg), dim3(NT), 0, s, (const E*)logits,
                     teacher_logp, teacher_idx, a, weight, loss, (E*)grad, parts);
        if (a.nseg > 1) {
            int pieces, piece;
            gradient_pieces(a, grad != nullptr, sizeof(E), pieces, piece);
            TIMED_LAUNCH("distill_join", (k_join_distill<E>), dim3(a.R * pieces), dim3(kJoinThreads), 0, s,
                         (const E*)logits, teacher_logp, teacher_idx, a, weight, loss, (E*)grad, pieces, piece, parts);
        }
    });
    return check_launch();
}
