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
// products keeps the rounding of the recurrence within a wave's steps; the
// state that enters them comes from composed maps.
#include "lif_host.hpp"
#include "lif_types.hpp"
#include "lif_walk.hpp"

namespace lif {
namespace {

constexpr int kTS = 8;            // steps of a wave in a tile
constexpr int kMaxWaves = 8;      // waves of a workgroup
// The time axis is shared out where one step of one input has less than
// kSplitBytes, over about kSplitGroups workgroups that take at least
// kSplitBlocks blocks of LIF_GATED_MARK steps each.  32 KB a step (32 x 256
// f32, 1000 steps): forward and backward 70 -> 55 us; 40 KB (20 x 1000 bf16,
// 3000 steps): forward 114 -> 133, backward 199 -> 200.  Short sequences gain
// from it at narrower steps only: 30 KB, 500 steps 40 -> 52 us, 2 KB 32 -> 24.
constexpr int64_t kSplitBytes = 36 << 10;
constexpr int kSplitGroups = 1024;
constexpr int kSplitBlocks = 2;
constexpr int kSplitMin = 8;         // fewer blocks than this are not shared out
static_assert(LIF_GATED_MARK % kTS == 0 && kTS * kMaxWaves == LIF_GATED_MARK,
              "a mark is the state entering some wave's first step, and a backward tile starts at one");

// a = sigmoid(f) and 1 - a, to a relative error below (6 + 2 |f|) 2^-24 each:
// the exponent is rounded once, to |f| 2^-24, and its power squared (8 units of
// 2^-24 for |f| up to 5, 18 at 20, 64 at 80).  e = e^{-|f|} is the square of a power of two, so that it keeps values below
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

// The wave's index in its workgroup, in a scalar register.
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

// What a launch works on: `groups` = B * ceil(D / CPL) lanes in all, `S`
// segments of `seg_len` steps (a multiple of LIF_GATED_MARK) of the time axis.
// Where CPL does not divide D, a sample's last group starts at D - CPL: the
// channels that it shares with the group before get the same bits twice.
struct Geometry {
    int B, T, D, groups, per_sample, columns, S, seg_len;
    bool shared_lines;            // rows are not whole cache lines
    int64_t x_batch, x_time, f_batch, f_time, g_batch, g_time;
};

// A workgroup's column of 64 lanes and segment.  Where rows are not multiples
// of a cache line, neighbouring columns write parts of the same lines: they
// then go to one XCD, so that the parts meet in its L2 (4 x 8192 x 1001 bf16,
// forward and backward 227 -> 191 us; for whole lines the order of launch is
// better, 65521 x 512 bf16 87 -> 76 us).
__device__ __forceinline__ void work_item(const Geometry& g, int& column, int& segment)
{
    const int at = g.shared_lines ? xcd_remap(blockIdx.x, gridDim.x) : blockIdx.x;
    segment = at / g.columns;
    column = at - segment * g.columns;
}

// A lane's place: sample b, first channel d, flat channel c = b * D + d, the
// sample's steps n and the smallest and largest n of the wave.  Lanes past
// the last group repeat it and store nothing.
struct Place {
    int b, d, n, n_min, n_max;
    int64_t c;
    bool live;
};

template <int CPL>
__device__ __forceinline__ Place place_of(const Geometry& g, const int32_t* __restrict__ length, int column, int lane)
{
    Place p;
    const int64_t at = (int64_t)column * kWave + lane;
    p.live = at < g.groups;
    const int cg = p.live ? (int)at : g.groups - 1;
    p.b = cg / g.per_sample;
    p.d = min((cg - p.b * g.per_sample) * CPL, g.D - CPL);
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
template <typename E, int CPL, int TS, int N>
struct Raw {
    E v[N][TS][CPL];
};

// A row stride that the compiler takes for a new value each time: otherwise it
// keeps the multiples of every stride for all TS steps in scalar registers
// across the loops below, and spills them.
__device__ __forceinline__ int64_t fresh(int64_t stride)
{
    asm volatile("" : "+s"(stride));
    return stride;
}

// Loads steps t .. t + TS - 1 of one input; steps at or past the lane's n get
// `rest`.  With f = +infinity (a = 1, 1 - a = 0 exactly), x = 0 and grad_h = 0
// there, such a step is the identity in every composition below.
template <typename E, int CPL, int TS>
__device__ __forceinline__ void load_steps(E (&v)[TS][CPL], const E* __restrict__ base, int64_t stride, int t,
                                           const Place& p, float rest)
{
    stride = fresh(stride);
    const E* at = base + (int64_t)t * stride;
    if (t + TS <= p.n_min) {
#pragma unroll
        for (int i = 0; i < TS; ++i, at += stride) load_elems<E, CPL>(at, v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < TS; ++i, at += stride) {
#pragma unroll
            for (int k = 0; k < CPL; ++k) v[i][k] = from_f32<E>(rest);
            if (t + i < p.n) load_elems<E, CPL>(at, v[i]);
        }
    }
}

// The same for x or grad_h; 0 where there is none.
template <typename E, int CPL, int TS>
__device__ __forceinline__ void load_input(E (&v)[TS][CPL], const E* in, int64_t at, int64_t stride, int t,
                                           const Place& p)
{
    if (in) {
        load_steps<E, CPL, TS>(v, in + at, stride, t, p, 0.0f);
    } else {
#pragma unroll
        for (int i = 0; i < TS; ++i)
#pragma unroll
            for (int k = 0; k < CPL; ++k) v[i][k] = from_f32<E>(0.0f);
    }
}

// A wave's TS steps of the forward recurrence: gates and inputs of the raw
// elements, and the composed map.
template <typename E, int CPL, int TS, bool COUPLED>
__device__ __forceinline__ void compose_steps(const Raw<E, CPL, TS, 2>& r, float (&a)[TS][CPL], float (&u)[TS][CPL],
                                              float (&A)[CPL], float (&H)[CPL])
{
#pragma unroll
    for (int k = 0; k < CPL; ++k) A[k] = 1.0f, H[k] = 0.0f;
#pragma unroll
    for (int i = 0; i < TS; ++i)
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
            float na;
            gate(to_f32(r.v[0][i][k]), a[i][k], na);
            const float v = to_f32(r.v[1][i][k]);
            u[i][k] = COUPLED ? na * v : v;
            H[k] = fmaf(a[i][k], H[k], u[i][k]);
            A[k] *= a[i][k];
        }
}

// Runs a wave's steps from the state `h` that enters them, and stores them.
template <typename E, int CPL, int TS>
__device__ __forceinline__ void run_steps(float (&h)[CPL], const float (&a)[TS][CPL], const float (&u)[TS][CPL], int t,
                                          const Place& p, const Geometry& g, E* __restrict__ out,
                                          float* __restrict__ mk)
{
    if (!p.live) return;
    if (mk && t % LIF_GATED_MARK == 0 && t < g.T)
        store_elems<float, CPL>(mk + (int64_t)(t / LIF_GATED_MARK) * g.D, h);
    if (!out) return;
    const int64_t row = fresh(g.D);
    E* at = out + t * row;
    const bool full = t + TS <= p.n_min;
#pragma unroll
    for (int i = 0; i < TS; ++i, at += row) {
        E o[CPL];
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
            h[k] = fmaf(a[i][k], h[k], u[i][k]);
            o[k] = from_f32<E>(h[k]);
        }
        if (!full) {
            if (t + i >= g.T) return;
#pragma unroll
            for (int k = 0; k < CPL; ++k) o[k] = t + i < p.n ? o[k] : from_f32<E>(0.0f);
        }
        store_elems<E, CPL>(at, o);
    }
}

// Where there are few channels, the time axis is cut into segments that
// workgroups share out: a first launch composes each segment's map, a second
// one works on all segments at once, each from the state that the maps before
// it carry to it.  x and f (backward: f and grad_h) are then read twice, the
// second time in part from the cache behind the L2s.  (One pass, in which
// workgroups wait for the state of the chunk before theirs, keeps too little
// in flight while it waits: 65521 x 512 bf16 87 to 120 us, next to two passes
// of 99 that have since come to 76.)

// The composed map of a segment: of h from f and x, or (REVERSE) of mu from f
// and grad_h; 65521 x 512 bf16 33 us, 134 MB at 4.1 TB/s.  Each wave takes a contiguous part
// of the segment without a barrier; the waves' maps meet once at the end.
template <typename E, int CPL, bool COUPLED, bool REVERSE>
__global__ __launch_bounds__(kMaxWaves* kWave) void k_segment_maps(const E* __restrict__ in, const E* __restrict__ f,
                                                                   const int32_t* __restrict__ length, Geometry g,
                                                                   float2* __restrict__ maps)
{
    constexpr int TS = kTS;
    __shared__ float2 sh[kMaxWaves][CPL][kWave];
    const int lane = threadIdx.x & 63, w = wave_index();
    int column, seg;
    work_item(g, column, seg);
    if (REVERSE) ++seg;                                          // the walk's last segment needs no map
    const Place p = place_of<CPL>(g, length, column, lane);
    const int64_t in_batch = REVERSE ? g.g_batch : g.x_batch, in_time = REVERSE ? g.g_time : g.x_time;
    const int part = g.seg_len / kMaxWaves;                      // a multiple of TS
    const int t0 = seg * g.seg_len + w * part;
    const int blocks = (min(t0 + part, p.n_max) - t0 + TS - 1) / TS;
    float A[CPL], H[CPL];
#pragma unroll
    for (int k = 0; k < CPL; ++k) A[k] = 1.0f, H[k] = 0.0f;
    Raw<E, CPL, TS, 2> cur, nxt;
    auto load = [&](Raw<E, CPL, TS, 2>& r, int j) {
        const int t = t0 + (REVERSE ? blocks - 1 - j : j) * TS;
        load_steps<E, CPL, TS>(r.v[0], f + p.b * g.f_batch + p.d, g.f_time, t, p, INFINITY);
        load_input<E, CPL, TS>(r.v[1], in, p.b * in_batch + p.d, in_time, t, p);
    };
    if (blocks > 0) load(cur, 0);
    for (int j = 0; j < blocks; ++j) {
        if (j + 1 < blocks) load(nxt, j + 1);
#pragma unroll
        for (int q = 0; q < TS; ++q) {
            const int i = REVERSE ? TS - 1 - q : q;
#pragma unroll
            for (int k = 0; k < CPL; ++k) {
                float a, na;
                gate(to_f32(cur.v[0][i][k]), a, na);
                const float v = to_f32(cur.v[1][i][k]);
                H[k] = REVERSE ? a * (H[k] + v) : fmaf(a, H[k], COUPLED ? na * v : v);
                A[k] *= a;
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
            for (int q = 0; q < kMaxWaves; ++q) {
                const float2 m = sh[REVERSE ? kMaxWaves - 1 - q : q][k][lane];
                h = fmaf(m.x, h, m.y);
                a *= m.x;
            }
            maps[(int64_t)seg * g.B * g.D + p.c + k] = make_float2(a, h);
        }
    }
}

// c: the first state c carried through the maps of `count` segments, from
// segment `from` on in direction `step`.  Each of the nw waves composes a part
// of them, all its loads in flight at once, and the parts meet in LDS.
template <int CPL>
__device__ __forceinline__ void carry_to_segment(float (&c)[CPL], const float2* __restrict__ maps, int64_t chans,
                                                 int64_t at, int from, int count, int step,
                                                 float2 (*sh)[CPL][kWave], int lane, int w, int nw)
{
    if (count == 0) return;
    float A[CPL], H[CPL];
#pragma unroll
    for (int k = 0; k < CPL; ++k) A[k] = 1.0f, H[k] = 0.0f;
    const int q1 = count * (w + 1) / nw;
#pragma unroll 8
    for (int q = count * w / nw; q < q1; ++q) {
        const float2* m = maps + (int64_t)(from + q * step) * chans + at;
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
            H[k] = fmaf(m[k].x, H[k], m[k].y);
            A[k] *= m[k].x;
        }
    }
#pragma unroll
    for (int k = 0; k < CPL; ++k) sh[w][k][lane] = make_float2(A[k], H[k]);
    __syncthreads();
    for (int q = 0; q < nw; ++q)
#pragma unroll
        for (int k = 0; k < CPL; ++k) c[k] = fmaf(sh[q][k][lane].x, c[k], sh[q][k][lane].y);
    __syncthreads();
}

// A workgroup walks its column of channels through its segment.  Bound by
// memory, with the vector units busy for two thirds of the time (33
// instructions an element, two of them at a fraction of the rate: the
// exponential and the reciprocal of the gate): 128 x 1000 x 512 bf16 83 us,
// 393 MB at 4.7 TB/s; second half of 65521 x 512 bf16 43 us, 201 MB.
template <typename E, int CPL, bool COUPLED>
__global__ __launch_bounds__(kMaxWaves* kWave) void k_scan(const E* __restrict__ x, const E* __restrict__ f,
                                                           const int32_t* __restrict__ length,
                                                           const float* __restrict__ h_first, Geometry g,
                                                           const float2* __restrict__ maps, E* __restrict__ h_out,
                                                           float* __restrict__ h_last, float* __restrict__ marks)
{
    constexpr int TS = kTS;
    __shared__ float2 sh[2][kMaxWaves][CPL][kWave];
    const int lane = threadIdx.x & 63, w = wave_index(), nw = blockDim.x >> 6;
    int column, seg;
    work_item(g, column, seg);
    const int tile = nw * TS;
    const int t0 = seg * g.seg_len, t1 = min(t0 + g.seg_len, g.T);
    const Place p = place_of<CPL>(g, length, column, lane);
    E* out = h_out ? h_out + (int64_t)p.b * g.T * g.D + p.d : nullptr;
    const int nm = (g.T + LIF_GATED_MARK - 1) / LIF_GATED_MARK;
    float* mk = marks ? marks + (int64_t)p.b * nm * g.D + p.d : nullptr;

    Raw<E, CPL, TS, 2> cur, nxt;
    auto load = [&](Raw<E, CPL, TS, 2>& r, int t) {
        load_steps<E, CPL, TS>(r.v[0], f + p.b * g.f_batch + p.d, g.f_time, t, p, INFINITY);
        load_steps<E, CPL, TS>(r.v[1], x + p.b * g.x_batch + p.d, g.x_time, t, p, 0.0f);
    };
    load(cur, t0 + w * TS);

    float c[CPL];                       // the state carried into the tile, the same in every wave
#pragma unroll
    for (int k = 0; k < CPL; ++k) c[k] = h_first ? h_first[p.c + k] : 0.0f;
    carry_to_segment<CPL>(c, maps, (int64_t)g.B * g.D, p.c, 0, seg, 1, sh[0], lane, w, nw);

    int buf = 0;
    for (int tt = t0; tt < t1; tt += tile, buf ^= 1) {
        const int t = tt + w * TS;
        float a[TS][CPL], u[TS][CPL], in[CPL];
        if (tt < p.n_max) {
            if (tt + tile < t1) load(nxt, t + tile);
            float A[CPL], H[CPL];
            compose_steps<E, CPL, TS, COUPLED>(cur, a, u, A, H);
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
                for (int i = 0; i < TS; ++i) a[i][k] = 1.0f, u[i][k] = 0.0f;
            }
        }
        run_steps<E, CPL, TS>(in, a, u, t, p, g, out, mk);
        cur = nxt;
    }
    if (h_last && seg == g.S - 1 && w == 0 && p.live) store_elems<float, CPL>(h_last + p.c, c);
}

// Backward, a wave's TS steps: the gates, the composed map of h (A, H) and of
// mu (A, M; the products are the same).
template <typename E, int CPL, int TS, bool COUPLED>
__device__ __forceinline__ void compose_back(const Raw<E, CPL, TS, 3>& r, float (&a)[TS][CPL], float (&na)[TS][CPL],
                                             float (&A)[CPL], float (&H)[CPL], float (&M)[CPL])
{
#pragma unroll
    for (int k = 0; k < CPL; ++k) A[k] = 1.0f, H[k] = 0.0f, M[k] = 0.0f;
#pragma unroll
    for (int i = 0; i < TS; ++i)
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
            gate(to_f32(r.v[0][i][k]), a[i][k], na[i][k]);
            const float v = to_f32(r.v[1][i][k]);
            H[k] = fmaf(a[i][k], H[k], COUPLED ? na[i][k] * v : v);
            A[k] *= a[i][k];
        }
#pragma unroll
    for (int i = TS - 1; i >= 0; --i)
#pragma unroll
        for (int k = 0; k < CPL; ++k) M[k] = a[i][k] * (M[k] + to_f32(r.v[2][i][k]));
}

// Runs a wave's steps from the entering state h upwards and from the adjoint
// lam (mu of the last step) downwards, and stores the gradients.
template <typename E, int CPL, int TS, bool COUPLED>
__device__ __forceinline__ void run_back(const Raw<E, CPL, TS, 3>& r, float (&h)[CPL], float (&lam)[CPL],
                                         const float (&a)[TS][CPL], const float (&na)[TS][CPL], int t, const Place& p,
                                         const Geometry& g, E* __restrict__ grad_x, E* __restrict__ grad_f)
{
    float df[TS][CPL];                  // d h_t / d f_t
#pragma unroll
    for (int i = 0; i < TS; ++i)
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
            const float v = to_f32(r.v[1][i][k]);
            df[i][k] = (COUPLED ? h[k] - v : h[k]) * (a[i][k] * na[i][k]);
            h[k] = fmaf(a[i][k], h[k], COUPLED ? na[i][k] * v : v);
        }
    if (!p.live) return;
    const int64_t row = fresh(g.D);
    const int64_t last = ((int64_t)p.b * g.T + t + TS - 1) * row + p.d;
    E *to_x = grad_x + last, *to_f = grad_f + last;
    const bool full = t + TS <= p.n_min;
#pragma unroll
    for (int i = TS - 1; i >= 0; --i, to_x -= row, to_f -= row) {
        E ox[CPL], of[CPL];
#pragma unroll
        for (int k = 0; k < CPL; ++k) {
            lam[k] += to_f32(r.v[2][i][k]);
            ox[k] = from_f32<E>(COUPLED ? lam[k] * na[i][k] : lam[k]);
            of[k] = from_f32<E>(lam[k] * df[i][k]);
            lam[k] *= a[i][k];
        }
        if (!full) {
            if (t + i >= g.T) continue;
#pragma unroll
            for (int k = 0; k < CPL; ++k) {
                ox[k] = t + i < p.n ? ox[k] : from_f32<E>(0.0f);
                of[k] = t + i < p.n ? of[k] : from_f32<E>(0.0f);
            }
        }
        store_elems<E, CPL>(to_x, ox);
        store_elems<E, CPL>(to_f, of);
    }
}

// The three inputs of a backward tile.
template <typename E, int CPL, int TS>
__device__ __forceinline__ void load_back(Raw<E, CPL, TS, 3>& r, const E* f, const E* x, const E* gh,
                                          const Geometry& g, int t, const Place& p)
{
    load_steps<E, CPL, TS>(r.v[0], f + p.b * g.f_batch + p.d, g.f_time, t, p, INFINITY);
    load_steps<E, CPL, TS>(r.v[1], x + p.b * g.x_batch + p.d, g.x_time, t, p, 0.0f);
    load_input<E, CPL, TS>(r.v[2], gh, p.b * g.g_batch + p.d, g.g_time, t, p);
}

// Backward: tiles of LIF_GATED_MARK steps of the segment from the last to the
// first.  The states of a tile are recomputed from its mark, so h is not read;
// both directions' maps meet in the same LDS exchange.  128 x 1000 x 512 bf16
// 145 us, 655 MB at 4.5 TB/s, with the vector units busy for 60 %.
template <typename E, int CPL, bool COUPLED>
__global__ __launch_bounds__(kMaxWaves* kWave) void k_back(const E* __restrict__ x, const E* __restrict__ f,
                                                           const int32_t* __restrict__ length,
                                                           const float* __restrict__ marks,
                                                           const E* __restrict__ grad_h,
                                                           const float* __restrict__ grad_last, Geometry g,
                                                           const float2* __restrict__ maps, E* __restrict__ grad_x,
                                                           E* __restrict__ grad_f, float* __restrict__ grad_first)
{
    constexpr int TS = kTS, tile = LIF_GATED_MARK;
    __shared__ float sh[2][kMaxWaves][CPL][3][kWave];
    __shared__ float2 sh_maps[kMaxWaves][CPL][kWave];
    const int lane = threadIdx.x & 63, w = wave_index();
    int column, seg;
    work_item(g, column, seg);
    const int t0 = seg * g.seg_len, t1 = min(t0 + g.seg_len, g.T);
    const Place p = place_of<CPL>(g, length, column, lane);
    const int nm = (g.T + LIF_GATED_MARK - 1) / LIF_GATED_MARK;
    const float* mk = marks + (int64_t)p.b * nm * g.D + p.d;

    Raw<E, CPL, TS, 3> cur, nxt;
    float h_cur[CPL], h_nxt[CPL];
    auto load = [&](Raw<E, CPL, TS, 3>& r, float (&h)[CPL], int tt) {
        load_back<E, CPL, TS>(r, f, x, grad_h, g, tt + w * TS, p);
        load_elems<float, CPL>(mk + (int64_t)(tt / LIF_GATED_MARK) * g.D, h);
    };
    int tt = t0 + (t1 - t0 + tile - 1) / tile * tile - tile;
    if (tt >= t0) load(cur, h_cur, tt);

    float mu[CPL];                      // the adjoint carried into the tile from the later side
#pragma unroll
    for (int k = 0; k < CPL; ++k) mu[k] = grad_last ? grad_last[p.c + k] : 0.0f;
    carry_to_segment<CPL>(mu, maps, (int64_t)g.B * g.D, p.c, g.S - 1, g.S - 1 - seg, -1, sh_maps, lane, w, kMaxWaves);

    int buf = 0;
    for (; tt >= t0; tt -= tile, buf ^= 1) {
        const int t = tt + w * TS;
        if (tt > t0) load(nxt, h_nxt, tt - tile);
        if (tt >= p.n_max) {            // past every lane's length
            const int64_t row = ((int64_t)p.b * g.T + t) * g.D + p.d;
            E o[CPL];
#pragma unroll
            for (int k = 0; k < CPL; ++k) o[k] = from_f32<E>(0.0f);
            if (p.live)
#pragma unroll
                for (int i = 0; i < TS; ++i)
                    if (t + i < g.T) {
                        store_elems<E, CPL>(grad_x + row + (int64_t)i * g.D, o);
                        store_elems<E, CPL>(grad_f + row + (int64_t)i * g.D, o);
                    }
        } else {
            float a[TS][CPL], na[TS][CPL], A[CPL], H[CPL], M[CPL], h[CPL], lam[CPL];
            compose_back<E, CPL, TS, COUPLED>(cur, a, na, A, H, M);
#pragma unroll
            for (int k = 0; k < CPL; ++k) {
                sh[buf][w][k][0][lane] = A[k];
                sh[buf][w][k][1][lane] = H[k];
                sh[buf][w][k][2][lane] = M[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < CPL; ++k) {
                h[k] = h_cur[k];
                for (int q = 0; q < w; ++q) h[k] = fmaf(sh[buf][q][k][0][lane], h[k], sh[buf][q][k][1][lane]);
                for (int q = kMaxWaves - 1; q >= 0; --q) {
                    if (q == w) lam[k] = mu[k];
                    mu[k] = fmaf(sh[buf][q][k][0][lane], mu[k], sh[buf][q][k][2][lane]);
                }
            }
            run_back<E, CPL, TS, COUPLED>(cur, h, lam, a, na, t, p, g, grad_x, grad_f);
        }
        cur = nxt;
#pragma unroll
        for (int k = 0; k < CPL; ++k) h_cur[k] = h_nxt[k];
    }
    if (grad_first && seg == 0 && w == 0 && p.live) store_elems<float, CPL>(grad_first + p.c, mu);
}

// One step of every stream: one lane per CPL channels, nothing to share.  Its
// time is the launch's for one stream (2 us), the memory's for many (256 x
// 4096 f32 5 us, 21 MB at 4.2 TB/s).
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
    // a launch has fewer than 2^32 threads, and steps are counted in 32 bits
    if ((int64_t)p->B * p->D >= ((int64_t)1 << 28) || p->T > (1 << 30)) return LIF_ERR_SIZE;
    if ((int64_t)p->B * p->D * p->T >= ((int64_t)1 << 48)) return LIF_ERR_SIZE;
    return LIF_OK;
}

// The way a call takes: channels per lane and segments of the time axis.
struct Plan {
    int cpl;
    Geometry g;
};

Plan plan_of(const lif_gated_params& p, bool back)
{
    Plan q;
    const int64_t elem = p.dtype == LIF_F32 ? 4 : 2;
    auto groups = [&](int cpl) { return (int64_t)p.B * ((p.D + cpl - 1) / cpl); };
    auto columns = [&](int cpl) { return (int)((groups(cpl) + kWave - 1) / kWave); };
    const int blocks = (p.T + LIF_GATED_MARK - 1) / LIF_GATED_MARK;
    const bool split = blocks >= kSplitMin && p.B * (int64_t)p.D * elem < kSplitBytes * (blocks < 16 ? blocks : 16) / 16;
    // The widest group that leaves enough workgroups: four channels take 136
    // registers, so they pay from two workgroups per CU on (128 x 1000 x 512
    // bf16, ragged, 256 columns: 74 us, 66 with two channels); two 16-bit
    // channels fill a 4-byte load (157 columns: 114 us, 126 with one); two
    // float32 ones from 256 columns on (76 us, 81 with one; at 192 columns 102
    // and 95).  Where the time axis is shared out, two channels if that still
    // gives all workgroups (65521 x 512 bf16: 76 us, 85 with one).  Backward
    // always one: two halve the waves (60000 x 512 67 -> 82, 128 x 1000 x 512
    // 145 -> 151 us).
    q.cpl = back ? 1 : elem == 4 ? 2 : 4;
    auto fits = [&](int cpl) {
        if (p.D < cpl) return false;
        if (split) return cpl == 2 && (int64_t)columns(2) * (blocks / kSplitBlocks) >= kSplitGroups;
        return columns(cpl) >= (cpl == 4 ? 512 : elem == 4 ? 256 : 150);
    };
    while (q.cpl > 1 && !fits(q.cpl)) q.cpl >>= 1;
    q.g.columns = columns(q.cpl);
    int S = 1;
    if (split) {
        S = (kSplitGroups + q.g.columns - 1) / q.g.columns;
        if (S > blocks / kSplitBlocks) S = blocks / kSplitBlocks;
    }
    const int per = blocks > 0 ? (blocks + S - 1) / S : 1;
    Geometry& g = q.g;
    g.seg_len = per * LIF_GATED_MARK;
    g.S = blocks > 0 ? (blocks + per - 1) / per : 1;
    g.B = p.B;
    g.T = p.T;
    g.D = p.D;
    g.groups = (int)groups(q.cpl);
    g.per_sample = (p.D + q.cpl - 1) / q.cpl;
    g.shared_lines = p.D * elem % 128 != 0;
    g.x_batch = p.x_batch;
    g.x_time = p.x_time;
    g.f_batch = p.f_batch;
    g.f_time = p.f_time;
    g.g_batch = p.g_batch;
    g.g_time = p.g_time;
    return q;
}

size_t maps_size(const Plan& q) { return q.g.S > 1 ? (size_t)q.g.S * q.g.B * q.g.D * sizeof(float2) : 0; }

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
    using namespace lif;
    if (check_gated(p) != LIF_OK) return 0;
    const size_t a = maps_size(plan_of(*p, false)), b = maps_size(plan_of(*p, true));
    return a > b ? a : b;
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
    if (need > 0 && (!ws || (uintptr_t)ws % sizeof(float2))) return LIF_ERR_ARG;
    if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    if (chans == 0) return LIF_OK;
    const Plan q = plan_of(*p, false);
    const hipStream_t s = (hipStream_t)stream;
    int nw = 1;                          // no more waves than the sequence has groups of TS steps
    while (nw < kMaxWaves && nw * kTS < p->T) nw *= 2;
    dispatch(q, *p, [&](auto e, auto cpl, auto coupled) {
        using E = decltype(e);
        constexpr int C = decltype(cpl)::value;
        constexpr bool K = decltype(coupled)::value;
        if (q.g.S > 1)
            TIMED_LAUNCH("gated_maps", (k_segment_maps<E, C, K, false>), dim3(q.g.columns * (q.g.S - 1)),
                         dim3(kMaxWaves * kWave), 0, s, (const E*)x, (const E*)f, length, q.g, (float2*)ws);
        TIMED_LAUNCH("gated_scan", (k_scan<E, C, K>), dim3(q.g.columns * q.g.S), dim3(nw * kWave), 0, s, (const E*)x,
                     (const E*)f, length, h_first, q.g, (const float2*)ws, (E*)h, h_last, marks);
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
    if (need > 0 && (!ws || (uintptr_t)ws % sizeof(float2))) return LIF_ERR_ARG;
    if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    if (chans == 0) return LIF_OK;
    const Plan q = plan_of(*p, true);
    const hipStream_t s = (hipStream_t)stream;
    dispatch(q, *p, [&](auto e, auto cpl, auto coupled) {
        using E = decltype(e);
        constexpr int C = decltype(cpl)::value;
        constexpr bool K = decltype(coupled)::value;
        if constexpr (C == 1) {
            if (q.g.S > 1)
                TIMED_LAUNCH("gated_maps_back", (k_segment_maps<E, C, K, true>), dim3(q.g.columns * (q.g.S - 1)),
                             dim3(kMaxWaves * kWave), 0, s, (const E*)grad_h, (const E*)f, length, q.g, (float2*)ws);
            TIMED_LAUNCH("gated_back", (k_back<E, C, K>), dim3(q.g.columns * q.g.S), dim3(kMaxWaves * kWave), 0, s,
                         (const E*)x, (const E*)f, length, marks, (const E*)grad_h, grad_last, q.g, (const float2*)ws,
                         (E*)grad_x, (E*)grad_f, grad_h_first);
        }
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
    // Four channels per lane where a row divides by them and every CU still has
    // a workgroup: 256 x 4096 f32 7.5 -> 6.3 us, 512 x 8192 bf16 17.1 -> 12.5 (in
    // graphs); at 256 x 1024 and below either form takes the launch's 5 us.
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
